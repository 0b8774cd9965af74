// Element access that the kernels of both translation units share: fp32 tensors, or bfloat16 tensors (as their bits) read
// exactly and written rounded to nearest even.  Included inside an anonymous namespace; not a stand-alone header.

// fp32 -> bfloat16 bits, round to nearest even; NaN stays a (quiet) NaN
__device__ __forceinline__ unsigned short bf16_round(float f)
{
    const unsigned u = __float_as_uint(f);
    unsigned r = (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) r = (u >> 16) | 0x40u;
    return (unsigned short)r;
}

__device__ __forceinline__ float ld_elem(const float *p, int64_t i) { return p[i]; }
__device__ __forceinline__ float ld_elem(const unsigned short *p, int64_t i)
{
    return __uint_as_float((unsigned)p[i] << 16);
}
__device__ __forceinline__ void st_elem(float *p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st_elem(unsigned short *p, int64_t i, float v) { p[i] = bf16_round(v); }
