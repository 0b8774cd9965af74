// Values into blocks with a shared power of two, and back.  Part of block_ops.hip: included there, inside its anonymous
// namespace, after block_formats.h.
//
// A thread takes eight neighbouring values; four neighbouring lanes share a block, whose largest magnitude is a maximum of
// integers (the bits of magnitudes are ordered as they are, infinities and NaN above).  The codes' rows are whole blocks, so
// the values are gone through as one long row of eights.  Bound by memory: 4096 x 9216 fp32 into 4 bits 40 us, 4.3 TB/s, and back 28,
// 6.1 (what is written stays in the last cache for a while); one row of 70001 2.4 us each way, a launch.
struct BlockArgs {
    const void *in;              // values, or codes
    void *out;                   // codes, or values
    unsigned char *scales;
    int64_t stride;              // of the values' rows
    int64_t total;               // eights of all rows
    int per_row;                 // eights of a row of codes
    int C;
    FastDiv div;                 // by per_row
};

__device__ __forceinline__ void load8(const float *p, int n, float (&v)[8])
{
    const Vec<float>::Raw a = n >= 4 ? Vec<float>::load(p) : Vec<float>::some(p, n);
    const Vec<float>::Raw b = n >= 8 ? Vec<float>::load(p + 4) : Vec<float>::some(p + 4, n - 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[k] = a[k]; v[4 + k] = b[k]; }
}
__device__ __forceinline__ void load8(const unsigned short *p, int n, float (&v)[8])
{
    Vec<unsigned short>::open(n >= 8 ? Vec<unsigned short>::load(p) : Vec<unsigned short>::some(p, n), v);
}
__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8])
{
    if (n >= 8) {
        *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4_any *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) p[k] = v[k];
}
__device__ __forceinline__ void store8(unsigned short *p, int n, const float (&v)[8])
{
    if (n >= 8) { Vec<unsigned short>::store(p, v); return; }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) Vec<unsigned short>::put(p, k, v[k]);
}

// the maximum over the four lanes that share a block
__device__ __forceinline__ unsigned block_max(unsigned m)
{
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));     // lane ^ 1
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));  // lane ^ 2
}

// eight values of a block: the block's exponent byte, the codes in word
template <int FORM>
__device__ __forceinline__ int into_codes(const float (&v)[8], unsigned (&word)[2])
{
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(v[k]) & 0x7FFFFFFFu);
    const int byte = block_exponent<FORM>(block_max(m));
    const float inv = __uint_as_float((unsigned)(254 - byte) << 23);         // 2^-e, a normal number; not used for 255
    word[0] = word[1] = 0;
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = byte == 255 ? 0.f : v[k] * inv;       // a product with a power of two: exact, or far below
    if constexpr (FORM == kE4M3) {                                           // the least code
        int a = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false), b = __builtin_amdgcn_cvt_pk_fp8_f32(w[4], w[5], 0, false);
        word[0] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], a, true);
        word[1] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(w[6], w[7], b, true);
    } else {
        unsigned q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, w[0], w[1], 1.f, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, w[2], w[3], 1.f, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, w[4], w[5], 1.f, 2);
        word[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, w[6], w[7], 1.f, 3);
    }
    return byte;
}

template <typename T, int FORM>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const BlockArgs a)
{
    const int64_t base = (int64_t)blockIdx.x * 256;
    const int64_t row0 = base / a.per_row;
    const unsigned at = (unsigned)(base - row0 * a.per_row) + threadIdx.x;
    const unsigned down = fastdiv(at, a.div);
    const int64_t row = row0 + down;
    const int c = (int)(at - down * a.per_row) * 8;
    if (base + threadIdx.x >= a.total) return;                               // whole blocks of lanes: totals are multiples of 16
    float v[8];
    load8(static_cast<const T *>(a.in) + row * a.stride + c, a.C - c, v);
    unsigned word[2];
    const int byte = into_codes<FORM>(v, word);
    const int64_t i = base + threadIdx.x;
    if constexpr (FORM == kE4M3) static_cast<u32x2 *>(a.out)[i] = u32x2{word[0], word[1]};
    else static_cast<unsigned *>(a.out)[i] = word[0];
    if (threadIdx.x % 4 == 0) a.scales[i >> 2] = (unsigned char)byte;
}

template <typename T, int FORM>
__global__ __launch_bounds__(256) void dequantize_blocks_kernel(const BlockArgs a)
{
    const int64_t base = (int64_t)blockIdx.x * 256;
    const int64_t row0 = base / a.per_row;
    const unsigned at = (unsigned)(base - row0 * a.per_row) + threadIdx.x;
    const unsigned down = fastdiv(at, a.div);
    const int64_t row = row0 + down;
    const int c = (int)(at - down * a.per_row) * 8;
    const int64_t i = base + threadIdx.x;
    if (i >= a.total || c >= a.C) return;
    const float scale = block_scale(a.scales[i >> 2]);
    float v[8];
    if constexpr (FORM == kE4M3) {
        const u32x2 w = static_cast<const u32x2 *>(a.in)[i];
        open_e4m3(w[0], scale, v);
        open_e4m3(w[1], scale, v + 4);
    } else {
        const unsigned w = static_cast<const unsigned *>(a.in)[i];
        const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3)};
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = p[k >> 1][k & 1] * scale;
    }
    store8(static_cast<T *>(a.out) + row * a.stride + c, a.C - c, v);
}
