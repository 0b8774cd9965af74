// Tensors held in blocks: 32 neighbouring values of a row share a power of two, each is an E4M3 (8 bits) or E2M1 (4 bits)
// number times it.  Reading codes, 4 or 8 values at a time, and the exponent's byte.  Included inside an anonymous namespace
// after vectors.h; not a stand-alone header.

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 32;          // values to an exponent
constexpr int kE4M3 = CONV_BLOCKS_E4M3, kE2M1 = CONV_BLOCKS_E2M1;

// largest magnitude (mantissa bits of its fp32 form, exponent) and the least exponent of a block: from there on every value
// read back is a normal number of fp32 and bfloat16 (2^-9 2^-117 and 2^-1 2^-125 are 2^-126), which all units take as it is
template <int FORM>
struct BlockFormat;
template <>
struct BlockFormat<kE4M3> {
    static constexpr unsigned kTopMantissa = 0x600000u;      // 448 = 1.75 2^8
    static constexpr int kTopExponent = 8, kLeast = -117;
};
template <>
struct BlockFormat<kE2M1> {
    static constexpr unsigned kTopMantissa = 0x400000u;      // 6 = 1.5 2^2
    static constexpr int kTopExponent = 2, kLeast = -125;
};

// Byte of the smallest allowed exponent under which a block's largest magnitude (its bits) is within the format; 255 where the
// block holds an infinity or a NaN (whose bits are the larger ones).
template <int FORM>
__device__ __forceinline__ int block_exponent(unsigned largest)
{
    const int e = (int)(largest >> 23) - BlockFormat<FORM>::kTopExponent + ((largest & 0x7FFFFFu) > BlockFormat<FORM>::kTopMantissa);
    return largest >= 0x7F800000u ? 255 : max(e, BlockFormat<FORM>::kLeast + 127);
}

// 2^(byte - 127); infinity for 255, which makes a NaN of the zeros that such a block's codes are
__device__ __forceinline__ float block_scale(unsigned byte) { return __uint_as_float(byte << 23); }

// eight E4M3 values, as they are in memory
__device__ __forceinline__ void open_e4m3(unsigned word, float scale, float *v)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
    v[0] = a[0] * scale; v[1] = a[1] * scale; v[2] = b[0] * scale; v[3] = b[1] * scale;
}
