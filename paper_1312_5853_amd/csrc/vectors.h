// 16-byte vectors of the row kernels (4 fp32 or 8 bfloat16 values) at any element's address, and sums and maxima over a
// wavefront.  Included inside an anonymous namespace after elements.h; not a stand-alone header.

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <typename T>
struct Vec;

template <>
struct Vec<float> {
    static constexpr int V = 4;
    typedef f32x4 Raw;
    static __device__ __forceinline__ Raw load(const float *p) { return *reinterpret_cast<const f32x4_any *>(p); }
    static __device__ __forceinline__ void store(float *p, const float (&v)[4])
    {
        *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0], v[1], v[2], v[3]};
    }
    static __device__ __forceinline__ void put(float *p, int i, float v) { p[i] = v; }
    static __device__ __forceinline__ void open(const Raw &r, float (&v)[4])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = r[k];
    }
    static __device__ __forceinline__ void drop(Raw &r, int k0, int k1)      // -infinity in place of values before k0, from k1 on
    {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < k0 || k >= k1) r[k] = -INFINITY;
    }
    static __device__ __forceinline__ Raw some(const float *p, int n)        // the first n values, zeros after them
    {
        Raw r = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < 4; ++k)
            if (k < n) r[k] = p[k];
        return r;
    }
    static __device__ __forceinline__ Raw ends(const float *p, int n)        // the values from the n-th on, zeros before them
    {
        Raw r = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < 4; ++k)
            if (k >= n) r[k] = p[k];
        return r;
    }
    static __device__ __forceinline__ void clear_first(Raw &r, int n)        // zeros in place of the first n values, n < V
    {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < n) r[k] = 0.f;
    }
};

template <>
struct Vec<unsigned short> {
    static constexpr int V = 8;
    typedef u32x4 Raw;
    static __device__ __forceinline__ Raw load(const unsigned short *p)
    {
        return *reinterpret_cast<const u32x4_any *>(p);
    }
    static __device__ __forceinline__ void store(unsigned short *p, const float (&v)[8])
    {
        u32x4 q;
#pragma unroll
        for (int k = 0; k < 4; ++k)          // both at once, to nearest even (v_cvt_pk_bf16_f32)
            q[k] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){v[2 * k], v[2 * k + 1]}, bf16x2));
        *reinterpret_cast<u32x4_any *>(p) = q;
    }
    static __device__ __forceinline__ void put(unsigned short *p, int i, float v)
    {
        p[i] = __builtin_bit_cast(unsigned short, (__bf16)v);
    }
    static __device__ __forceinline__ void open(const Raw &r, float (&v)[8])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(r[k] << 16);
            v[2 * k + 1] = __uint_as_float(r[k] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void drop(Raw &r, int k0, int k1)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (2 * k < k0 || 2 * k >= k1) r[k] = (r[k] & 0xFFFF0000u) | 0xFF80u;
            if (2 * k + 1 < k0 || 2 * k + 1 >= k1) r[k] = (r[k] & 0xFFFFu) | 0xFF800000u;
        }
    }
    static __device__ __forceinline__ Raw some(const unsigned short *p, int n)
    {
        Raw r = {0u, 0u, 0u, 0u};
        for (int k = 0; k < 8; ++k)
            if (k < n) r[k >> 1] |= (unsigned)p[k] << (16 * (k & 1));
        return r;
    }
    static __device__ __forceinline__ Raw ends(const unsigned short *p, int n)
    {
        Raw r = {0u, 0u, 0u, 0u};
        for (int k = 0; k < 8; ++k)
            if (k >= n) r[k >> 1] |= (unsigned)p[k] << (16 * (k & 1));
        return r;
    }
    static __device__ __forceinline__ void clear_first(Raw &r, int n)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (2 * k + 1 < n) r[k] = 0u;
            else if (2 * k < n) r[k] &= 0xFFFF0000u;
        }
    }
};

// Makes the compiler take vectors for new ones.  It would else keep values that it has opened for one use, bfloat16 ones
// in twice the registers, for the next, and spill; opening them again is one instruction.
template <typename Raw, int R>
__device__ __forceinline__ void open_again(Raw (&raw)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) asm volatile("" : "+v"(raw[r]));
}

// In a branch that few wavefronts take: keeps it one.  The compiler would else compute both sides and select (1024 x 64 planes
// of 16 fp32 in 64 groups, none of which needs the branch: 16.1 us, and 15.1).
__device__ __forceinline__ void as_branch() { asm volatile(""); }

// Sum and maximum over the 64 lanes, the same in every lane: within the rows of 16 lanes by data-parallel-primitive
// moves, then the four row results by scalar reads.
__device__ __forceinline__ float max3(float a, float b, float c)          // the largest; a NaN is passed over
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

template <int CTRL>
__device__ __forceinline__ float dpp_move(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp_move<0xB1>(v);                  // lane ^ 1
    v += dpp_move<0x4E>(v);                  // lane ^ 2
    v += dpp_move<0x141>(v);                 // mirrored within 8
    v += dpp_move<0x140>(v);                 // mirrored within 16
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    v = fmaxf(v, dpp_move<0x140>(v));
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
template <int CTRL>
__device__ __forceinline__ double dpp_move(double v)
{
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, false),
                            __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ double lane_value(double v, int lane)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                            __builtin_amdgcn_readlane(__double2loint(v), lane));
}
__device__ __forceinline__ double wave_sum(double v)
{
    v += dpp_move<0xB1>(v);
    v += dpp_move<0x4E>(v);
    v += dpp_move<0x141>(v);
    v += dpp_move<0x140>(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
// sum over the aligned runs of `width` lanes (a power of two), the same in every lane of a run
__device__ __forceinline__ float run_sum(float v, int width)
{
    if (width > 1) v += dpp_move<0xB1>(v);
    if (width > 2) v += dpp_move<0x4E>(v);
    if (width > 4) v += dpp_move<0x141>(v);
    if (width > 8) v += dpp_move<0x140>(v);
    for (int o = 16; o < width; o <<= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
