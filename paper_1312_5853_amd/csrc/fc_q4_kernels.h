// Forward pass of a fully connected layer with both operands in blocks of 4 bits:
//   y[n][o] = f(sum_i x[n][i] w[o][i] + bias[o]),  x and w E2M1 numbers times a power of two for every 32 of i
// Part of block_ops.hip: included there, inside its anonymous namespace, after block_formats.h.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies them as they are: a lane holds 32 neighbouring values of a row (16 bytes), and
// the byte of their exponent.  Rows are filled up to 128 values, so a step of the sum is one 64-byte piece and one 4-byte word
// of exponents of every row.  w is the first operand: a lane then has four neighbouring outputs of one sample.
struct Q4Args {
    const unsigned char *xc, *xs, *wc, *ws;      // codes, exponents
    const float *bias;
    void *y;
    int N, I, O, steps;                          // steps of 128
    int relu;
    int ntiles, otiles;
};

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma_q4(const i32x4 &w, const i32x4 &x, const f32x4 &c, unsigned ws, unsigned xs)
{
    const i32x8 a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)ws, 0, (int)xs);
}

// four neighbouring outputs of sample n
template <typename T>
__device__ __forceinline__ void store_q4(const Q4Args &a, int n, int o, const f32x4 &s)
{
    if (n >= a.N) return;
    T *const y = static_cast<T *>(a.y) + (int64_t)n * a.O;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (o + k < a.O) {
            float v = s[k] + (a.bias ? a.bias[o + k] : 0.f);
            if (a.relu) v = v > 0.f ? v : (v != v ? v : 0.f);
            st_elem(y, o + k, v);
        }
}

// 128 x 128 outputs to a work-group, 64 x 64 to a wavefront, operands straight from memory
template <typename T>
__global__ __launch_bounds__(256) void fc_q4_tiles(const Q4Args a)
{
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int nt = blockIdx.x % a.ntiles, ot = blockIdx.x / a.ntiles;
    const int n0 = nt * 128 + (wave & 1) * 64, o0 = ot * 128 + (wave >> 1) * 64;
    const int r = lane & 15, g = lane >> 4;
    const int64_t cpitch = (int64_t)a.steps * 64, spitch = (int64_t)a.steps * 4;
    const unsigned char *xc[4], *wc[4], *xs[4], *ws[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {                // rows past the end read the last one; their sums are not stored
        const int64_t n = min(n0 + k * 16 + r, a.N - 1), o = min(o0 + k * 16 + r, a.O - 1);
        xc[k] = a.xc + n * cpitch + g * 16; wc[k] = a.wc + o * cpitch + g * 16;
        xs[k] = a.xs + n * spitch + g; ws[k] = a.ws + o * spitch + g;
    }
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.steps; ++s) {
        i32x4 x[4], w[4];
        unsigned sx[4], sw[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] = *reinterpret_cast<const i32x4 *>(xc[k] + (int64_t)s * 64);
            w[k] = *reinterpret_cast<const i32x4 *>(wc[k] + (int64_t)s * 64);
            sx[k] = xs[k][(int64_t)s * 4];
            sw[k] = ws[k][(int64_t)s * 4];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma_q4(w[i], x[j], acc[i][j], sw[i], sx[j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) store_q4<T>(a, n0 + j * 16 + r, o0 + i * 16 + g * 4, acc[i][j]);
}
