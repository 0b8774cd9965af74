// Filter gradient of a fully connected layer from inputs held in blocks of 8 bits:
//   dw[o][i] = sum_n dy[n][o] x[n][i],   x[n][i] = code 2^e
// Part of block_ops.hip: included there, inside its anonymous namespace, after block_formats.h.
//
// An E4M3 number times a power of two has four significant bits: it is a bfloat16 number as it is, and the product runs on
// v_mfma_f32_32x32x16_bf16.  fp32 gradients go in as three bfloat16 parts of eight bits each, cut off one after the other, which
// hold them exactly (from 2^-110 on; bfloat16 ends at 2^-133): three products instead of one, and no error but that of the sums.
//
// Both operands lie in memory with the sum's index n outermost.  They are staged in LDS as they lie, rows of n, and read
// transposed (ds_read_b64_tr_b16: 16 lanes read a block of 4 n x 16 columns and get a column of it each).  A row of 128 values is
// 256 bytes and 64 more, so that the four rows of such a block, and the two blocks that 32 lanes read, lie in different banks.
struct KeptGradArgs {
    const unsigned char *codes, *scales;
    const void *dy;
    float *dw;                   // [O][I], or one such for every split
    int64_t pitch, dy_stride;
    int N, I, O;
    int itiles, otiles, splits, rows_per_split;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kGradTile = 128, kGradStep = 32, kGradPitch = kGradTile * 2 + 64;     // bytes of a staged row

// 16 codes with their exponent as bfloat16
__device__ __forceinline__ void kept_to_bf16(const u32x4 &w, unsigned byte, u32x4 (&out)[2])
{
    const float scale = block_scale(byte);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int q = byte == 255 ? 0x7F7F7F7F : (int)w[k];                  // a block that holds no numbers
        out[k >> 1][2 * (k & 1)] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, false));
        out[k >> 1][2 * (k & 1) + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, true));
    }
}

// the three parts of eight fp32 values, their upper halves cut off; an infinity has one part
__device__ __forceinline__ void three_parts(const float (&v)[8], u32x4 (&part)[3])
{
    unsigned u[3][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        u[0][k] = __float_as_uint(v[k]) & 0xFFFF0000u;
        float rest = v[k] - __uint_as_float(u[0][k]);
        rest = fabsf(v[k]) == INFINITY ? 0.f : rest;
        u[1][k] = __float_as_uint(rest) & 0xFFFF0000u;
        u[2][k] = __float_as_uint(rest - __uint_as_float(u[1][k]));
    }
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k) part[p][k] = __builtin_amdgcn_perm(u[p][2 * k + 1], u[p][2 * k], 0x07060302u);
}

__device__ __forceinline__ bf16x8 read_transposed(const char *p, int pitch)          // k 0..3 from p, 4..7 four rows on
{
    typedef __attribute__((address_space(3))) s16x4 *Lds;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * pitch));
    const __attribute__((ext_vector_type(8))) short r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, r);
}

template <typename T>
__global__ __launch_bounds__(256) void fc_grad_kept_kernel(const KeptGradArgs a)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int BYTES = kGradStep * kGradPitch;
    __shared__ __attribute__((aligned(16))) char lds[(PARTS + 1) * BYTES];
    char *const xs = lds, *const ds = lds + BYTES;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int tiles = a.itiles * a.otiles;
    const int split = blockIdx.x / tiles, tile = blockIdx.x - split * tiles;
    const int ot = tile / a.itiles, it = tile - ot * a.itiles;
    const int o0 = ot * kGradTile, i0 = it * kGradTile;
    const int wo = (wave >> 1) * 64, wi = (wave & 1) * 64;
    const int begin = split * a.rows_per_split, end = min(a.N, begin + a.rows_per_split);

    f32x16 acc[2][2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[p][q][v] = 0.f;

    const int row = tid >> 3, col = (tid & 7) * 16;
    // of a fragment: lane's row of n within 8, its 4 columns of 32
    const int fr = (lane >> 5) * 8 + ((lane & 15) >> 2), fc = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    for (int n0 = begin; n0 < end; n0 += kGradStep) {
        const int n = n0 + row;
        u32x4 w = {0u, 0u, 0u, 0u}, xv[2];
        unsigned byte = 127;
        if (n < end) {
            const int64_t at = (int64_t)n * a.pitch + i0 + col;
            w = *reinterpret_cast<const u32x4 *>(a.codes + at);
            byte = a.scales[at / kBlock];
        }
        kept_to_bf16(w, byte, xv);
        float d[2][8];
        const T *const dy = static_cast<const T *>(a.dy) + (int64_t)n * a.dy_stride + o0 + col;
#pragma unroll
        for (int h = 0; h < 2; ++h) load8(dy + 8 * h, n < end ? max(0, a.O - o0 - col - 8 * h) : 0, d[h]);
        __syncthreads();
        char *const at = xs + row * kGradPitch + col * 2, *const dat = ds + row * kGradPitch + col * 2;
        *reinterpret_cast<u32x4 *>(at) = xv[0];
        *reinterpret_cast<u32x4 *>(at + 16) = xv[1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (PARTS == 3) {
                u32x4 part[3];
                three_parts(d[h], part);
#pragma unroll
                for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4 *>(dat + p * BYTES + 16 * h) = part[p];
            } else {
                Vec<unsigned short>::store(reinterpret_cast<unsigned short *>(dat + 16 * h), d[h]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kGradStep; s += 16) {
            const char *const xf = xs + (s + fr) * kGradPitch + (wi + fc) * 2, *const df = ds + (s + fr) * kGradPitch + (wo + fc) * 2;
            bf16x8 xq[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) xq[q] = read_transposed(xf + q * 64, kGradPitch);
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)                             // the small parts first
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const bf16x8 dq = read_transposed(df + p * BYTES + m * 64, kGradPitch);
#pragma unroll
                    for (int q = 0; q < 2; ++q) acc[m][q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dq, xq[q], acc[m][q], 0, 0, 0);
                }
        }
    }
    float *const dw = a.dw + (int64_t)split * a.O * a.I;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int o = o0 + wo + m * 32 + (lane >> 5) * 4 + (v >> 2) * 8 + (v & 3), i = i0 + wi + q * 32 + (lane & 31);
                if (o < a.O && i < a.I) dw[(int64_t)o * a.I + i] = acc[m][q][v];
            }
}

// the splits' sums, one after the other
__global__ __launch_bounds__(256) void fc_grad_join(const float *part, float *dw, int64_t count, int splits)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float s = part[i];
    for (int p = 1; p < splits; ++p) s += part[p * count + i];
    dw[i] = s;
}
