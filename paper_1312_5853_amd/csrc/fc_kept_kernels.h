// Filter gradient of a fully connected layer from inputs held in blocks of 8 bits:
//   dw[o][i] = sum_n dy[n][o] x[n][i],   x[n][i] = code 2^e
// Part of block_ops.hip: included there, inside its anonymous namespace, after block_formats.h.
//
// An E4M3 number times a power of two has four significant bits: it is a bfloat16 number as it is, and the product runs on
// v_mfma_f32_32x32x16_bf16.  fp32 gradients go in as three bfloat16 parts of eight bits each, cut off one after the other, which
// hold them exactly (from 2^-110 on; bfloat16 ends at 2^-133): three products instead of one, and no error but that of the sums.
//
// Both operands lie in memory with the sum's index n outermost.  They are staged in LDS as they lie, rows of n, and read
// transposed (ds_read_b64_tr_b16: 16 lanes read a block of 4 n x 16 columns and get a column of it each).  The 16-byte piece c of
// row n stands at place c ^ 4 (n % 4): the four rows of such a block, and the two blocks that 32 lanes read, lie in different banks.
//
// Tiles of 64 TM outputs x 64 TN inputs, a quarter to each of four wavefronts, KS rows of n to a step.  Two buffers: while a step is
// multiplied, the next one's values, which have come into registers meanwhile, are converted and stored piece by piece, and each
// piece of the step after it is sent for as its registers become free.
// Bound by the matrix units and the clock that their power leaves them: 8192 rows 4096 -> 4096 bfloat16 229 us from idle, up to 313
// between 2 and 8 ms of such calls, 217 to 231 from 15 ms on, 1190 to 1270 TFLOP/s (a library product of bfloat16 tensors 8192^3
// 1176 to 1200 in the same state).

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// A value read back from a block of this exponent may be infinite (448 2^119 is below 2^128, 256 2^120 is not); 255 holds no numbers.
__device__ __forceinline__ bool may_be_infinite(unsigned byte) { return byte - 247u < 8u; }

// Of fp32 gradients one infinite value times three parts is no number wherever a part is zero.  If input i has one in the samples begin
// .. end - 1, its sums again, product by product: those of a lane's 16 outputs of a block of 32 (see the kernels) from `first` on.
__device__ __forceinline__ void infinite_input(const KeptGradArgs &a, float *dw, int begin, int end, int i, int first)
{
    if (i >= a.I) return;
    auto value = [&](int n) {
        const int64_t at = (int64_t)n * a.pitch + i;
        return __builtin_amdgcn_cvt_f32_fp8((int)a.codes[at], 0) * block_scale(a.scales[at / kBlock]);
    };
    bool infinite = false;
#pragma unroll 1
    for (int n = begin; n < end; ++n) infinite |= fabsf(value(n)) == INFINITY;
    if (!infinite) return;
#pragma unroll 1
    for (int v = 0; v < 16; ++v) {
        const int o = first + (v >> 2) * 8 + (v & 3);
        if (o >= a.O) break;                         // (they ascend)
        double s = 0.0;
#pragma unroll 1
        for (int n = begin; n < end; ++n) s += (double)static_cast<const float *>(a.dy)[(int64_t)n * a.dy_stride + o] * value(n);
        dw[(int64_t)o * a.I + i] = (float)s;
    }
}

__device__ __forceinline__ bf16x8 read_transposed(const char *p, int pitch)          // n 0..3 from p, 4..7 four rows on
{
    typedef __attribute__((address_space(3))) s16x4 *Lds;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * pitch));
    const __attribute__((ext_vector_type(8))) short r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, r);
}

template <typename T, int TM, int TN, int KS>
constexpr int grad_lds() { return 2 * KS * (64 * TN * 2 + 64 * TM * 2 * (sizeof(T) == 4 ? 3 : 1)); }

template <typename T, int TM, int TN, int KS, int OCC>
__global__ __launch_bounds__(256, OCC) void fc_grad_kept_kernel(const KeptGradArgs a)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int BO = 64 * TM, BI = 64 * TN;
    constexpr int XP = BI * 2, DP = BO * 2;                              // bytes of a staged row
    constexpr int XB = KS * XP, DB = KS * DP, STAGE = XB + PARTS * DB;
    constexpr int NX = (KS * BI / 16 + 255) / 256, ND = KS * BO / 8 / 256;       // pieces of 16 codes, of 8 gradients, to a thread
    constexpr int TX = KS * BI / 16 / NX;                                // (fewer pieces than threads: several take the same one)
    extern __shared__ __attribute__((aligned(16))) char lds_grad[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int unit = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (unit >= a.units) return;
    const int tiles = a.itiles * a.otiles;
    const int split = uniform(unit / tiles), tile = unit - split * tiles;
    // four columns of tiles at a time: what an XCD's work-groups take at once shares rows and columns
    const int panel = uniform(tile / (4 * a.otiles)), in_panel = tile - panel * 4 * a.otiles, deep = min(4, a.itiles - 4 * panel);
    const int ot = uniform(in_panel / deep), it = 4 * panel + in_panel - ot * deep;
    const int o0 = ot * BO, i0 = it * BI;
    const int begin = split * a.rows_per_split, end = min(a.N, begin + a.rows_per_split);
    const int steps = (end - begin + KS - 1) / KS, whole = (end - begin) / KS;         // the last step may be part of one

    // where this thread's pieces lie: rows of n and columns
    const int xrow = tid % TX / (BI / 16), xcol = tid % (BI / 16);       // piece u: KS / NX rows on
    const int drow = tid / (BO / 8), dcol = tid % (BO / 8);
    // A piece past the last output is the row's first one; one that goes past it has values of the next row, or of up to seven of
    // fewer than eight outputs.  No output is there, but the last rows of all have none behind them: steps up to `full` are read
    // without a look at rows and columns.
    const int dat = o0 + dcol * 8 < a.O ? o0 + dcol * 8 : 0;
    const int full = o0 + BO > a.O && a.O % 8 ? min(whole, (a.N - (a.O < 8 ? 7 : 1) - begin) / KS) : whole;
    // columns past the end of a row of codes are read from its start: no input is there
    const int64_t xat = i0 + xcol * 16 < a.pitch ? i0 + xcol * 16 : 0;
    u32x4 xraw[NX];
    unsigned xbyte[NX];
    int seen = 0;                                    // a value that may be infinite
    typename Vec<T>::Raw draw[ND][sizeof(T) / 2];
    const unsigned char *const xp = a.codes + (int64_t)(begin + xrow) * a.pitch + xat;
    const unsigned char *const ep = a.scales + ((int64_t)(begin + xrow) * a.pitch + xat) / kBlock;
    const T *const dp = static_cast<const T *>(a.dy) + (int64_t)(begin + drow) * a.dy_stride + dat;
    // piece u of step s: of the codes for u < NX, else of the gradients; all: every row, and see `full`
    auto load_piece = [&](int u, int s, bool all) {
        if (u < NX) {
            const int row = s * KS + u * (KS / NX);
            if (all || begin + row + xrow < end) {
                xraw[u] = *reinterpret_cast<const u32x4 *>(xp + (int64_t)row * a.pitch);
                xbyte[u] = ep[(int64_t)row * (a.pitch / kBlock)];
            } else {
                xraw[u] = u32x4{0u, 0u, 0u, 0u};
                xbyte[u] = 127;
            }
            return;
        }
        const int v = u - NX, row = s * KS + v * (KS / ND), left = begin + row + drow < end ? a.O - dat : 0;
        const T *const p = dp + (int64_t)row * a.dy_stride;
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            if (all) draw[v][h] = Vec<T>::load(p + h * Vec<T>::V);
            else draw[v][h] = Vec<T>::some(p + h * Vec<T>::V, left - h * Vec<T>::V);
        }
    };
    auto store_piece = [&](int u, char *p) {
        if (u < NX) {
            const int row = u * (KS / NX) + xrow;
            u32x4 v[2];
            kept_to_bf16(xraw[u], xbyte[u], v);
            if (PARTS == 3 && may_be_infinite(xbyte[u])) seen = 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<u32x4 *>(p + row * XP + (((2 * xcol + h) ^ (4 * (row & 3))) << 4)) = v[h];
            return;
        }
        const int row = (u - NX) * (KS / ND) + drow;
        char *const to = p + XB + row * DP + ((dcol ^ (4 * (row & 3))) << 4);
        if constexpr (PARTS == 3) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = draw[u - NX][k >> 2][k & 3];
            u32x4 part[3];
            three_parts(v, part);
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4 *>(to + q * DB) = part[q];
        } else {
            *reinterpret_cast<u32x4 *>(to) = __builtin_bit_cast(u32x4, draw[u - NX][0]);
        }
    };

    f32x16 acc[TM][TN];
#pragma unroll
    for (int p = 0; p < TM; ++p)
#pragma unroll
        for (int q = 0; q < TN; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[p][q][v] = 0.f;

    // a lane's part of a fragment: row of n within 8 (and 4 more), 4 columns of 32
    const int wo = (wave >> 1) * TM * 32, wi = (wave & 1) * TN * 32;
    const int fr = (lane >> 5) * 8 + ((lane & 15) >> 2), sw = 4 * ((lane & 15) >> 2);
    const int fc = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), within = (lane & 1) * 8;
    int xf[TN], df[TM];
#pragma unroll
    for (int q = 0; q < TN; ++q) xf[q] = fr * XP + ((((wi >> 3) + 4 * q + fc) ^ sw) << 4) + within;
#pragma unroll
    for (int m = 0; m < TM; ++m) df[m] = XB + fr * DP + ((((wo >> 3) + 4 * m + fc) ^ sw) << 4) + within;
    // A step is groups of TN products that share a fragment of dy: by 16 rows of n, parts (the small ones first) and blocks of outputs.
    constexpr int ROUND = PARTS * TM, GROUPS = KS / 16 * ROUND, PIECES = NX + ND;
    bf16x8 xq[2][TN], dq[2];
    auto read_x = [&](const char *p, int round, int q) { xq[round & 1][q] = read_transposed(p + xf[q] + round * 16 * XP, XP); };
    auto read_d = [&](const char *p, int g) {
        dq[g & 1] = read_transposed(p + df[g % TM] + (PARTS - 1 - g % ROUND / TM) * DB + g / ROUND * 16 * DP, DP);
    };
    auto start = [&](const char *p) {
#pragma unroll
        for (int q = 0; q < TN; ++q) read_x(p, 0, q);
        read_d(p, 0);
    };
    // One step.  PIPELINED: its first fragments have been read, the next two steps are there and whole, and everything else stands
    // between the products: the next group's fragments, a piece of the next step into LDS, the same of the one after it sent for;
    // all of them before the last group, at whose start the wavefronts meet, so that it covers the next step's first reads.
    int buf = 0;
    auto do_step = [&](int s, auto pipelined_c) {
        constexpr bool PIPELINED = decltype(pipelined_c)::value;
        char *const p = lds_grad + buf, *const other = lds_grad + (STAGE - buf);
        if constexpr (!PIPELINED) {
            if (s + 1 < steps)
#pragma unroll
                for (int u = 0; u < PIECES; ++u) store_piece(u, other);
            if (s + 2 < steps)
#pragma unroll
                for (int u = 0; u < PIECES; ++u) load_piece(u, s + 2, s + 2 < (u < NX ? whole : full));
            start(p);
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int round = g / ROUND, in = g % ROUND;
            if (PIPELINED && g == GROUPS - 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __syncthreads();
            }
            if constexpr (PIPELINED) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < TN; ++q) {
                acc[g % TM][q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dq[g & 1], xq[round & 1][q], acc[g % TM][q], 0, 0, 0);
                if constexpr (PIPELINED) __builtin_amdgcn_sched_barrier(0);
                if (q == 0) {
                    if (g + 1 < GROUPS) read_d(p, g + 1);
                    else if (PIPELINED) read_d(other, 0);
                }
                if (q == (TN > 2 ? 1 : 0)) {                             // the next sixteen rows' fragments of x, over this round's groups
#pragma unroll
                    for (int k = 0; k < TN; ++k)
                        if (round + 1 < KS / 16 && k * ROUND / TN == in) read_x(p, round + 1, k);
                }
                if (PIPELINED && g == GROUPS - 1) read_x(other, 0, q);
                if (PIPELINED && q == TN - 1) {
#pragma unroll
                    for (int u = 0; u < PIECES; ++u)
                        if (u * (GROUPS - 1) / PIECES == g) {
                            store_piece(u, other);
                            load_piece(u, s + 2, true);
                        }
                }
                if constexpr (PIPELINED) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (!PIPELINED) __syncthreads();
        buf = STAGE - buf;
    };
    if (steps > 0) {                                 // (always; without it the 256 x 256 tiles take 90 registers more and spill)
#pragma unroll
        for (int u = 0; u < PIECES; ++u) load_piece(u, 0, 0 < (u < NX ? whole : full));
#pragma unroll
        for (int u = 0; u < PIECES; ++u) store_piece(u, lds_grad);
        if (steps > 1)
#pragma unroll
            for (int u = 0; u < PIECES; ++u) load_piece(u, 1, 1 < (u < NX ? whole : full));
        __syncthreads();
        start(lds_grad);
        __builtin_amdgcn_s_waitcnt(0x0F70);                              // vmcnt(0): the loop's waits then count its own loads alone
        int s = 0;
        for (; s + 2 < full; ++s) do_step(s, std::true_type{});
        for (; s < steps; ++s) do_step(s, std::false_type{});
    }
    bool infinite = false;
    if constexpr (PARTS == 3) {                      // of any thread; the last step has left LDS free
        int *const all = reinterpret_cast<int *>(lds_grad);
        const int any = __ballot(seen) != 0;
        if (lane == 0) all[wave] = any;
        __syncthreads();
        infinite = uniform(all[0] | all[1] | all[2] | all[3]);
    }
    float *const dw = a.dw + (int64_t)split * a.O * a.I;
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int q = 0; q < TN; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int o = o0 + wo + m * 32 + (lane >> 5) * 4 + (v >> 2) * 8 + (v & 3), i = i0 + wi + q * 32 + (lane & 31);
                if (o < a.O && i < a.I) dw[(int64_t)o * a.I + i] = acc[m][q][v];
            }
    if (infinite) {
        __threadfence();                             // behind this lane's own stores
#pragma unroll 1
        for (int b = 0; b < TM * TN; ++b)
            infinite_input(a, dw, begin, end, i0 + wi + b % TN * 32 + (lane & 31), o0 + wo + b / TN * 32 + (lane >> 5) * 4);
    }
}

// ---------------------------------------------------------------------------
// Few samples: up to 16 SLICES of them, at least one
// ---------------------------------------------------------------------------
// Bound by writing dw.  A work-group has 128 outputs, 32 to a wavefront, which keeps their gradients as fragments in registers, all
// parts of all samples, made once; it goes through 64 inputs at a time, whose values alone pass through LDS, two buffers of them.
// Nothing waits for a store: those of one 64 inputs drain while the next ones are multiplied.  They are marked as not read again
// soon where they are whole cache lines (128 samples 9216 -> 4096 fp32 37 us, 40 without the mark, with an update that reads dw
// behind it 178 and 183; of parts of lines it costs: 9217 -> 4096 92 and 63).  (In tiles, whose work-groups load, multiply and
// store all at the same time, the first took 51 us.)
template <typename T, int SLICES, int OCC>
__global__ __launch_bounds__(256, OCC) void fc_grad_few_kernel(const KeptGradArgs a)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int ROWS = 16 * SLICES, XP = kFewInputs * 2, XB = ROWS * XP;
    constexpr int NX = (ROWS * kFewInputs / 16 + 255) / 256, TX = ROWS * kFewInputs / 16 / NX;
    __shared__ __attribute__((aligned(16))) char lds[2 * XB];
    __shared__ int any[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int ot = blockIdx.x / a.itiles, first = (blockIdx.x - ot * a.itiles) * a.rows_per_split;         // (of inputs here)
    const int count = min(a.rows_per_split, (a.I + kFewInputs - 1) / kFewInputs - first);
    const int o0 = ot * 128 + wave * 32, o = o0 + (lane & 31);

    // Pieces of 16 codes: sample tid / 4, and 64 more for the second.  Past the last sample it is the last one again, times gradients
    // of zero: where that is NaN, so is the sum with the last one itself; where it is infinite, bfloat16 gradients take 2^-127 for its
    // power of two, and for fp32 ones the sums are made again.  (No branch, behind which each load would be waited for.)
    const int xrow = tid % TX >> 2, xcol = (tid & 3) * 16;
    u32x4 xraw[NX];
    unsigned xbyte[NX];
    unsigned long long seen = 0;                     // lanes that have had a value that may be infinite
    unsigned xat[NX];                                // (all codes are fewer than 2^31)
#pragma unroll
    for (int u = 0; u < NX; ++u) xat[u] = (unsigned)min(u * (TX >> 2) + xrow, a.N - 1) * (unsigned)a.pitch + first * kFewInputs + xcol;
    auto load_x = [&](int j) {                       // past the last step that one again
        const int at = min(j, count - 1) * kFewInputs;
#pragma unroll
        for (int u = 0; u < NX; ++u) {
            xraw[u] = *reinterpret_cast<const u32x4 *>(a.codes + xat[u] + at);
            xbyte[u] = a.scales[(xat[u] + at) / kBlock];
        }
    };
    // piece c of row n at place c ^ 4 (n / 2 % 2): rows of 128 bytes, four of them and 64 bytes of each to a read
    auto store_x = [&](char *p) {
#pragma unroll
        for (int u = 0; u < NX; ++u) {
            const int row = u * (TX >> 2) + xrow;
            const unsigned byte = PARTS == 3 || row < a.N ? xbyte[u] : 0;
            u32x4 v[2];
            kept_to_bf16(xraw[u], byte, v);
            if (PARTS == 3) seen |= __ballot(may_be_infinite(byte));
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<u32x4 *>(p + row * XP + ((((xcol >> 3) + h) ^ (4 * (row >> 1 & 1))) << 4)) = v[h];
        }
    };
    load_x(0);

    // a lane has output o and samples 16 s + 8 (lane / 32) + 0 .. 7 of slice s; past the end it reads its first one, or the last of
    // all, which then is dropped
    bf16x8 d[SLICES][PARTS];
    const int n0 = min(8 * (lane >> 5), a.N - 1);
    const T *const dp = static_cast<const T *>(a.dy) + (int64_t)n0 * a.dy_stride + min(o, a.O - 1);
#pragma unroll
    for (int s = 0; s < SLICES; ++s) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {                // (masks: a choice between addresses becomes branches, which wait for each load)
            const int64_t there = (n0 + 16 * s + k - a.N) >> 31;
            v[k] = ld_elem(dp + ((16 * s + k) * a.dy_stride & there), 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 16 * s + 8 * (lane >> 5) + k < a.N && o < a.O ? v[k] : 0.f;
        if constexpr (PARTS == 3) {
            u32x4 part[3];
            three_parts(v, part);
#pragma unroll
            for (int p = 0; p < 3; ++p) d[s][p] = __builtin_bit_cast(bf16x8, part[p]);
        } else {
            u32x4 q;
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = __builtin_amdgcn_perm(__float_as_uint(v[2 * k + 1]), __float_as_uint(v[2 * k]), 0x07060302u);
            d[s][0] = __builtin_bit_cast(bf16x8, q);
        }
    }
    store_x(lds);
    load_x(1);
    __syncthreads();

    const int fr = (lane >> 5) * 8 + ((lane & 15) >> 2), sw = 4 * ((lane & 15) >> 3);
    const int fc = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), within = (lane & 1) * 8;
    int xf[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) xf[q] = fr * XP + (((4 * q + fc) ^ sw) << 4) + within;
    // One 64 inputs; lines: all of the wavefront's outputs and inputs are there, in whole cache lines.  Loads and stores are counted
    // together, in their order: where every path stores as often, the wait for the next values leaves this step's stores under way.
    auto do_step = [&](int j, auto lines_c) {
        constexpr bool lines = decltype(lines_c)::value;
        const char *const p = lds + (j & 1) * XB;
        store_x(lds + ((j + 1) & 1) * XB);
        load_x(j + 2);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 acc[2];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[q][v] = 0.f;
#pragma unroll
        for (int s = 0; s < SLICES; ++s) {
            bf16x8 x[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) x[q] = read_transposed(p + xf[q] + s * 16 * XP, XP);
#pragma unroll
            for (int part = PARTS - 1; part >= 0; --part)                // the small parts first
#pragma unroll
                for (int q = 0; q < 2; ++q) acc[q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d[s][part], x[q], acc[q], 0, 0, 0);
        }
        __syncthreads();
        const int i0 = (first + j) * kFewInputs + (lane & 31);
        float *const dw = a.dw + (int64_t)(o0 + (lane >> 5) * 4) * a.I + i0;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int down = (v >> 2) * 8 + (v & 3);
#pragma unroll
            for (int q = 0; q < 2; ++q)
                if (lines) __builtin_nontemporal_store(acc[q][v], dw + (int64_t)down * a.I + 32 * q);
                else if (o0 + (lane >> 5) * 4 + down < a.O && i0 + 32 * q < a.I) dw[(int64_t)down * a.I + 32 * q] = acc[q][v];
        }
    };
    __builtin_amdgcn_s_waitcnt(0x0F70);                                  // vmcnt(0): the loop's waits then count its own alone
    const bool lines = o0 + 32 <= a.O && a.I % 32 == 0 && (reinterpret_cast<uintptr_t>(a.dw) & 127) == 0;
    const int whole = lines ? min(count, a.I / kFewInputs - first) : 0;
    int j = 0;
    for (; j < whole; ++j) do_step(j, std::true_type{});
    for (; j < count; ++j) do_step(j, std::false_type{});
    if constexpr (PARTS == 3) {
        const int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));        // lane, which nothing has to hold until here
        if (l == 0) any[wave] = seen != 0;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // (the stores are not waited for)
        if (any[0] | any[1] | any[2] | any[3]) {
            __threadfence();                         // behind this lane's own stores
#pragma unroll 1
            for (int b = 0; b < 2 * count; ++b) infinite_input(a, a.dw, 0, a.N, first * kFewInputs + b * 32 + (l & 31), o0 + (l >> 5) * 4);
        }
    }
}

// the splits' sums, one after the other; zeros for no splits
__global__ __launch_bounds__(256) void fc_grad_join(const float *part, float *dw, int64_t count, int splits)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float s = splits > 0 ? part[i] : 0.f;
    for (int p = 1; p < splits; ++p) s += part[p * count + i];
    dw[i] = s;
}
