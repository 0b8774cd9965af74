// Forward pass of a fully connected layer with both operands in blocks of 4 bits:
//   y[n][o] = f(sum_i x[n][i] w[o][i] + bias[o]),  x and w E2M1 numbers times a power of two for every 32 of i
// Part of block_ops.hip: included there, inside its anonymous namespace, after block_formats.h.
//
// The matrix instructions multiply them as they are: a lane holds 32 neighbouring values of a row (16 bytes), and the byte of
// their exponent.  Rows are filled up to 128 values, so a step of the sum is one 64-byte piece and one 4-byte word of exponents of
// every row.  w is the first operand: a lane then has four neighbouring outputs of one sample.

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// f(s + bias); NaN stays
__device__ __forceinline__ float finish_q4(float s, float bias, int relu)
{
    s += bias;
    return relu && s < 0.f ? 0.f : s;
}

// 32 outputs from o0 on of sample n, as v_mfma_scale_f32_32x32x64 leaves them: value 4 q + k of a lane is output 8 q + 4 half + k.
// fp32: four neighbouring ones are 16 bytes.  bfloat16: the lanes of the two halves trade what makes eight of them (a lane of the
// lower half gets those from 8 q on, its partner those from 8 (q + 1) on), 16 bytes as well; with a store to every value, 256
// instructions to a wavefront that each touch 64 rows, the stores of a tile took as long as 40 of its steps.
// bias: those of the block's outputs, zeros past the last one.
template <typename T, typename Args>
__device__ __forceinline__ void store_block_q4(const Args &a, const float *bias, int n, int o0, int half, const f32x16 &s)
{
    T *const y = static_cast<T *>(a.y) + (int64_t)n * a.O;
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
        float v[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 b = *reinterpret_cast<const f32x4 *>(bias + 8 * (q + h) + 4 * half);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h][k] = finish_q4(s[4 * (q + h) + k], b[k], a.relu);
        }
        if constexpr (sizeof(T) == 2) {
            unsigned w[2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    w[h][k] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){v[h][2 * k], v[h][2 * k + 1]}, bf16x2));
            const auto p0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
            const auto p1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
            const int o = o0 + 8 * (q + half);
            const u32x4 r = {p0[0], p1[0], p0[1], p1[1]};
            if (n >= a.N) continue;
            if (o + 8 <= a.O) *reinterpret_cast<u32x4_any *>(y + o) = r;
            else
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (o + k < a.O) y[o + k] = (T)(r[k >> 1] >> (16 * (k & 1)));
        } else {
            if (n >= a.N) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int o = o0 + 8 * (q + h) + 4 * half;
                if (o + 4 <= a.O) *reinterpret_cast<f32x4_any *>(y + o) = f32x4{v[h][0], v[h][1], v[h][2], v[h][3]};
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (o + k < a.O) y[o + k] = v[h][k];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Many samples: tiles of TM WM 32 outputs x TN WN 32 samples
// ---------------------------------------------------------------------------
// v_mfma_scale_f32_32x32x64_f8f6f4: lane l has row l % 32 and the 32 values of block l / 32.  Both operands go from global memory
// straight into LDS, a row's 64 bytes of a step as four pieces of 16, the piece c of row r at place c ^ (r / 4 % 4): the rows are
// 64 bytes apart, and the 16 lanes of a phase of ds_read_b128 then cover all banks.  The exponents of a step lie together (see
// q4_prepare), four bytes to a row; a lane shifts its block's to the low byte.
//
// Bound by the matrix units at the clock that their power leaves: 8192 x 8192 -> 8192 261 us from idle, up to 334 between 2 and 6 ms
// of such calls, 250 to 260 in the long run: 3.3 to 4.4 PFLOP/s (the instruction alone, on random codes, 6.6).
//
// LDS: kQ4Stages buffers; step s is multiplied while those of s + 1 .. s + kQ4Stages - 1 are on their way.
struct Q4TileArgs {
    const unsigned char *xc, *wc;                // codes, rows of 64 steps bytes
    const unsigned char *xs, *ws;                // exponents [steps][rows filled up][4]
    const float *bias;
    void *y;
    int N, O, steps, relu;
    int nrows, orows;                            // rows of the exponents, multiples of the tile
    int ntiles, otiles, per_xcd;
};

constexpr int kQ4Stages = 4;

__device__ __forceinline__ void dma16(const void *base, unsigned offset, unsigned lds)       // 16 bytes to a lane, at lds + 16 lane
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void dma4(const void *base, unsigned offset, unsigned lds)        // 4 bytes to a lane, at lds + 4 lane
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(lds), "v"(offset), "s"(base) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

__device__ __forceinline__ f32x16 mfma_q4_wide(const i32x4 &w, const i32x4 &x, const f32x16 &c, unsigned ws, unsigned xs, int second)
{
    const i32x8 a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return second ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 2, (int)ws, 2, (int)xs)
                  : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 0, (int)ws, 0, (int)xs);
}

template <typename T, int TM, int TN, int WM, int WN, int OCC>
__global__ __launch_bounds__(WM * WN * 64, OCC) void fc_q4_tiles(const Q4TileArgs a)
{
    constexpr int NT = WM * WN * 64, BM = TM * WM * 32, BN = TN * WN * 32;
    constexpr int NA = BM * 4 / NT, NB = BN * 4 / NT;            // loads of codes to a thread and step
    constexpr int CODES = (BM + BN) * 64, STAGE = CODES + (BM + BN) * 4;
    constexpr int NE = (BM + BN) / NT;                           // ... of exponents
    constexpr int LOADS = NA + NB + NE;
    static_assert((BM + BN) % NT == 0 && BM % (64 * NE) == 0, "a wavefront's exponents are of one operand");
    extern __shared__ __attribute__((aligned(16))) char lds_q4[];
    const unsigned lds0 = (unsigned)(size_t)lds_q4;
    const int unit = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (unit >= a.ntiles * a.otiles) return;
    // four rows of tiles at a time: the tiles that an XCD's work-groups take at once are 8 x 4, not 32 x 1
    const int panel = uniform(unit / (4 * a.otiles)), in_panel = unit - panel * 4 * a.otiles, deep = min(4, a.ntiles - 4 * panel);
    const int ot = uniform(in_panel / deep), nt = 4 * panel + in_panel - ot * deep;
    const int o0 = ot * BM, n0 = nt * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const unsigned pitch = (unsigned)a.steps * 64;
    float *const bias = reinterpret_cast<float *>(lds_q4 + kQ4Stages * STAGE);
    for (int i = tid; i < BM; i += NT) bias[i] = a.bias && o0 + i < a.O ? a.bias[o0 + i] : 0.f;

    // load u of a thread: piece q % 4 of row q / 4, q = (wave loads + u) 64 + lane; rows past the end read the last one
    unsigned aoff[NA], boff[NB];
#pragma unroll
    for (int u = 0; u < NA; ++u) {
        const int q = (wave * NA + u) * 64 + lane, row = q >> 2, c = (q & 3) ^ ((row >> 2) & 3);
        aoff[u] = (unsigned)min(row, a.O - 1 - o0) * pitch + c * 16;
    }
#pragma unroll
    for (int u = 0; u < NB; ++u) {
        const int q = (wave * NB + u) * 64 + lane, row = q >> 2, c = (q & 3) ^ ((row >> 2) & 3);
        boff[u] = (unsigned)min(row, a.N - 1 - n0) * pitch + c * 16;
    }
    const unsigned char *wc = a.wc + (int64_t)o0 * pitch, *xc = a.xc + (int64_t)n0 * pitch;
    // exponents: the wavefront's part of the stage's BM + BN words, w's first
    const int sfirst = wave * NE * 64;
    const bool of_w = sfirst < BM;
    const unsigned char *sp = of_w ? a.ws + (int64_t)(o0 + sfirst) * 4 : a.xs + (int64_t)(n0 + sfirst - BM) * 4;
    const int64_t s_step = (int64_t)(of_w ? a.orows : a.nrows) * 4;

    auto load_one = [&](int u, int s, unsigned l) {              // u < LOADS, known when unrolled; s: the step, l: its stage's place
        if (u < NA) dma16(wc + s * 64, aoff[u], l + (wave * NA + u) * 1024);
        else if (u < NA + NB) dma16(xc + s * 64, boff[u - NA], l + BM * 64 + (wave * NB + u - NA) * 1024);
        else dma4(sp + s * s_step, (u - NA - NB) * 256 + lane * 4, l + CODES + sfirst * 4 + (u - NA - NB) * 256);
    };

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    const int r = lane & 31, half = lane >> 5, swz = (r >> 2) & 3;
    const int arow = (wm * TM * 32 + r) * 64, brow = BM * 64 + (wn * TN * 32 + r) * 64;
    const int sa = CODES + (wm * TM * 32 + r) * 4, sb = CODES + (BM + wn * TN * 32 + r) * 4;

    i32x4 w[2][TM], x[2][TN];                                    // fragments of the two halves of a step
    unsigned en[TM], fn[TN];                                     // exponents of the next step
    constexpr int FRAGMENTS = TM + TN, EXPONENTS = (TM + TN) / 2;
    auto read_exponents = [&](const char *p, int u) {            // two words, u < EXPONENTS
        const int e = 2 * u;
        if (e < TM) {
            en[e] = *reinterpret_cast<const unsigned *>(p + sa + e * 128);
            en[e + 1] = *reinterpret_cast<const unsigned *>(p + sa + e * 128 + 128);
        } else {
            fn[e - TM] = *reinterpret_cast<const unsigned *>(p + sb + (e - TM) * 128);
            fn[e - TM + 1] = *reinterpret_cast<const unsigned *>(p + sb + (e - TM) * 128 + 128);
        }
    };
    auto read_codes = [&](const char *p, int k, int u) {         // fragment u < FRAGMENTS of half k
        const int at = ((2 * k + half) ^ swz) * 16;
        if (u < TN) x[k][u] = *reinterpret_cast<const i32x4 *>(p + brow + u * 2048 + at);
        else w[k][u - TN] = *reinterpret_cast<const i32x4 *>(p + arow + (u - TN) * 2048 + at);
    };

    const int steps = a.steps;
#pragma unroll
    for (int s = 0; s < kQ4Stages - 1; ++s)
        if (s < steps) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) load_one(u, s, lds0 + s * STAGE);
        }
    // this wavefront's loads of step 0 have landed
    if (kQ4Stages - 1 <= steps) wait_vmcnt<(kQ4Stages - 2) * LOADS>();
    else wait_vmcnt<0>();
    __syncthreads();
#pragma unroll
    for (int u = 0; u < EXPONENTS; ++u) read_exponents(lds_q4, u);
#pragma unroll
    for (int u = 0; u < FRAGMENTS; ++u) read_codes(lds_q4, 0, u);
    int buf = 0;
    // One step, in two halves of 64 values.  While the first is multiplied, the second one's fragments are read and the step
    // kQ4Stages - 1 on is sent for, into the buffer of the step before this one: every wavefront is past that.  Before the second
    // is multiplied the next step has to have landed; its first half's fragments and exponents are read meanwhile.  The reads and
    // loads stand between the matrix instructions: eight reads at once, of four wavefronts, hold up the instructions behind them.
    constexpr int PER = TM * TN, EARLY = LOADS - LOADS / 5, LATE = LOADS - EARLY;
    static_assert(TM % 2 == 0 && TN % 2 == 0, "exponents are read in twos");
    auto do_step = [&](int s, auto more_c, auto next_c) {        // more: there is a step to send for; next: there is a next one
        constexpr bool more = decltype(more_c)::value, has_next = decltype(next_c)::value;
        const char *const p = lds_q4 + buf * STAGE;
        const int next = buf == kQ4Stages - 1 ? 0 : buf + 1, free = buf == 0 ? kQ4Stages - 1 : buf - 1;
        const char *const after = lds_q4 + next * STAGE;
        const unsigned to = lds0 + free * STAGE;
        unsigned es[TM], ex[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) es[i] = en[i] >> (8 * half);
#pragma unroll
        for (int j = 0; j < TN; ++j) ex[j] = fn[j] >> (8 * half);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                acc[i][j] = mfma_q4_wide(w[0][i], x[0][j], acc[i][j], es[i], ex[j], 0);
                const int m = i * TN + j;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = m * (FRAGMENTS + EARLY) / PER; u < (m + 1) * (FRAGMENTS + EARLY) / PER; ++u)
                    if (u < FRAGMENTS) read_codes(p, 1, u);
                    else if (more) load_one(u - FRAGMENTS, s + kQ4Stages - 1, to);
                __builtin_amdgcn_sched_barrier(0);
            }
        if (has_next) {
            if (more) wait_vmcnt<(kQ4Stages - 3) * LOADS + EARLY>();
            else wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __syncthreads();
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                acc[i][j] = mfma_q4_wide(w[1][i], x[1][j], acc[i][j], es[i], ex[j], 1);
                const int m = i * TN + j;
                __builtin_amdgcn_sched_barrier(0);
                constexpr int READS = FRAGMENTS + EXPONENTS;
#pragma unroll
                for (int u = m * (READS + LATE) / PER; u < (m + 1) * (READS + LATE) / PER; ++u)
                    if (u < READS) {
                        if (has_next && u < FRAGMENTS) read_codes(after, 0, u);
                        else if (has_next) read_exponents(after, u - FRAGMENTS);
                    } else if (more) {
                        load_one(u - READS + EARLY, s + kQ4Stages - 1, to);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        buf = next;
    };
    int s = 0;
    for (; s + kQ4Stages - 1 < steps; ++s) do_step(s, std::true_type{}, std::true_type{});
    for (; s + 1 < steps; ++s) do_step(s, std::false_type{}, std::true_type{});
    do_step(s, std::false_type{}, std::false_type{});
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            store_block_q4<T>(a, bias + (wm * TM + i) * 32, n0 + (wn * TN + j) * 32 + r, o0 + (wm * TM + i) * 32, half, acc[i][j]);
}

// Before the tiles: x in blocks, and the exponents of both operands as the tiles load them, [step][row][4 bytes], in one launch.
// Bound by memory: 8192 x 8192 bfloat16 41 us, 4.3 TB/s.
struct Q4PrepArgs {
    BlockArgs x;                                 // total, per_row and so on; scales unused
    const unsigned *w_scales;                    // [O][steps] words
    unsigned *xs, *ws;                           // [steps][nrows], [steps][orows]
    int O, steps, nrows, orows;
    int x_blocks, s_tiles;                       // work-groups that take x; tiles of 32 steps to a row of tiles
};

template <typename T>
__global__ __launch_bounds__(256) void q4_prepare(const Q4PrepArgs p)
{
    if ((int)blockIdx.x < p.x_blocks) {
        const BlockArgs &a = p.x;
        const int64_t base = (int64_t)blockIdx.x * 256, i = base + threadIdx.x;
        const int64_t row0 = base / a.per_row;
        const unsigned at = (unsigned)(base - row0 * a.per_row) + threadIdx.x;
        const unsigned down = fastdiv(at, a.div);
        const int64_t row = row0 + down;
        const int v8 = (int)(at - down * a.per_row);
        if (i >= a.total) return;
        float v[8];
        load8(static_cast<const T *>(a.in) + row * a.stride + v8 * 8, a.C - v8 * 8, v);
        unsigned word[2];
        const int byte = into_codes<kE2M1>(v, word);
        static_cast<unsigned *>(a.out)[i] = word[0];
        if (v8 % 4 == 0) reinterpret_cast<unsigned char *>(p.xs)[((int64_t)(v8 >> 4) * p.nrows + row) * 4 + ((v8 >> 2) & 3)] = (unsigned char)byte;
        return;
    }
    // 32 x 32 words of w's exponents turned round
    __shared__ unsigned turned[32][33];
    const int b = blockIdx.x - p.x_blocks;
    const int rt = b / p.s_tiles, st = b - rt * p.s_tiles;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        const int o = rt * 32 + ty + k, s = st * 32 + tx;
        if (o < p.O && s < p.steps) turned[ty + k][tx] = p.w_scales[(int64_t)o * p.steps + s];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        const int s = st * 32 + ty + k, o = rt * 32 + tx;
        if (o < p.O && s < p.steps) p.ws[(int64_t)s * p.orows + o] = turned[tx][ty + k];
    }
}

// ---------------------------------------------------------------------------
// Few samples: AO 16 outputs x J 16 samples to a work-group, whose wavefronts (eight; four for more than 32 samples) share the sum
// ---------------------------------------------------------------------------
// Bound by reading w once.  v_mfma_scale_f32_16x16x128_f8f6f4: lane l has row l % 16 and the 32 values of block l / 16.  The
// wavefronts of a work-group take parts of the sum, each with a ring of STAGES buffers of its own in LDS, so that none waits for
// another; their sums are joined through LDS.  A buffer holds 256 values of every row (128 bytes, a cache line), loaded directly,
// the piece c of 16 bytes of row r at place c ^ (r / 2 % 8).  (Fragments loaded into registers take a cache line to every lane of
// sixteen: 128 samples 9216 -> 4096 19 us.)
// One sample 4096 -> 4096 4.9 us, 1.8 TB/s; 128 samples 9216 -> 4096 11.5 us, where x's codes come from the L2s 128 times.
// FUSED: every work-group puts all of x into blocks itself, in LDS, while its first loads of w are on their way: a launch less.
// Else the exponents of both operands come by steps, as the tiles have them.
struct Q4RowsArgs {
    const void *x;                               // FUSED: the values
    const unsigned char *xc, *xs;                // else their codes, and exponents [steps][nrows][4]
    const unsigned char *wc, *ws;                // codes, and exponents: FUSED [O][steps][4], else [steps][orows][4]
    const float *bias;
    void *y;
    int N, I, O, steps, relu;
    int nrows, orows;
    int ntiles, units, per_xcd;
    int held;                                    // FUSED: bytes of x's codes and exponents, in front of the rings
    FastDiv div_row;                             // by 16 steps: eights of a row
};

__device__ __forceinline__ f32x4 mfma_q4(const i32x4 &w, const i32x4 &x, const f32x4 &c, unsigned ws, unsigned xs)
{
    const i32x8 a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)ws, 0, (int)xs);
}

// a ring's buffer: codes of the rows, then words of exponents, by steps and rows (a load of 64 words at least)
constexpr int q4_rows_stage(int AO, int J, bool fused)
{
    const int rows = 16 * (fused ? AO : AO + J), words = 32 * AO < 64 ? 64 : 32 * AO;
    return rows * 128 + 4 * (words + (fused ? 0 : 32 * J < 64 ? 64 : 32 * J));
}

template <typename TX, typename TY, int AO, int J, bool FUSED, int WAVES, int STAGES>
__global__ __launch_bounds__(WAVES * 64) void fc_q4_rows(const Q4RowsArgs a)
{
    constexpr int RA = 16 * AO, RB = FUSED ? 0 : 16 * J;                 // rows of a buffer, w's first
    constexpr int NA = RA / 8, NB = RB / 8;                              // loads of codes
    constexpr int EA = RA * 2 < 64 ? 1 : RA * 2 / 64, EB = FUSED ? 0 : RB * 2 < 64 ? 1 : RB * 2 / 64;
    constexpr int LOADS = NA + NB + EA + EB, STAGE = q4_rows_stage(AO, J, FUSED);
    constexpr int EXPA = (RA + RB) * 128, EXPB = EXPA + EA * 256;
    extern __shared__ __attribute__((aligned(16))) char lds_rows[];      // x's codes and exponents; rings; at last the sums
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int unit = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);   // an XCD's work-groups share rows of w
    if (unit >= a.units) return;
    const int ot = uniform(unit / a.ntiles), nt = unit - ot * a.ntiles;
    const int o0 = ot * RA, n0 = nt * J * 16;
    const int r = lane & 15, g = lane >> 4;
    const unsigned cpitch = (unsigned)a.steps * 64, spitch = (unsigned)a.steps * 4;

    // load u of codes: rows 8 u .. 8 u + 7; rows past the end read the last one, not stored.  A last step of 128 values is read twice.
    unsigned arow[NA], brow[NB + 1], aexp[EA], bexp[EB + 1];
    const unsigned piece = ((lane & 7) ^ (lane >> 4)) * 16;
#pragma unroll
    for (int u = 0; u < NA; ++u) arow[u] = (unsigned)min(8 * u + (lane >> 3), a.O - 1 - o0) * cpitch;
#pragma unroll
    for (int u = 0; u < NB; ++u) brow[u] = (unsigned)min(8 * u + (lane >> 3), a.N - 1 - n0) * cpitch;
    // load u of exponents: words 64 u .. of [step][row] (twice the same 32 where there are no more)
    const int half_a = (lane / RA) & 1;
#pragma unroll
    for (int u = 0; u < EA; ++u) {
        const int word = (64 * u + lane) % (2 * RA), row = word % RA;
        aexp[u] = FUSED ? (unsigned)min(row, a.O - 1 - o0) * spitch : (unsigned)row * 4;
    }
#pragma unroll
    for (int u = 0; u < EB; ++u) bexp[u] = (unsigned)((64 * u + lane) % (16 * J)) * 4;
    const unsigned char *const wc = a.wc + (int64_t)o0 * cpitch, *const xc = FUSED ? nullptr : a.xc + (int64_t)n0 * cpitch;
    const unsigned char *const we = a.ws + (FUSED ? (int64_t)o0 * spitch : (int64_t)o0 * 4), *const xe = FUSED ? nullptr : a.xs + (int64_t)n0 * 4;
    const int pairs = (a.steps + 1) >> 1;
    const int first = (int)((int64_t)pairs * wave / WAVES), last = (int)((int64_t)pairs * (wave + 1) / WAVES);
    char *const ring = lds_rows + a.held + wave * STAGES * STAGE;
    const unsigned ring_at = (unsigned)(size_t)lds_rows + a.held + wave * STAGES * STAGE;
    const unsigned w_step = FUSED ? 4 : (unsigned)a.orows * 4, x_step = (unsigned)a.nrows * 4;
    auto load = [&](int p, int slot) {
        const unsigned l = ring_at + slot * STAGE;
        const bool whole = 2 * p + 1 < a.steps;
        const unsigned keep = whole ? 127 : 63;
#pragma unroll
        for (int u = 0; u < NA; ++u) dma16(wc + p * 128, arow[u] + ((piece ^ (u & 1) * 64) & keep), l + u * 1024);
#pragma unroll
        for (int u = 0; u < NB; ++u) dma16(xc + p * 128, brow[u] + ((piece ^ (u & 1) * 64) & keep), l + RA * 128 + u * 1024);
        // the second step's words; the first one's again where there is none
        const unsigned second = whole ? 1 : 0;
#pragma unroll
        for (int u = 0; u < EA; ++u) {
            const unsigned h = RA * 2 <= 64 ? half_a : 64 * u / RA;
            dma4(we + (int64_t)2 * p * w_step, aexp[u] + (h & second) * w_step, l + EXPA + u * 256);
        }
#pragma unroll
        for (int u = 0; u < EB; ++u) {
            const unsigned h = J <= 2 ? (lane / (16 * J)) & 1 : 64 * u / (16 * J);
            dma4(xe + (int64_t)2 * p * x_step, bexp[u] + (h & second) * x_step, l + EXPB + u * 256);
        }
    };
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k)
        if (first + k < last) load(first + k, k);
    const char *const fc = lds_rows + (int64_t)min(r, a.N - 1) * cpitch + g * 16;
    const char *const fe = lds_rows + (int64_t)a.N * cpitch + (int64_t)min(r, a.N - 1) * spitch + g;
    if constexpr (FUSED) {
        const int per_row = a.steps * 16, total = a.N * per_row;         // a multiple of 16: blocks of lanes stay whole
        for (int i = tid; i < total; i += WAVES * 64) {
            const int n = (int)fastdiv((unsigned)i, a.div_row), c = (i - n * per_row) * 8;
            float v[8];
            load8(static_cast<const TX *>(a.x) + (int64_t)n * a.I + c, a.I - c, v);
            unsigned word[2];
            const int byte = into_codes<kE2M1>(v, word);
            *reinterpret_cast<unsigned *>(lds_rows + i * 4) = word[0];
            if (i % 4 == 0) lds_rows[(int64_t)a.N * cpitch + (i >> 2)] = (char)byte;
        }
        __syncthreads();
    }
    f32x4 acc[AO][J];
#pragma unroll
    for (int i = 0; i < AO; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int swz = (r >> 1) & 7;
    int slot = 0;
    for (int p = first; p < last; ++p) {
        // the buffer of the pair before this one is sent for again: what was read of it has arrived
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (p + STAGES - 1 < last) {
            load(p + STAGES - 1, slot == 0 ? STAGES - 1 : slot - 1);
            wait_vmcnt<(STAGES - 1) * LOADS>();
        } else {
            wait_vmcnt<0>();
        }
        const char *const buf = ring + slot * STAGE;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // Where there is no second step it is the first one again, times zero: a block that is NaN has made its sums NaN before.
            // (A branch costs a copy of all sums, 32 instructions to 16 products.)
            const int keep = 2 * p + h < a.steps ? -1 : 0;
            const int at = ((4 * h + g) ^ swz) * 16;
            i32x4 w[AO], x[J];
            unsigned ew[AO], ex[J];
#pragma unroll
            for (int i = 0; i < AO; ++i) {
                w[i] = *reinterpret_cast<const i32x4 *>(buf + (16 * i + r) * 128 + at) & keep;
                ew[i] = static_cast<unsigned char>(buf[EXPA + (h * RA + 16 * i + r) * 4 + g]);
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if constexpr (FUSED) {
                    const int step = 2 * p + (h & keep);
                    x[j] = *reinterpret_cast<const i32x4 *>(fc + step * 64);
                    ex[j] = static_cast<unsigned char>(fe[step * 4]);
                } else {
                    x[j] = *reinterpret_cast<const i32x4 *>(buf + (RA + 16 * j + r) * 128 + at);
                    ex[j] = static_cast<unsigned char>(buf[EXPB + (h * RB + 16 * j + r) * 4 + g]);
                }
            }
#pragma unroll
            for (int i = 0; i < AO; ++i)
#pragma unroll
                for (int j = 0; j < J; ++j) acc[i][j] = mfma_q4(w[i], x[j], acc[i][j], ew[i], ex[j]);
        }
        slot = slot == STAGES - 1 ? 0 : slot + 1;
    }
    __syncthreads();
    f32x4 *const sums = reinterpret_cast<f32x4 *>(lds_rows);             // [wavefront][block of 16 x 16][lane]
#pragma unroll
    for (int i = 0; i < AO; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) sums[(wave * AO * J + i * J + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int t = tid; t < AO * J * 64; t += WAVES * 64) {
        f32x4 s = sums[t];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) s += sums[k * AO * J * 64 + t];
        const int block = t >> 6, i = block / J, j = block - i * J;
        const int n = n0 + j * 16 + (t & 15), o = o0 + i * 16 + ((t >> 4) & 3) * 4;
        if (n >= a.N) continue;
        TY *const y = static_cast<TY *>(a.y) + (int64_t)n * a.O;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (o + k < a.O) st_elem(y, o + k, finish_q4(s[k], a.bias ? a.bias[o + k] : 0.f, a.relu));
    }
}
