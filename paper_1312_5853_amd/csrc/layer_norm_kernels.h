// Layer normalisation: forward, and backward from the values themselves or from values held in blocks of 8 bits.
// Part of block_ops.hip: included there, inside its anonymous namespace, after block_formats.h.
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  xh = (x - mean) rstd,  y = gamma xh + beta
//   g = gamma dy,  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//
// A row is read once and kept in registers (R vectors to a thread) from its sums to its result.  `waves` wavefronts take a row,
// as many rows as fit run side by side in a work-group, and a work-group goes through rows so far apart as there are, the next
// one's values on their way while one is summed and written: backward, the sums of the columns stay in its registers.

// The last vector of a row may be part of one.  It is read whole, as the row's last V values, and moved down when it is used, so
// that no load is waited for at once (value by value 6001 x 5003 bfloat16 forward took 36 us, 28 with 5008); rows of fewer than V
// values are read one by one.  It is stored in pieces of 8, 4 and 2 bytes.
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef unsigned u32_any __attribute__((aligned(2)));
typedef f32x2 f32x2_any __attribute__((aligned(4)));

__device__ __forceinline__ f32x4 move_down(f32x4 r, int n)            // drops the first n values, zeros behind the others
{
    if (n & 2) r = f32x4{r[2], r[3], 0.f, 0.f};
    if (n & 1) r = f32x4{r[1], r[2], r[3], 0.f};
    return r;
}
__device__ __forceinline__ u32x4 move_down(u32x4 r, int n)
{
    if (n & 4) r = u32x4{r[2], r[3], 0u, 0u};
    if (n & 2) r = u32x4{r[1], r[2], r[3], 0u};
    if (n & 1)
        r = u32x4{__builtin_amdgcn_alignbit(r[1], r[0], 16), __builtin_amdgcn_alignbit(r[2], r[1], 16),
                  __builtin_amdgcn_alignbit(r[3], r[2], 16), r[3] >> 16};
    return r;
}
__device__ __forceinline__ f32x4 move_round(f32x4 r, int n)           // puts the first n values behind the others
{
    if (n & 2) r = f32x4{r[2], r[3], r[0], r[1]};
    if (n & 1) r = f32x4{r[1], r[2], r[3], r[0]};
    return r;
}
__device__ __forceinline__ u32x4 move_round(u32x4 r, int n)
{
    if (n & 4) r = u32x4{r[2], r[3], r[0], r[1]};
    if (n & 2) r = u32x4{r[1], r[2], r[3], r[0]};
    if (n & 1)
        r = u32x4{__builtin_amdgcn_alignbit(r[1], r[0], 16), __builtin_amdgcn_alignbit(r[2], r[1], 16),
                  __builtin_amdgcn_alignbit(r[3], r[2], 16), __builtin_amdgcn_alignbit(r[0], r[3], 16)};
    return r;
}
__device__ __forceinline__ void store_first(float *p, const float (&v)[4], int n)        // n < 4
{
    if (n & 2) *reinterpret_cast<f32x2_any *>(p) = f32x2{v[0], v[1]};
    if (n & 1) p[n & 2] = n & 2 ? v[2] : v[0];
}
__device__ __forceinline__ void store_first(unsigned short *p, const float (&v)[8], int n)
{
    u32x4 q;
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){v[2 * k], v[2 * k + 1]}, bf16x2));
    if (n & 4) {
        *reinterpret_cast<u32x2_any *>(p) = u32x2{q[0], q[1]};
        q = u32x4{q[2], q[3], 0u, 0u};
    }
    if (n & 2) {
        *reinterpret_cast<u32_any *>(p + (n & 4)) = q[0];
        q[0] = q[1];
    }
    if (n & 1) p[n & 6] = (unsigned short)q[0];
}

// of a vector with `left` values of the row from it on: how many of those read for it belong to the vector before
template <int V>
__device__ __forceinline__ int skipped(int left) { return max(0, V - left); }

// the first value of a vector in place of those from the n-th on, 0 < n
__device__ __forceinline__ void repeat_first(f32x4 &r, int n)
{
#pragma unroll
    for (int k = 1; k < 4; ++k) r[k] = k < n ? r[k] : r[0];
}
__device__ __forceinline__ void repeat_first(u32x4 &r, int n)
{
    const unsigned both = __builtin_amdgcn_perm(r[0], r[0], 0x05040504u);
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = 2 * k + 1 < n ? r[k] : 2 * k < n ? (r[k] & 0xFFFFu) | (both & 0xFFFF0000u) : both;
}

// vectors of x of one row: of an array, or of codes
template <typename T, bool HELD>
struct RowSource;

template <typename T>
struct RowSource<T, false> {
    typedef typename Vec<T>::Raw Raw;
    const T *p;
    __device__ __forceinline__ RowSource(const LayerNormArgs &a, int64_t row) : p(static_cast<const T *>(a.x) + row * a.x_stride) {}
    __device__ __forceinline__ Raw load(int v, int left, int C) const                    // left > 0
    {
        return C >= Vec<T>::V ? Vec<T>::load(p + (v * Vec<T>::V - skipped<Vec<T>::V>(left))) : Vec<T>::some(p, C);
    }
    static __device__ __forceinline__ void settle(Raw &r, int skip) { r = move_down(r, skip); }
    static __device__ __forceinline__ void settle_round(Raw &r, int skip) { r = move_round(r, skip); }
    static __device__ __forceinline__ void repeat(Raw &r, int n) { repeat_first(r, n); }
    static __device__ __forceinline__ void open(const Raw &r, float (&v)[Vec<T>::V]) { Vec<T>::open(r, v); }
    __device__ __forceinline__ float at(int c) const { return ld_elem(p, c); }
};

template <typename T>
struct RowSource<T, true> {
    static constexpr int V = Vec<T>::V;
    struct Raw {
        unsigned word[V / 4];
        unsigned byte;
    };
    const unsigned char *p, *s;
    __device__ __forceinline__ RowSource(const LayerNormArgs &a, int64_t row)
        : p(a.codes + row * a.pitch), s(a.scales + row * (a.pitch / kBlock)) {}
    __device__ __forceinline__ Raw load(int v, int, int) const                           // rows are filled up: whole vectors
    {
        Raw r;
        if constexpr (V == 8) {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(p + (int64_t)v * 8);
            r.word[0] = w[0]; r.word[1] = w[1];
        } else {
            r.word[0] = *reinterpret_cast<const unsigned *>(p + (int64_t)v * 4);
        }
        r.byte = s[v / (kBlock / V)];
        return r;
    }
    static __device__ __forceinline__ void settle(Raw &, int) {}
    static __device__ __forceinline__ void settle_round(Raw &r, int skip) { repeat(r, V - skip); }
    static __device__ __forceinline__ void repeat(Raw &r, int n)
    {
        const unsigned all = (r.word[0] & 0xFFu) * 0x01010101u;
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            const unsigned keep = n >= 4 * k + 4 ? ~0u : n > 4 * k ? (1u << 8 * (n - 4 * k)) - 1 : 0u;
            r.word[k] = (r.word[k] & keep) | (all & ~keep);
        }
    }
    static __device__ __forceinline__ void open(const Raw &r, float (&v)[V])
    {
#pragma unroll
        for (int k = 0; k < V / 4; ++k) open_e4m3(r.word[k], block_scale(r.byte), v + 4 * k);
    }
    __device__ __forceinline__ float at(int c) const
    {
        return __builtin_amdgcn_cvt_f32_fp8((int)p[c], 0) * block_scale(s[c / kBlock]);
    }
};

// Two sums over the 64 lanes: over the rows of 16, then from each row into the next (row_bcast), the last lane's at the end; the two
// chains fill each other's wait states.  Half the instructions of two wave_sum.
__device__ __forceinline__ void wave_sums(float &a, float &b)
{
    a += dpp_move<0xB1>(a);  b += dpp_move<0xB1>(b);
    a += dpp_move<0x4E>(a);  b += dpp_move<0x4E>(b);
    a += dpp_move<0x141>(a); b += dpp_move<0x141>(b);
    a += dpp_move<0x140>(a); b += dpp_move<0x140>(b);
    auto from_row = [](float v, auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
    };
    typedef std::integral_constant<int, 0x142> Bcast15;
    typedef std::integral_constant<int, 0x143> Bcast31;
    a += from_row(a, Bcast15{}, std::integral_constant<int, 0xA>{});
    b += from_row(b, Bcast15{}, std::integral_constant<int, 0xA>{});
    a += from_row(a, Bcast31{}, std::integral_constant<int, 0xC>{});
    b += from_row(b, Bcast31{}, std::integral_constant<int, 0xC>{});
    a = lane_value(a, 63);
    b = lane_value(b, 63);
}
// ... of up to 16 lanes, zeros in the others
__device__ __forceinline__ void row_sums(float &a, float &b)
{
    a += dpp_move<0xB1>(a);  b += dpp_move<0xB1>(b);
    a += dpp_move<0x4E>(a);  b += dpp_move<0x4E>(b);
    a += dpp_move<0x141>(a); b += dpp_move<0x141>(b);
    a += dpp_move<0x140>(a); b += dpp_move<0x140>(b);
    a = lane_value(a, 0);
    b = lane_value(b, 0);
}

// sum of every wavefront's v over the wavefronts of a row; all of the work-group take part (several of them to a row)
__device__ __forceinline__ float row_sum(float v, float *lds, int wave, int lane, int first, int waves)
{
    v = wave_sum(v);
    if (waves == 1) return v;
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    return wave_sum(lane < waves ? lds[first + lane] : 0.f);
}

// what a thread has of a vector's gamma or beta: the values, `rest` past the row's end or where there are none
template <int V>
__device__ __forceinline__ void load_affine(const float *p, int at, int left, float rest, float (&v)[V])
{
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = rest;
    if (!p) return;
    if (left >= V) {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            const f32x4 r = *reinterpret_cast<const f32x4_any *>(p + at + h);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h + k] = r[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < left) v[k] = p[at + k];
    }
}

// Up to 16 values to a thread gamma and beta stay in registers; with 32 they are read again for every row, from the cache.  Bound by
// memory: 16384 x 4096 bfloat16 51 us, 5.2 TB/s, as a copy; one row 4 us, most of it the launch.  With 32 values fp32 spills 40 registers
// (bfloat16 2), and the rows take 1.6 to 2 times a copy of their bytes: 2000 x 16384 fp32 62 us, 4.2 TB/s, 2000 x 20000 120, 2.7,
// 2000 x 32768 157, 3.3; bfloat16 33, 59 and 78.
template <typename T, int R>
__global__ __launch_bounds__(1024) void layer_norm_fwd_rows(const LayerNormArgs a)
{
    constexpr int V = Vec<T>::V;
    constexpr bool STAY = R * V <= 16;
    __shared__ float lds[2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int group = wave / a.waves, first = group * a.waves;
    const int t = (wave - first) * 64 + lane, step = a.waves * 64;
    float gamma[STAY ? R : 1][V], beta[STAY ? R : 1][V];
    int left[R];                                     // of the row's values, from this vector on
    const bool partial = a.C >= V && a.C % V;        // (the rows of fewer values are read as they are)
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int v = t + r * step;
        left[r] = v < a.vectors ? a.C - v * V : 0;
        if constexpr (STAY) {
            load_affine(a.gamma, v * V, left[r], 1.f, gamma[r]);
            load_affine(a.beta, v * V, left[r], 0.f, beta[r]);
        }
    }
    const int64_t rows = (int64_t)gridDim.x * a.groups;
    typedef RowSource<T, false> X;
    typename X::Raw raw[R], next[R];
    auto load = [&](int64_t row, typename X::Raw (&to)[R]) {
        const X x(a, row);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row < a.N && left[r] > 0) to[r] = x.load(t + r * step, left[r], a.C);
            else to[r] = {};
        }
    };
    load((int64_t)blockIdx.x * a.groups + group, raw);
    for (int64_t base = (int64_t)blockIdx.x * a.groups; base < a.N; base += rows) {
        const int64_t row = base + group;
        load(row + rows, next);
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v[V];
            if (partial && left[r] > 0 && left[r] < V) X::settle(raw[r], V - left[r]);
            Vec<T>::open(raw[r], v);
#pragma unroll
            for (int k = 0; k < V; ++k) s += v[k];
        }
        const float mean = row_sum(s, lds[0], wave, lane, first, a.waves) / (float)a.C;
        s = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v[V];
            Vec<T>::open(raw[r], v);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float d = v[k] - mean;
                s += k < left[r] ? d * d : 0.f;
            }
        }
        const float rstd = 1.f / sqrtf(row_sum(s, lds[1], wave, lane, first, a.waves) * a.inv_c + a.eps);
        if (row < a.N) {
            T *const y = static_cast<T *>(a.out) + row * a.out_stride;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int v = t + r * step;
                float z[V], ga[V], be[V];
                Vec<T>::open(raw[r], z);
                if constexpr (!STAY) {
                    load_affine(a.gamma, v * V, left[r], 1.f, ga);
                    load_affine(a.beta, v * V, left[r], 0.f, be);
                }
#pragma unroll
                for (int k = 0; k < V; ++k)
                    z[k] = (z[k] - mean) * rstd * (STAY ? gamma[STAY ? r : 0][k] : ga[k]) + (STAY ? beta[STAY ? r : 0][k] : be[k]);
                if (left[r] >= V) Vec<T>::store(y + (int64_t)v * V, z);
                else if (left[r] > 0) store_first(y + (int64_t)v * V, z, left[r]);
            }
            if (t == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = next[r];
    }
}

// Rows longer than a work-group keeps: one of 1024 threads to a row, which goes through it three times, four vectors to a thread on
// their way at a time; a vector is summed in fp32 and then in 64 bits, as a row may have any number of them.  Bound by memory and what
// is read again: 2000 x 40000 fp32 218 us, 5.9 TB/s over three reads and a write, bfloat16 108 (value by value 250 and 184).
constexpr int kWideAhead = 4;

template <typename T>
__global__ __launch_bounds__(kWideThreads) void layer_norm_fwd_wide(const LayerNormArgs a)
{
    constexpr int V = Vec<T>::V;
    typedef RowSource<T, false> X;
    __shared__ float lds[2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const X x(a, row);
        T *const y = static_cast<T *>(a.out) + row * a.out_stride;
        auto each = [&](auto use) {
            for (int first = threadIdx.x; first < a.vectors; first += kWideAhead * kWideThreads) {
                typename X::Raw raw[kWideAhead];
#pragma unroll
                for (int u = 0; u < kWideAhead; ++u) {               // past the end the last one again
                    const int v = min(first + u * kWideThreads, a.vectors - 1);
                    raw[u] = x.load(v, a.C - v * V, a.C);
                }
#pragma unroll
                for (int u = 0; u < kWideAhead; ++u) {
                    const int v = first + u * kWideThreads, left = a.C - v * V;
                    if (v >= a.vectors) continue;
                    if (left < V) X::settle(raw[u], V - left);
                    float z[V];
                    Vec<T>::open(raw[u], z);
                    use(v, left, z);
                }
            }
        };
        double sum = 0.0;
        each([&](int, int, const float (&z)[V]) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) s += z[k];
            sum += s;
        });
        const float mean = row_sum((float)sum, lds[0], wave, lane, 0, 16) / (float)a.C;
        sum = 0.0;
        each([&](int, int left, const float (&z)[V]) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float d = z[k] - mean;
                s += k < left ? d * d : 0.f;
            }
            sum += s;
        });
        const float rstd = 1.f / sqrtf(row_sum((float)sum, lds[1], wave, lane, 0, 16) * a.inv_c + a.eps);
        each([&](int v, int left, float (&z)[V]) {
            float gamma[V], beta[V];
            load_affine(a.gamma, v * V, left, 1.f, gamma);
            load_affine(a.beta, v * V, left, 0.f, beta);
#pragma unroll
            for (int k = 0; k < V; ++k) z[k] = (z[k] - mean) * rstd * gamma[k] + beta[k];
            if (left >= V) Vec<T>::store(y + (int64_t)v * V, z);
            else store_first(y + (int64_t)v * V, z, left);
        });
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Sums of 64 columns over the rows from `begin` on, before `end`, by the work-group's wavefronts: a row to each at a time, four
// rows' loads together, and a sum of four rows after the other in 64 bits, as a part may have any number of rows.
template <typename T, bool HELD>
__device__ __forceinline__ void column_sums(const LayerNormArgs &a, int tile, int64_t begin, int64_t end, float *lds, float *dgamma,
                                            float *dbeta)
{
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int c = tile * 64 + lane;
    double sg = 0.0, sb = 0.0;
    if (c < a.C)
        for (int64_t row = begin + wave; row < end; row += 4 * waves) {
            float d[4], x[4], mean[4], rstd[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {            // past the end the last row again, times zero
                const int64_t at = min(row + k * waves, end - 1);
                d[k] = ld_elem(static_cast<const T *>(a.dy) + at * a.dy_stride, c);
                x[k] = RowSource<T, HELD>(a, at).at(c);
                mean[k] = a.mean[at];
                rstd[k] = a.rstd[at];
            }
            float fg = 0.f, fb = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (row + k * waves < end) {
                    fg += d[k] * ((x[k] - mean[k]) * rstd[k]);
                    fb += d[k];
                }
            sg += fg;
            sb += fb;
        }
    lds[wave * 64 + lane] = (float)sg;
    lds[(waves + wave) * 64 + lane] = (float)sb;
    __syncthreads();
    if (wave < 2 && c < a.C) {                       // one wavefront, or two, join them
        for (int which = wave; which < 2; which += waves > 1 ? 2 : 1) {
            double s = 0.0;
            for (int w = 0; w < waves; ++w) s += lds[(which * waves + w) * 64 + lane];
            float *const out = which ? dbeta : dgamma;
            if (out) out[c] = (float)s;
        }
    }
}

// dx, and every work-group's sums of the columns over its rows (SUMS); or, over few rows, dgamma and dbeta by work-groups of their
// own, which read the rows once more, from the cache, and save the launch that joins.  gamma lies in LDS.  With 8 values to a
// thread the next row's are on their way (a call of 8192 x 4096 bfloat16, its columns joined, 44 to 46 us; when it was chosen 43, and
// 56 with 16 values, which leave room for half the wavefronts).
// U rows at a time, with one barrier to all, where a work-group has no more rows side by side.
// Bound by memory between a start and an end of 10 us together, and for few rows by those: 6001 x 5003 bfloat16 from 8 bits 45 us,
// 3.4 TB/s, from 3000 rows on another thousand takes what a copy of its bytes does; 128 x 9216 fp32 8.7 us.
template <typename T, bool HELD, int R, bool SUMS, int U>
__global__ __launch_bounds__(64 * layer_norm_bwd_waves(R * Vec<T>::V)) void layer_norm_bwd_rows(const LayerNormArgs a)
{
    constexpr int V = Vec<T>::V;
    constexpr bool AHEAD = SUMS && R * V <= 8;
    static_assert(U == 1 || AHEAD, "the next rows are on their way too");
    typedef RowSource<T, HELD> X;
    extern __shared__ __attribute__((aligned(16))) float shared[];       // gamma [vectors * V], then [groups][2][vectors * V]
    __shared__ float lds[2][2 * U][16];
    if (!SUMS && (int)blockIdx.x >= a.row_blocks) {
        column_sums<T, HELD>(a, blockIdx.x - a.row_blocks, 0, a.N, shared, a.dgamma, a.dbeta);
        return;
    }
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int group = wave / a.waves, first = group * a.waves;
    const int t = (wave - first) * 64 + lane, step = a.waves * 64;
    const int width = a.vectors * V;
    float dgamma[SUMS ? R : 1][V], dbeta[SUMS ? R : 1][V];
    int left[R];                                     // of the row's values, from this vector on
    const bool partial = a.C >= V && a.C % V;        // (the rows of fewer values are read as they are)
#pragma unroll
    for (int r = 0; r < R; ++r) {
        left[r] = t + r * step < a.vectors ? a.C - (t + r * step) * V : 0;
        if constexpr (SUMS)
#pragma unroll
            for (int k = 0; k < V; ++k) dgamma[r][k] = dbeta[r][k] = 0.f;
    }
    const int64_t rows = (int64_t)a.row_blocks * a.groups * U;
    struct Row {
        typename X::Raw x[R];
        typename Vec<T>::Raw d[R];
        float mean, rstd;
    } now[U], next[U];
    auto load = [&](int64_t row, Row &to) {
        const X x(a, row);
        const T *const dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        const bool live = row < a.N;
        to.mean = live ? a.mean[row] : 0.f;
        to.rstd = live ? a.rstd[row] : 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (live) {                              // a thread without a vector takes x's first one, as said below
                const int v = t + r * step;
                to.x[r] = x.load(left[r] > 0 ? v : 0, left[r] > 0 ? left[r] : a.C, a.C);
                if (left[r] > 0) to.d[r] = a.C >= V ? Vec<T>::load(dy + (v * V - skipped<V>(left[r]))) : Vec<T>::some(dy, a.C);
                else to.d[r] = {};
            } else {
                to.x[r] = {};
                to.d[r] = {};
            }
    };
    const int64_t begin = (int64_t)blockIdx.x * a.groups * U;
#pragma unroll
    for (int u = 0; u < U; ++u) load(begin + u * a.groups + group, now[u]);
    // every thread puts down what it will read itself (rows side by side the same), as loads that do not wait for each other
    float own[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) load_affine(a.gamma, (t + r * step) * V, left[r], 1.f, own[r]);
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (left[r] > 0)
#pragma unroll
            for (int h = 0; h < V; h += 4)
                *reinterpret_cast<f32x4 *>(shared + (t + r * step) * V + h) = f32x4{own[r][h], own[r][h + 1], own[r][h + 2], own[r][h + 3]};
    __syncthreads();
    auto gamma_of = [&](int r, float (&v)[V]) {      // (a thread without a vector reads the first one)
        const float *const p = shared + (left[r] > 0 ? (t + r * step) * V : 0);
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            const f32x4 g = *reinterpret_cast<const f32x4 *>(p + h);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h + k] = g[k];
        }
    };
    int turn = 0;
    for (int64_t base = begin; base < a.N; base += rows, turn ^= 1) {
        if constexpr (AHEAD)
#pragma unroll
            for (int u = 0; u < U; ++u) load(base + rows + u * a.groups + group, next[u]);
        // Past the row's end dy is zero and x one of the row's values, so that xh is finite there where it is in the row, and what is
        // added is zero.  (With zeros for x, xh is mean times rstd, which may be past fp32 where none of the row is, and zero times an
        // infinity is no number.  Masks on xh instead keep it in registers up to the result: 6001 x 5003 bfloat16 from 8 bits 81 us, 49.)
        float s1[U], s2[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Row &row = now[u];
            s1[u] = s2[u] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float x[V], d[V], g[V];
                if (partial && left[r] > 0 && left[r] < V) {
                    X::settle_round(row.x[r], V - left[r]);
                    row.d[r] = move_down(row.d[r], V - left[r]);
                }
                if (a.C < V) {
                    as_branch();
                    X::repeat(row.x[r], a.C);
                }
                X::open(row.x[r], x);
                Vec<T>::open(row.d[r], d);
                gamma_of(r, g);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float xh = (x[k] - row.mean) * row.rstd, gd = d[k] * g[k];
                    s1[u] += gd;
                    s2[u] += gd * xh;
                    if constexpr (SUMS) {
                        dgamma[r][k] += d[k] * xh;
                        dbeta[r][k] += d[k];
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) wave_sums(s1[u], s2[u]);
        if (a.waves > 1) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (lane == 0) { lds[turn][2 * u][wave] = s1[u]; lds[turn][2 * u + 1][wave] = s2[u]; }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s1[u] = lane < a.waves ? lds[turn][2 * u][first + lane] : 0.f;
                s2[u] = lane < a.waves ? lds[turn][2 * u + 1][first + lane] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) row_sums(s1[u], s2[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = base + u * a.groups + group;
            if (at >= a.N) continue;
            Row &row = now[u];
            const float m1 = s1[u] * a.inv_c, m2 = s2[u] * a.inv_c;
            T *const dx = static_cast<T *>(a.out) + at * a.out_stride;
            open_again(row.d);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int v = t + r * step;
                float x[V], d[V], g[V];
                X::open(row.x[r], x);
                Vec<T>::open(row.d[r], d);
                gamma_of(r, g);
#pragma unroll
                for (int k = 0; k < V; ++k) d[k] = row.rstd * (d[k] * g[k] - m1 - (x[k] - row.mean) * row.rstd * m2);
                if (left[r] >= V) Vec<T>::store(dx + (int64_t)v * V, d);
                else if (left[r] > 0) store_first(dx + (int64_t)v * V, d, left[r]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (AHEAD) now[u] = next[u];
            else if (base + rows < a.N) load(base + rows + u * a.groups + group, now[u]);
        }
    }
    if constexpr (SUMS) {
        float *const out = a.part + (int64_t)blockIdx.x * 2 * a.C;
        auto put = [&](float *to, const float (&v)[V], int n) {
            if (n >= V) {
#pragma unroll
                for (int h = 0; h < V; h += 4) *reinterpret_cast<f32x4_any *>(to + h) = f32x4{v[h], v[h + 1], v[h + 2], v[h + 3]};
                return;
            }
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < n) to[k] = v[k];
        };
        if (a.groups > 1) {
            __syncthreads();                         // gamma is no longer needed
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int v = t + r * step;
                if (v < a.vectors) {
                    put(shared + 2 * group * width + v * V, dgamma[r], V);
                    put(shared + (2 * group + 1) * width + v * V, dbeta[r], V);
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < 2 * width; i += blockDim.x) {
                const int c = i < width ? i : i - width;
                float s = 0.f;
                for (int g = 0; g < a.groups; ++g) s += shared[2 * g * width + i];
                if (c < a.C) out[(i < width ? 0 : a.C) + c] = s;
            }
            return;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            put(out + (t + r * step) * V, dgamma[r], left[r]);
            put(out + a.C + (t + r * step) * V, dbeta[r], left[r]);
        }
    }
}

// dx of rows longer than a work-group keeps, as forward, in two passes (2000 x 40000 fp32 with the columns' sums 402 us, 5.6 TB/s over
// three reads of both and a write; bfloat16 229, value by value 270)
template <typename T, bool HELD>
__global__ __launch_bounds__(kWideThreads) void layer_norm_bwd_wide(const LayerNormArgs a)
{
    constexpr int V = Vec<T>::V;
    typedef RowSource<T, HELD> X;
    __shared__ float lds[2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const X x(a, row);
        const T *const dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        T *const dx = static_cast<T *>(a.out) + row * a.out_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        auto each = [&](auto use) {                  // xh and gamma dy of a vector, zeros past the row's end
            for (int first = threadIdx.x; first < a.vectors; first += kWideAhead * kWideThreads) {
                typename X::Raw raw[kWideAhead];
                typename Vec<T>::Raw draw[kWideAhead];
#pragma unroll
                for (int u = 0; u < kWideAhead; ++u) {               // past the end the last one again
                    const int v = min(first + u * kWideThreads, a.vectors - 1), left = a.C - v * V;
                    raw[u] = x.load(v, left, a.C);
                    draw[u] = Vec<T>::load(dy + (v * V - skipped<V>(left)));
                }
#pragma unroll
                for (int u = 0; u < kWideAhead; ++u) {
                    const int v = first + u * kWideThreads, left = a.C - v * V;
                    if (v >= a.vectors) continue;
                    if (left < V) {
                        X::settle(raw[u], V - left);
                        draw[u] = move_down(draw[u], V - left);
                    }
                    float xh[V], g[V], gamma[V];
                    X::open(raw[u], xh);
                    Vec<T>::open(draw[u], g);
                    load_affine(a.gamma, v * V, left, 1.f, gamma);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        xh[k] = k < left ? (xh[k] - mean) * rstd : 0.f;          // (mean times rstd may be past fp32)
                        g[k] *= gamma[k];
                    }
                    use(v, left, xh, g);
                }
            }
        };
        double sum1 = 0.0, sum2 = 0.0;
        each([&](int, int, const float (&xh)[V], const float (&g)[V]) {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                s1 += g[k];
                s2 += g[k] * xh[k];
            }
            sum1 += s1;
            sum2 += s2;
        });
        const float m1 = row_sum((float)sum1, lds[0], wave, lane, 0, 16) * a.inv_c;
        const float m2 = row_sum((float)sum2, lds[1], wave, lane, 0, 16) * a.inv_c;
        each([&](int v, int left, const float (&xh)[V], float (&g)[V]) {
#pragma unroll
            for (int k = 0; k < V; ++k) g[k] = rstd * (g[k] - m1 - xh[k] * m2);
            if (left >= V) Vec<T>::store(dx + (int64_t)v * V, g);
            else store_first(dx + (int64_t)v * V, g, left);
        });
        __syncthreads();
    }
}

// Sums of the columns over a part of the rows, where the rows' own work-groups keep none: x and dy once more, bound by memory (3000 x
// 16384 fp32 with dx 199 us, 5 TB/s over what both read and write)
template <typename T, bool HELD>
__global__ __launch_bounds__(1024) void layer_norm_columns(const LayerNormArgs a)
{
    __shared__ float lds[2 * 16 * 64];
    const int tiles = (a.C + 63) / 64, part = blockIdx.x / tiles;
    const int64_t begin = (int64_t)part * a.rows_per_part;
    float *const out = a.part + (int64_t)part * 2 * a.C;
    column_sums<T, HELD>(a, blockIdx.x - part * tiles, begin, min((int64_t)a.N, begin + a.rows_per_part), lds, out, out + a.C);
}

// dgamma or dbeta from the parts' sums, in 64 bits: 64 columns to a work-group, a wavefront to a sixteenth of the parts (256 parts of
// 5003 columns 4.6 us, little more than a launch)
__global__ __launch_bounds__(1024) void layer_norm_join(const LayerNormArgs a)
{
    __shared__ double lds[16][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    for (int b = blockIdx.x; b < 2 * ((a.C + 63) / 64); b += gridDim.x) {
        const int which = b & 1, c = (b >> 1) * 64 + lane;
        float *const out = which ? a.dbeta : a.dgamma;
        if (!out) continue;
        double s = 0.0;
        if (c < a.C) {
            const float *p = a.part + (int64_t)which * a.C + c;
            const int64_t pitch = 2 * (int64_t)a.C;
            int i = wave;
            for (; i + 48 < a.part_rows; i += 64) {
                const float v[4] = {p[i * pitch], p[(i + 16) * pitch], p[(i + 32) * pitch], p[(i + 48) * pitch]};
#pragma unroll
                for (int k = 0; k < 4; ++k) s += v[k];
            }
            for (; i < a.part_rows; i += 16) s += p[i * pitch];
        }
        lds[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < a.C) {
            s = 0.0;
#pragma unroll
            for (int w = 0; w < 16; ++w) s += lds[w][lane];
            out[c] = (float)s;
        }
        __syncthreads();
    }
}
