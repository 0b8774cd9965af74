// Layer normalisation: forward, and backward from the values themselves or from values held in blocks of 8 bits.
// Part of block_ops.hip: included there, inside its anonymous namespace, after block_formats.h.
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  xh = (x - mean) rstd,  y = gamma xh + beta
//   g = gamma dy,  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//
// A row is read once and kept in registers (R vectors to a thread) from its sums to its result.  `waves` wavefronts take a row,
// as many rows as fit run side by side in a work-group, and a work-group goes through rows so far apart as there are: gamma,
// beta and the sums of the columns stay in its registers.
struct LayerNormArgs {
    const void *x, *dy;
    const unsigned char *codes, *scales;     // x in blocks
    void *out;                               // y or dx
    const float *gamma, *beta;
    float *mean, *rstd, *dgamma, *dbeta;
    float *part;                             // [part_rows][2][C]: sums of columns over a part of the rows, dgamma's and dbeta's
    int64_t x_stride, dy_stride, out_stride;
    int64_t pitch;                           // values from row to row of the codes
    int N, C;
    int vectors;                             // of a row, the last one perhaps part of one
    int waves, groups;                       // wavefronts to a row, rows side by side
    int part_rows, rows_per_part;
    int row_blocks;                          // work-groups that take rows; those after them take columns
    float inv_c, eps;
};

// vectors of x of one row: of an array, or of codes
template <typename T, bool HELD>
struct RowSource;

template <typename T>
struct RowSource<T, false> {
    typedef typename Vec<T>::Raw Raw;
    const T *p;
    __device__ __forceinline__ RowSource(const LayerNormArgs &a, int64_t row) : p(static_cast<const T *>(a.x) + row * a.x_stride) {}
    __device__ __forceinline__ Raw load(int v, int n) const
    {
        return n >= Vec<T>::V ? Vec<T>::load(p + (int64_t)v * Vec<T>::V) : Vec<T>::some(p + (int64_t)v * Vec<T>::V, n);
    }
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
    __device__ __forceinline__ Raw load(int v, int) const     // rows are filled up: whole vectors
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

// sum of every wavefront's v over the wavefronts of a row; all of the work-group take part (several of them to a row)
__device__ __forceinline__ float row_sum(float v, float *lds, int wave, int lane, int first, int waves)
{
    v = wave_sum(v);
    if (waves == 1) return v;
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    return wave_sum(lane < waves ? lds[first + lane] : 0.f);
}

template <typename T, int R>
__global__ __launch_bounds__(1024) void layer_norm_fwd_rows(const LayerNormArgs a)
{
    constexpr int V = Vec<T>::V;
    __shared__ float lds[2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int group = wave / a.waves, first = group * a.waves;
    const int t = (wave - first) * 64 + lane, step = a.waves * 64;
    float gamma[R][V], beta[R][V];
    int left[R];                                     // of the row's values, from this vector on
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int v = t + r * step;
        left[r] = v < a.vectors ? a.C - v * V : 0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            gamma[r][k] = k < left[r] && a.gamma ? a.gamma[v * V + k] : 1.f;
            beta[r][k] = k < left[r] && a.beta ? a.beta[v * V + k] : 0.f;
        }
    }
    const int64_t rows = (int64_t)gridDim.x * a.groups;
    for (int64_t base = (int64_t)blockIdx.x * a.groups; base < a.N; base += rows) {
        const int64_t row = base + group;
        const bool live = row < a.N;
        const RowSource<T, false> x(a, row);
        typename Vec<T>::Raw raw[R];
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = x.load(t + r * step, live ? left[r] : 0);
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v[V];
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
        if (!live) continue;
        T *const y = static_cast<T *>(a.out) + row * a.out_stride;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int v = t + r * step;
            float w[V];
            Vec<T>::open(raw[r], w);
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = (w[k] - mean) * rstd * gamma[r][k] + beta[r][k];
            if (left[r] >= V) Vec<T>::store(y + (int64_t)v * V, w);
            else
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (k < left[r]) Vec<T>::put(y + (int64_t)v * V, k, w[k]);
        }
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows longer than a work-group keeps: one of 1024 threads to a row, which goes through it three times.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_fwd_wide(const LayerNormArgs a)
{
    __shared__ float lds[2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const T *const x = static_cast<const T *>(a.x) + row * a.x_stride;
        T *const y = static_cast<T *>(a.out) + row * a.out_stride;
        // a thread's sums run over C / 1024 values: in 64 bits
        double s = 0.0;
        for (int c = threadIdx.x; c < a.C; c += 1024) s += ld_elem(x, c);
        const float mean = row_sum((float)s, lds[0], wave, lane, 0, 16) / (float)a.C;
        s = 0.0;
        for (int c = threadIdx.x; c < a.C; c += 1024) {
            const float d = ld_elem(x, c) - mean;
            s += d * d;
        }
        const float rstd = 1.f / sqrtf(row_sum((float)s, lds[1], wave, lane, 0, 16) * a.inv_c + a.eps);
        for (int c = threadIdx.x; c < a.C; c += 1024)
            Vec<T>::put(y + c, 0, (ld_elem(x, c) - mean) * rstd * (a.gamma ? a.gamma[c] : 1.f) + (a.beta ? a.beta[c] : 0.f));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// dx, and every work-group's sums of the columns over its rows
template <typename T, bool HELD, int R>
__global__ __launch_bounds__(1024) void layer_norm_bwd_rows(const LayerNormArgs a)
{
    constexpr int V = Vec<T>::V;
    typedef RowSource<T, HELD> X;
    extern __shared__ float joined[];                // [groups][2][vectors * V] when several rows run side by side
    __shared__ float lds[2][2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int group = wave / a.waves, first = group * a.waves;
    const int t = (wave - first) * 64 + lane, step = a.waves * 64;
    float gamma[R][V], dgamma[R][V], dbeta[R][V];
    int left[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int v = t + r * step;
        left[r] = v < a.vectors ? a.C - v * V : 0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            gamma[r][k] = k < left[r] && a.gamma ? a.gamma[v * V + k] : 1.f;
            dgamma[r][k] = dbeta[r][k] = 0.f;
        }
    }
    const int64_t rows = (int64_t)gridDim.x * a.groups;
    int turn = 0;
    for (int64_t base = (int64_t)blockIdx.x * a.groups; base < a.N; base += rows, turn ^= 1) {
        const int64_t row = base + group;
        const bool live = row < a.N;
        typename X::Raw xr[R];
        typename Vec<T>::Raw dr[R];
        float mean = 0.f, rstd = 0.f;
        if (live) {
            const X x(a, row);
            const T *const dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
            mean = a.mean[row]; rstd = a.rstd[row];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int v = t + r * step;
                if (left[r] > 0) xr[r] = x.load(v, left[r]);
                else xr[r] = {};
                dr[r] = left[r] >= V ? Vec<T>::load(dy + (int64_t)v * V) : Vec<T>::some(dy + (int64_t)v * V, left[r]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) { xr[r] = {}; dr[r] = {}; }
        }
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[V], d[V];
            X::open(xr[r], x);
            Vec<T>::open(dr[r], d);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float xh = k < left[r] ? (x[k] - mean) * rstd : 0.f;
                s1 += d[k] * gamma[r][k];
                s2 += d[k] * gamma[r][k] * xh;
                dgamma[r][k] += d[k] * xh;
                dbeta[r][k] += d[k];
            }
        }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if (a.waves > 1) {
            if (lane == 0) { lds[turn][0][wave] = s1; lds[turn][1][wave] = s2; }
            __syncthreads();
            s1 = wave_sum(lane < a.waves ? lds[turn][0][first + lane] : 0.f);
            s2 = wave_sum(lane < a.waves ? lds[turn][1][first + lane] : 0.f);
        }
        if (!live) continue;
        s1 *= a.inv_c;
        s2 *= a.inv_c;
        T *const dx = static_cast<T *>(a.out) + row * a.out_stride;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int v = t + r * step;
            float x[V], d[V];
            X::open(xr[r], x);
            Vec<T>::open(dr[r], d);
#pragma unroll
            for (int k = 0; k < V; ++k) d[k] = rstd * (d[k] * gamma[r][k] - s1 - (x[k] - mean) * rstd * s2);
            if (left[r] >= V) Vec<T>::store(dx + (int64_t)v * V, d);
            else
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (k < left[r]) Vec<T>::put(dx + (int64_t)v * V, k, d[k]);
        }
    }
    if (!a.part) return;
    const int width = a.vectors * V;
    if (a.groups > 1) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int v = t + r * step;
            if (v < a.vectors)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    joined[(2 * group) * width + v * V + k] = dgamma[r][k];
                    joined[(2 * group + 1) * width + v * V + k] = dbeta[r][k];
                }
        }
        __syncthreads();
        float *const out = a.part + (int64_t)blockIdx.x * 2 * a.C;
        for (int i = threadIdx.x; i < 2 * width; i += blockDim.x) {
            const int c = i < width ? i : i - width;
            float s = 0.f;
            for (int g = 0; g < a.groups; ++g) s += joined[2 * g * width + i];
            if (c < a.C) out[(i < width ? 0 : a.C) + c] = s;
        }
        return;
    }
    float *const out = a.part + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < left[r]) {
                out[(t + r * step) * V + k] = dgamma[r][k];
                out[a.C + (t + r * step) * V + k] = dbeta[r][k];
            }
}

// dx of rows longer than a work-group keeps
template <typename T, bool HELD>
__global__ __launch_bounds__(1024) void layer_norm_bwd_wide(const LayerNormArgs a)
{
    __shared__ float lds[2][16];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const RowSource<T, HELD> x(a, row);
        const T *const dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        T *const dx = static_cast<T *>(a.out) + row * a.out_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        double s1 = 0.0, s2 = 0.0;
        for (int c = threadIdx.x; c < a.C; c += 1024) {
            const float g = ld_elem(dy, c) * (a.gamma ? a.gamma[c] : 1.f);
            s1 += g;
            s2 += g * ((x.at(c) - mean) * rstd);
        }
        const float m1 = row_sum((float)s1, lds[0], wave, lane, 0, 16) * a.inv_c;
        const float m2 = row_sum((float)s2, lds[1], wave, lane, 0, 16) * a.inv_c;
        for (int c = threadIdx.x; c < a.C; c += 1024) {
            const float g = ld_elem(dy, c) * (a.gamma ? a.gamma[c] : 1.f);
            Vec<T>::put(dx + c, 0, rstd * (g - m1 - (x.at(c) - mean) * rstd * m2));
        }
        __syncthreads();
    }
}

// Sums of 64 columns over a part of the rows, a wavefront to a sixteenth of them: where the rows' own work-groups keep none.
template <typename T, bool HELD>
__global__ __launch_bounds__(1024) void layer_norm_columns(const LayerNormArgs a)
{
    __shared__ float lds[2][16][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int tiles = (a.C + 63) / 64;
    const int part = blockIdx.x / tiles, c = (blockIdx.x - part * tiles) * 64 + lane;
    const int64_t end = min((int64_t)a.N, (int64_t)(part + 1) * a.rows_per_part);
    float sg = 0.f, sb = 0.f;
    if (c < a.C)
        for (int64_t row = (int64_t)part * a.rows_per_part + wave; row < end; row += 16) {
            const float d = ld_elem(static_cast<const T *>(a.dy) + row * a.dy_stride, c);
            sg += d * ((RowSource<T, HELD>(a, row).at(c) - a.mean[row]) * a.rstd[row]);
            sb += d;
        }
    lds[0][wave][lane] = sg;
    lds[1][wave][lane] = sb;
    __syncthreads();
    if (wave < 2 && c < a.C) {
        float s = 0.f;
        for (int w = 0; w < 16; ++w) s += lds[wave][w][lane];
        a.part[((int64_t)part * 2 + wave) * a.C + c] = s;
    }
}

// dgamma and dbeta from the parts' sums, in 64 bits: 64 columns to a work-group, a wavefront to a sixteenth of the parts
__global__ __launch_bounds__(1024) void layer_norm_join(const LayerNormArgs a)
{
    __shared__ double lds[16][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int c = blockIdx.x * 64 + lane;
    for (int which = 0; which < 2; ++which) {
        float *const out = which ? a.dbeta : a.dgamma;
        double s = 0.0;
        if (c < a.C)
            for (int p = wave; p < a.part_rows; p += 16) s += a.part[((int64_t)p * 2 + which) * a.C + c];
        lds[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < a.C && out) {
            s = 0.0;
            for (int w = 0; w < 16; ++w) s += lds[w][lane];
            out[c] = (float)s;
        }
        __syncthreads();
    }
}
