// Loss of a row of logits against a label and a teacher's top logits, and its gradient.
// Part of train_ops.hip: included there, inside its anonymous namespace, after vectors.h.
//
//   m = max z, sT = sum exp((z - m) / T), s1 = sum exp(z - m); p = softmax(t / T) over the row's entries
//   loss = wk T^2 sum_k p_k (log p_k - (z_k - m) / T + log sT) + wl (log s1 - (z_label - m))
//   dz = g [wk T (exp((z - m) / T) / sT - p scattered) + wl (exp(z - m) / s1 - onehot)]
// A row's maximum is taken off before the division by T, so no finite logit overflows.  exp(v) is taken as 2^(v log2 e).
//
// Bound by memory: z is read and dz written, once; two exponentials to a value and sum, and two more for the gradient, fit
// beside that.  A row stays in the registers of a wave (SOLO) or a work-group between the reads and the result.  Rows that
// do not fit, and rows too few to fill the card, are cut into parts: one launch leaves each part's m, sT and s1, another
// joins them and writes the gradient, reading z again.
//
// The classes that a target names are written twice: the softmax's share with all the others, then, after a barrier, the
// whole value by the first entry that names the class, which adds up the entries that name it too.  So no atomics, and an
// order that does not change.

struct LossArgs {
    const void *z;
    void *dz;
    int64_t z_stride, dz_stride;
    const void *labels, *top_idx, *top_val;
    float *loss, *stats;
    const float *row_stats;          // backward: what the forward call left
    const float *grad;
    float *part, *named;             // parts: {m, sT, s1}; the logits that the row's targets name (K, then the label's)
    float grad_scale, T, wk, wl;
    float to_2T, to_21;              // log2 e / T, log2 e
    int N, V, K, wide_index, top_bf16;
    int run, parts, part_chunks, chunks;      // vectors of 64 lanes: of a wave, (parts to a row), of a part, of a row
    FastDiv div_parts;
};

// index i of an array of 4- or 8-byte integers; -1 where it names no class
__device__ __forceinline__ int class_at(const void *p, int64_t i, int wide, int V)
{
    const int64_t v = wide ? static_cast<const int64_t *>(p)[i] : (int64_t)static_cast<const int32_t *>(p)[i];
    return v >= 0 && v < V ? (int)v : -1;
}

__device__ __forceinline__ float teacher_logit(const LossArgs &a, int64_t i)
{
    return a.top_bf16 ? ld_elem(static_cast<const unsigned short *>(a.top_val), i)
                      : ld_elem(static_cast<const float *>(a.top_val), i);
}

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// ---------------------------------------------------------------------------
// A row's vectors
// ---------------------------------------------------------------------------
// The last vector is moved back so that it ends where the row ends: its first k0 values are the vector's before it too.
// Lanes past the end hold that vector with no value of their own (k0 = V).
struct RowLane { int off, k0, k1; };

template <int V>
__device__ __forceinline__ RowLane row_lane(int width, int chunk, int lane)
{
    RowLane l;
    const int pos = (chunk * 64 + lane) * V;
    if (width >= V) {
        l.off = min(pos, width - V);
        l.k0 = min(pos - l.off, V);
        l.k1 = V;
    } else {
        l.off = 0;
        l.k0 = 0;
        l.k1 = pos == 0 ? width : 0;
    }
    return l;
}

// A lane's vectors, R from chunk c0 on, n of them the wave's; -infinity (no share in maximum and sums) for values that are
// not the lane's own
template <typename T, int R>
__device__ __forceinline__ void row_read(typename Vec<T>::Raw (&raw)[R], const T *z, int width, int c0, int n, int lane)
{
    constexpr int V = Vec<T>::V;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < n) raw[r] = width >= V ? Vec<T>::load(z + row_lane<V>(width, c0 + r, lane).off) : Vec<T>::some(z, width);
    const int last = (width - 1) / (64 * V);             // the chunk that may hold a moved-back vector
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r >= n || c0 + r >= last) {
            const RowLane l = row_lane<V>(width, c0 + r, lane);
            Vec<T>::drop(raw[r], r < n ? l.k0 : V, l.k1);
        }
}

// (What a moved-back vector does not hold of its own is left to the vector before.)
template <typename T>
__device__ __forceinline__ void row_store(const LossArgs &a, T *dz, const RowLane &l, const float (&v)[Vec<T>::V])
{
    if (l.k0 == 0 && l.k1 == Vec<T>::V) {
        Vec<T>::store(dz + l.off, v);
    } else {
#pragma unroll
        for (int k = 0; k < Vec<T>::V; ++k)
            if (k >= l.k0 && k < l.k1) st_elem(dz, l.off + k, v[k]);
    }
}

// the maximum of a lane's vectors
template <typename T, int R>
__device__ __forceinline__ float row_max(const typename Vec<T>::Raw (&raw)[R])
{
    constexpr int V = Vec<T>::V;
    float m = -INFINITY;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float v[V];
        Vec<T>::open(raw[r], v);
#pragma unroll
        for (int k = 0; k < V; k += 2) m = max3(m, v[k], v[k + 1]);
    }
    return m;
}

// The exponentials of a row, relative to its maximum m.  exp((z - m) / T) is 2^(z c - m c) with c = log2 e / T.  m c is
// rounded to `mc`, so that one multiply-add gives the exponent; what that leaves out, m c - mc, is the same for every value,
// and a factor 2^-(m c - mc) on their sum puts it right.  (`fix` is that factor.)
struct Scale { float c, mc, fix; };

__device__ __forceinline__ Scale scale_of(float c, float m)
{
    const float mc = m * c;
    return {c, mc, exp2_of(-fmaf(m, c, -mc))};
}

// Which exponentials a row needs: kOne: one of them (only one term has a target, or T = 1: they are the same); kTwo: both;
// kSquare, kFourth: both, with T = 2 or 4: exp(z - m) is then the second or fourth power of exp((z - m) / T), one
// exponential (four times a vector operation) and a multiplication or two instead of two exponentials.  kFar: both, the
// maximum taken off first; for maxima whose product with c leaves the range (a row of the type's lowest values, say).
enum { kOne, kTwo, kSquare, kFourth, kFar };

template <int HOW>
__device__ __forceinline__ void add_exps(float v, const Scale &t, const Scale &o, float &sT, float &s1)
{
    if (HOW == kFar) {
        sT += exp2_of((v - t.mc) * t.c);
        s1 += exp2_of((v - t.mc) * o.c);
        return;
    }
    const float e = exp2_of(fmaf(v, t.c, -t.mc));
    sT += e;
    if (HOW == kTwo) s1 += exp2_of(fmaf(v, o.c, -o.mc));
    if (HOW == kSquare) s1 = fmaf(e, e, s1);
    if (HOW == kFourth) s1 = fmaf(e * e, e * e, s1);
}

template <typename T, int R, int HOW>
__device__ __forceinline__ void row_sums(const typename Vec<T>::Raw (&raw)[R], const Scale &t, const Scale &o, float &sT, float &s1)
{
    constexpr int V = Vec<T>::V;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float v[V];
        Vec<T>::open(raw[r], v);
#pragma unroll
        for (int k = 0; k < V; ++k) add_exps<HOW>(v[k], t, o, sT, s1);
        __builtin_amdgcn_sched_barrier(0);               // vectors one after the other: their opened values need registers
    }
}

// dz without the targets: ck exp((z - m) / T) + cl exp(z - m)
template <int HOW>
__device__ __forceinline__ float mix_exps(float v, const Scale &t, const Scale &o, float ck, float cl)
{
    if (HOW == kFar) return exp2_of((v - t.mc) * t.c) * ck + exp2_of((v - t.mc) * o.c) * cl;
    const float e = exp2_of(fmaf(v, t.c, -t.mc));
    if (HOW == kOne) return e * ck;
    if (HOW == kTwo) return fmaf(exp2_of(fmaf(v, o.c, -o.mc)), cl, e * ck);
    if (HOW == kSquare) return e * fmaf(e, cl, ck);
    return e * fmaf(e * e * e, cl, ck);
}

template <typename T, int R, int HOW>
__device__ __forceinline__ void row_write(const LossArgs &a, const typename Vec<T>::Raw (&raw)[R], T *dz, int c0, int n, int lane,
                                          const Scale &t, const Scale &o, float ck, float cl)
{
    constexpr int V = Vec<T>::V;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < n) {
            float v[V];
            Vec<T>::open(raw[r], v);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = mix_exps<HOW>(v[k], t, o, ck, cl);
            row_store(a, dz, row_lane<V>(a.V, c0 + r, lane), v);
            __builtin_amdgcn_sched_barrier(0);
        }
}

// A row's exponentials as its targets need them: sums, gradient of a lane's vectors, and of one value.  temp, one: whether
// exp((z - m) / T), exp(z - m) is needed.
struct RowExps {
    Scale t, o;
    int how;
    bool temp;
    __device__ __forceinline__ RowExps(const LossArgs &a, float m, bool temp_needed, bool one_needed) : temp(temp_needed)
    {
        t = scale_of(temp ? a.to_2T : a.to_21, m);
        o = scale_of(a.to_21, m);
        const bool both = temp_needed && one_needed && a.T != 1.f;
        how = !both ? kOne : a.T == 2.f ? kSquare : a.T == 4.f ? kFourth : kTwo;
        if (!(fabsf(t.mc) < 1e30f && fabsf(o.mc) < 1e30f)) {
            how = kFar;
            t.mc = m;
            t.fix = o.fix = 1.f;
        }
    }
    template <typename T, int R>
    __device__ __forceinline__ void sums(const typename Vec<T>::Raw (&raw)[R], float &sT, float &s1) const
    {
        if (how == kOne) row_sums<T, R, kOne>(raw, t, o, sT, s1);
        else if (how == kTwo) row_sums<T, R, kTwo>(raw, t, o, sT, s1);
        else if (how == kSquare) row_sums<T, R, kSquare>(raw, t, o, sT, s1);
        else if (how == kFourth) row_sums<T, R, kFourth>(raw, t, o, sT, s1);
        else row_sums<T, R, kFar>(raw, t, o, sT, s1);
    }
    __device__ __forceinline__ float one_fix() const
    {
        const float f2 = t.fix * t.fix;
        return how == kSquare ? f2 : how == kFourth ? f2 * f2 : o.fix;
    }
    // the factors of 2^-(m c - mc), on sums of all lanes
    __device__ __forceinline__ void finish(float &sT, float &s1) const
    {
        sT *= t.fix;
        s1 = how == kOne ? sT : s1 * one_fix();
    }
    // ck / sT and cl / s1 as factors of the raw exponentials
    __device__ __forceinline__ void factors(float &ck, float &cl) const
    {
        if (how == kOne) {
            ck = (ck + cl) * t.fix;
            return;
        }
        ck *= t.fix;
        cl *= one_fix();
    }
    template <typename T, int R>
    __device__ __forceinline__ void write(const LossArgs &a, const typename Vec<T>::Raw (&raw)[R], T *dz, int c0, int n, int lane,
                                          float ck, float cl) const
    {
        if (how == kOne) row_write<T, R, kOne>(a, raw, dz, c0, n, lane, t, o, ck, cl);
        else if (how == kTwo) row_write<T, R, kTwo>(a, raw, dz, c0, n, lane, t, o, ck, cl);
        else if (how == kSquare) row_write<T, R, kSquare>(a, raw, dz, c0, n, lane, t, o, ck, cl);
        else if (how == kFourth) row_write<T, R, kFourth>(a, raw, dz, c0, n, lane, t, o, ck, cl);
        else row_write<T, R, kFar>(a, raw, dz, c0, n, lane, t, o, ck, cl);
    }
    __device__ __forceinline__ float mix(float v, float ck, float cl) const
    {
        return how == kOne ? mix_exps<kOne>(v, t, o, ck, cl) : how == kTwo ? mix_exps<kTwo>(v, t, o, ck, cl)
             : how == kSquare ? mix_exps<kSquare>(v, t, o, ck, cl) : how == kFourth ? mix_exps<kFourth>(v, t, o, ck, cl)
             : mix_exps<kFar>(v, t, o, ck, cl);
    }
};

template <typename T, int R>
__device__ __forceinline__ void row_clear(const LossArgs &a, T *dz, int c0, int n, int lane)
{
    constexpr int V = Vec<T>::V;
    const float zero[V] = {};
    for (int r = 0; r < n; ++r) row_store(a, dz, row_lane<V>(a.V, c0 + r, lane), zero);
}

// ---------------------------------------------------------------------------
// The threads that work on a row: a wave (its LDS to itself, no barrier), or a work-group
// ---------------------------------------------------------------------------
template <bool SOLO>
struct RowTeam {
    int lane, wave, waves, id, size;
    __device__ __forceinline__ RowTeam()
    {
        lane = threadIdx.x & 63;
        wave = SOLO ? 0 : uniform((int)(threadIdx.x >> 6));
        waves = SOLO ? 1 : (int)(blockDim.x >> 6);
        id = SOLO ? lane : (int)threadIdx.x;
        size = waves * 64;
    }
    // what a lane has written to LDS or memory is there for the others of the team afterwards
    __device__ __forceinline__ void sync() const
    {
        if (SOLO) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
    // `red`: one float per wave, used by one call between two barriers; a barrier is in the call
    template <int COUNT>
    __device__ __forceinline__ void max_of(float (&v)[COUNT], float (*red)[16]) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = wave_max(v[i]);
        if (SOLO) return;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) red[i][wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = red[i][0];
            for (int w = 1; w < waves; ++w) v[i] = fmaxf(v[i], red[i][w]);
        }
    }
    template <int COUNT>
    __device__ __forceinline__ void sum_of(float (&v)[COUNT], float (*red)[16]) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = wave_sum(v[i]);
        if (SOLO) return;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) red[i][wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = red[i][0];
            for (int w = 1; w < waves; ++w) v[i] += red[i][w];
        }
    }
};

// The row's entries in LDS: classes, probabilities (up to 1 / sum), logits of the student there.
struct Entries { int *idx; float *prob, *zk; };

__device__ __forceinline__ Entries entries_at(float *lds, int K)
{
    return {reinterpret_cast<int *>(lds), lds + K, lds + 2 * K};
}

// Reads a thread's share of the entries; has: whether one names a class; returns the largest of the teacher's logits.
// zk: the student's logit where the class lies in [lo, hi).
template <typename T, bool SOLO>
__device__ __forceinline__ float read_entries(const LossArgs &a, const RowTeam<SOLO> &team, const Entries &e, const T *z, int n, int lo,
                                              int hi, float &has)
{
    float tm = -INFINITY;
    has = 0.f;
    for (int k = team.id; k < a.K; k += team.size) {
        const int64_t i = (int64_t)n * a.K + k;
        const int v = class_at(a.top_idx, i, a.wide_index, a.V);
        const float t = teacher_logit(a, i);
        e.idx[k] = v;
        e.prob[k] = v >= 0 ? t : -INFINITY;
        e.zk[k] = v >= lo && v < hi ? ld_elem(z, v) : 0.f;
        if (v >= 0) {
            has = 1.f;
            tm = fmaxf(tm, t);
        }
    }
    return tm;
}

// exp((t - tm) / T) of a thread's share, into prob; returns their sum
template <bool SOLO>
__device__ __forceinline__ float weigh_entries(const LossArgs &a, const RowTeam<SOLO> &team, const Entries &e, float tm)
{
    float ts = 0.f;
    for (int k = team.id; k < a.K; k += team.size) {
        const float p = e.idx[k] >= 0 ? exp2_of((e.prob[k] - tm) * a.to_2T) : 0.f;
        e.prob[k] = p;
        ts += p;
    }
    return ts;
}

// T sum_k p_k (log p_k - log q_k) over a thread's share, as sum_k p_k (T (log p_k + log sT) - (z_k - m)), in which no
// distance is divided by a small T; zk from `named` where given
template <bool SOLO>
__device__ __forceinline__ float divergence(const LossArgs &a, const RowTeam<SOLO> &team, const Entries &e, const float *named,
                                            float inv_ts, float m, float sT)
{
    float kd = 0.f;
    const float log_sT = logf(sT);
    for (int k = team.id; k < a.K; k += team.size) {
        const float p = e.prob[k] * inv_ts;
        if (e.idx[k] >= 0 && !(p <= 0.f)) kd += p * (a.T * (logf(p) + log_sT) - ((named ? named[k] : e.zk[k]) - m));
    }
    return kd;
}

// the classes in [lo, hi) that the targets name, whole
template <typename T, bool SOLO>
__device__ __forceinline__ void write_named(const LossArgs &a, const RowTeam<SOLO> &team, const Entries &e, T *dz, int label, float zl,
                                            int lo, int hi, const RowExps &x, float ck, float cl, float share, float gl)
{
    for (int k = team.id; k <= a.K; k += team.size) {
        const int v = k < a.K ? e.idx[k] : label;
        if (v < lo || v >= hi) continue;
        float p = 0.f;
        bool first = true;
        for (int j = 0; j < a.K; ++j)
            if (e.idx[j] == v) {
                p += e.prob[j];
                if (j < k) first = false;
            }
        if (first) st_elem(dz, v, x.mix(k < a.K ? e.zk[k] : zl, ck, cl) - (share * p + (v == label ? gl : 0.f)));
    }
}

// ---------------------------------------------------------------------------
// Whole rows: loss (and statistics), and with GRAD the gradient
// ---------------------------------------------------------------------------
template <typename T, int R, bool SOLO, bool GRAD>
__global__ __launch_bounds__(SOLO ? 256 : 1024, GRAD ? 8 : 6) void distill_rows(LossArgs a)
{
    extern __shared__ float lds[];
    __shared__ float red[7][16];
    const RowTeam<SOLO> team;
    const int n = SOLO ? uniform((int)(blockIdx.x * 4 + (threadIdx.x >> 6))) : (int)blockIdx.x;
    if (SOLO && n >= a.N) return;
    const T *z = static_cast<const T *>(a.z) + n * a.z_stride;
    T *dz = static_cast<T *>(a.dz) + n * a.dz_stride;
    const int c0 = team.wave * a.run, cn = min(a.run, a.chunks - c0);
    typename Vec<T>::Raw raw[R];
    row_read<T, R>(raw, z, a.V, c0, cn, team.lane);
    const int label = a.labels ? class_at(a.labels, n, a.wide_index, a.V) : -1;
    const float zl = label >= 0 ? ld_elem(z, label) : 0.f;
    const Entries e = entries_at(lds + (SOLO ? (int)(threadIdx.x >> 6) * 3 * a.K : 0), a.K);
    float most[3];
    most[1] = read_entries(a, team, e, z, n, 0, a.V, most[2]);
    most[0] = row_max<T, R>(raw);
    team.max_of(most, red);
    const float m = most[0], tm = most[1];
    const bool has = most[2] > 0.f;
    if (!has && label < 0) {                              // nothing to learn from, whatever the logits are
        if (team.id == 0) a.loss[n] = 0.f;
        if (a.stats && team.id < 3) a.stats[(int64_t)n * 3 + team.id] = 0.f;
        if (GRAD) row_clear<T, R>(a, dz, c0, cn, team.lane);
        return;
    }
    // statistics are asked for whole; without them a term without target needs no sum
    const RowExps x(a, m, a.K > 0 && (has || a.stats), label >= 0 || a.stats);
    float sums[3] = {0.f, 0.f, 0.f};
    sums[2] = weigh_entries(a, team, e, tm);
    open_again(raw);
    x.template sums<T, R>(raw, sums[0], sums[1]);
    team.sum_of(sums, red + 3);
    float sT = sums[0], s1 = sums[1];
    x.finish(sT, s1);
    const float inv_ts = has ? 1.f / sums[2] : 0.f;
    if (a.stats && team.id == 0) {
        a.stats[(int64_t)n * 3] = m;
        a.stats[(int64_t)n * 3 + 1] = sT;
        a.stats[(int64_t)n * 3 + 2] = s1;
    }
    float gk = 0.f, gl = 0.f, ck = 0.f, cl = 0.f;
    if (GRAD) {
        const float g = a.grad_scale * (a.grad ? a.grad[n] : 1.f);
        if (has) { gk = g * a.wk * a.T; ck = gk / sT; }
        if (label >= 0) { gl = g * a.wl; cl = gl / s1; }
        x.factors(ck, cl);
        open_again(raw);
        x.template write<T, R>(a, raw, dz, c0, cn, team.lane, ck, cl);
    }
    float kd[1] = {has ? divergence(a, team, e, nullptr, inv_ts, m, sT) : 0.f};
    team.sum_of(kd, red + 6);
    if (team.id == 0)
        a.loss[n] = (has ? a.wk * a.T * kd[0] : 0.f) + (label >= 0 ? a.wl * (logf(s1) - (zl - m)) : 0.f);
    if (GRAD) {
        team.sync();
        write_named(a, team, e, dz, label, zl, 0, a.V, x, ck, cl, gk * inv_ts, gl);
    }
}

// ---------------------------------------------------------------------------
// Parts of rows
// ---------------------------------------------------------------------------
// m, sT and s1 of a part; the first part's work-group also puts aside the logits that the targets name, as the gradient
// may take their place.
template <typename T, int R>
__global__ __launch_bounds__(512, 8) void distill_part_sums(LossArgs a)
{
    __shared__ float red[3][16];
    const RowTeam<false> team;
    const int n = fastdiv(blockIdx.x, a.div_parts), part = blockIdx.x - n * a.parts;
    const T *z = static_cast<const T *>(a.z) + n * a.z_stride;
    const int first = part * a.part_chunks, last = min(first + a.part_chunks, a.chunks);
    const int c0 = first + team.wave * a.run, cn = min(a.run, last - c0);
    typename Vec<T>::Raw raw[R];
    row_read<T, R>(raw, z, a.V, c0, cn, team.lane);
    if (part == 0) {
        float *named = a.named + (int64_t)n * (a.K + 1);
        for (int k = team.id; k <= a.K; k += team.size) {
            const int v = k < a.K ? class_at(a.top_idx, (int64_t)n * a.K + k, a.wide_index, a.V)
                                  : a.labels ? class_at(a.labels, n, a.wide_index, a.V) : -1;
            named[k] = v >= 0 ? ld_elem(z, v) : 0.f;
        }
    }
    float m[1] = {row_max<T, R>(raw)};
    team.max_of(m, red);
    float s[2] = {0.f, 0.f};
    // of a part without any class left the sums are 0
    const float top = m[0] == -INFINITY ? 0.f : m[0];
    const RowExps x(a, top, a.K > 0, true);
    open_again(raw);
    x.template sums<T, R>(raw, s[0], s[1]);
    team.sum_of(s, red + 1);
    x.finish(s[0], s[1]);
    if (team.id == 0) {
        float *p = a.part + (int64_t)blockIdx.x * 3;
        p[0] = m[0];
        p[1] = s[0];
        p[2] = s[1];
    }
}

// Joins the parts (or takes the statistics given).  GRAD: a work-group writes its part's gradient, and the first part's
// also the row's loss where asked for; otherwise one work-group per row writes the loss.
template <typename T, int R, bool GRAD>
__global__ __launch_bounds__(512, 8) void distill_part_apply(LossArgs a)
{
    constexpr int V = Vec<T>::V;
    extern __shared__ float lds[];
    __shared__ float red[3][16];
    const RowTeam<false> team;
    const int n = GRAD ? fastdiv(blockIdx.x, a.div_parts) : (int)blockIdx.x, part = GRAD ? blockIdx.x - n * a.parts : 0;
    const T *z = static_cast<const T *>(a.z) + n * a.z_stride;
    T *dz = static_cast<T *>(a.dz) + n * a.dz_stride;
    const int first = part * a.part_chunks, last = min(first + a.part_chunks, a.chunks);
    const int c0 = first + team.wave * a.run, cn = min(a.run, last - c0);
    typename Vec<T>::Raw raw[R];
    if (GRAD) row_read<T, R>(raw, z, a.V, c0, cn, team.lane);
    // classes [lo, hi) are this work-group's to write
    const int lo = first * 64 * V, hi = (int)min((int64_t)last * 64 * V, (int64_t)a.V);
    const int label = a.labels ? class_at(a.labels, n, a.wide_index, a.V) : -1;
    const float zl = GRAD && label >= lo && label < hi ? ld_elem(z, label) : 0.f;
    const Entries e = entries_at(lds, a.K);
    float most[1], dummy;
    most[0] = read_entries(a, team, e, z, n, GRAD ? lo : 0, GRAD ? hi : 0, dummy);
    // every wave for itself: whether an entry names a class
    bool has = false;
    for (int k = team.lane; k < a.K; k += 64) has |= class_at(a.top_idx, (int64_t)n * a.K + k, a.wide_index, a.V) >= 0;
    has = __any(has);
    const bool lead = part == 0 && a.loss;
    if (!has && label < 0) {
        if (lead && team.id == 0) a.loss[n] = 0.f;
        if (lead && a.stats && team.id < 3) a.stats[(int64_t)n * 3 + team.id] = 0.f;
        if (GRAD) row_clear<T, R>(a, dz, c0, cn, team.lane);
        return;
    }
    float m, sT, s1;
    if (a.row_stats) {
        m = a.row_stats[(int64_t)n * 3];
        sT = a.row_stats[(int64_t)n * 3 + 1];
        s1 = a.row_stats[(int64_t)n * 3 + 2];
    } else {
        const float *p = a.part + (int64_t)n * a.parts * 3;
        m = -INFINITY;
        for (int i = team.lane; i < a.parts; i += 64) m = fmaxf(m, p[3 * i]);
        m = wave_max(m);
        sT = s1 = 0.f;
        for (int i = team.lane; i < a.parts; i += 64) {
            const float d = p[3 * i] - m;
            sT += p[3 * i + 1] * exp2_of(d * a.to_2T);
            s1 += p[3 * i + 2] * exp2_of(d * a.to_21);
        }
        sT = wave_sum(sT);
        s1 = wave_sum(s1);
        if (!a.K) sT = s1;
    }
    const RowExps x(a, m, has, label >= 0);
    team.max_of(most, red);                  // (a barrier: the logits that targets name are read, their places may be written)
    float gk = 0.f, gl = 0.f, ck = 0.f, cl = 0.f;
    if (GRAD) {
        const float g = a.grad_scale * (a.grad ? a.grad[n] : 1.f);
        if (has) { gk = g * a.wk * a.T; ck = gk / sT; }
        if (label >= 0) { gl = g * a.wl; cl = gl / s1; }
        x.factors(ck, cl);
        open_again(raw);
        x.template write<T, R>(a, raw, dz, c0, cn, team.lane, ck, cl);
    }
    float ts[1] = {weigh_entries(a, team, e, most[0])};
    team.sum_of(ts, red + 1);                // (a barrier: the softmax's share is written, targets may be written over it)
    const float inv_ts = has ? 1.f / ts[0] : 0.f;
    if (lead) {
        const float *named = a.named + (int64_t)n * (a.K + 1);
        float kd[1] = {has ? divergence(a, team, e, named, inv_ts, m, sT) : 0.f};
        team.sum_of(kd, red + 2);
        if (team.id == 0) {
            a.loss[n] = (has ? a.wk * a.T * kd[0] : 0.f) + (label >= 0 ? a.wl * (logf(s1) - (named[a.K] - m)) : 0.f);
            if (a.stats) {
                a.stats[(int64_t)n * 3] = m;
                a.stats[(int64_t)n * 3 + 1] = sT;
                a.stats[(int64_t)n * 3 + 2] = s1;
            }
        }
    }
    if (GRAD) write_named(a, team, e, dz, label, zl, lo, hi, x, ck, cl, gk * inv_ts, gl);
}
