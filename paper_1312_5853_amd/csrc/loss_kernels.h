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
// joins them and writes the gradient, reading z again.  A large copy moves 5.0 TB/s on this card: both on 2048 x 65536 bf16
// take 111 us, 4.8 TB/s, the gradient alone on 700 x 32003 fp32 39 us, 4.6 TB/s.  Smaller calls are bound by latency: targets
// and row, then what the targets name, then the joins; 4096 x 1000 bf16, loss alone, 7 us, 128 x 1000 fp32, both, 5.4 us,
// 33 x 50021 fp32, both, 4.2 us for the sums and 7.9 for the rest.
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
            if (k >= l.k0 && k < l.k1) Vec<T>::put(dz, l.off + k, v[k]);
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
// and a factor 2^-(m c - mc) on their sum puts it right.  (`fix` is that factor.)  It is half an ulp of mc at most, and has
// to stay small for that: see kFar.
struct Scale { float c, mc, fix; };

__device__ __forceinline__ Scale scale_of(float c, float m)
{
    const float mc = m * c;
    return {c, mc, exp2_of(-fmaf(m, c, -mc))};
}

// Which exponentials a row needs: kOne: one of them (only one term has a target, or T = 1: they are the same); kTwo: both;
// kSquare, kFourth: both, with T = 2 or 4: exp(z - m) is then the second or fourth power of exp((z - m) / T), one
// exponential (four times a vector operation) and a multiplication or two instead of two exponentials.  kFar: both, the
// maximum taken off first; for maxima whose product with c is kFarFrom or more (a share of a row at a mask's -1e9 or at the
// type's lowest value, say).  Below that m c - mc is 1/4 at most, so that the exponentials, their fourth powers and `fix`'s
// stay within a factor of 2 of those relative to m; at 2^32 the difference passes 128 and an exponential the range.
enum { kOne, kTwo, kSquare, kFourth, kFar };
constexpr float kFarFrom = 8388608.f;                    // 2^23

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
        if (!(fabsf(t.mc) < kFarFrom && fabsf(o.mc) < kFarFrom)) {
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
// The threads that work on a row: a wave (SOLO: four rows to a work-group, LDS to each, no barrier), or a work-group
// ---------------------------------------------------------------------------
template <bool SOLO>
struct RowTeam {
    int lane, wave, waves, id, size;        // id, size: the thread in the team, its threads
    __device__ __forceinline__ RowTeam()
    {
        lane = threadIdx.x & 63;
        wave = SOLO ? 0 : uniform((int)(threadIdx.x >> 6));
        waves = SOLO ? 1 : (int)(blockDim.x >> 6);
        id = SOLO ? lane : (int)threadIdx.x;
        size = waves * 64;
    }
    // what a lane has read or written before, in LDS or memory, is done for the others of the team afterwards
    __device__ __forceinline__ void sync() const
    {
        if (SOLO) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
};

// The row's entries in LDS: classes and probabilities, by fours (class -1, probability 0 after the last), then the
// student's logits there.
struct Entries {
    int *idx;
    float *prob, *zk;
};

__device__ __forceinline__ int entry_floats(int K) { return 3 * ((K + 3) & ~3); }

__device__ __forceinline__ Entries entries_at(float *lds, int K)
{
    const int k4 = (K + 3) & ~3;
    return {reinterpret_cast<int *>(lds), lds + k4, lds + 2 * k4};
}

// A row's label and the first 64 entries, one to a lane.  Asked for before the row, as loads come back in order and what the
// entries name is read next.  (The width of an index and the type of a teacher's logit are known at run time only, and behind
// each such branch its load is waited for: the index, and a bfloat16 teacher's logit, are there before the row is asked for.)
struct Targets {
    int label, v;                    // classes, or -1
    float t;                         // the teacher's logit
    __device__ __forceinline__ Targets(const LossArgs &a, int n, int lane)
    {
        label = a.labels ? class_at(a.labels, n, a.wide_index, a.V) : -1;
        v = -1;
        t = -INFINITY;
        if (lane < a.K) {
            v = class_at(a.top_idx, (int64_t)n * a.K + lane, a.wide_index, a.V);
            t = teacher_logit(a, (int64_t)n * a.K + lane);
        }
    }
    // whether an entry of the row names a class; every wave finds out for itself
    __device__ __forceinline__ bool any(const LossArgs &a, int n, int lane) const
    {
        bool has = v >= 0;
        for (int k = lane + 64; k < a.K; k += 64) has |= class_at(a.top_idx, (int64_t)n * a.K + k, a.wide_index, a.V) >= 0;
        return __any(has);
    }
};

// One wave fills the entries in and takes the teacher's softmax.  zk: the student's logit where the class lies in [lo, hi).
template <typename T>
__device__ __forceinline__ void read_entries(const LossArgs &a, const Entries &e, const Targets &first, const T *z, int n, int lo, int hi,
                                             int lane)
{
    const int k4 = (a.K + 3) & ~3;
    float tm = -INFINITY;
    if (a.K <= 64 && lane < k4) {
        tm = first.v < 0 ? -INFINITY : first.t;
        e.zk[lane] = first.v >= lo && first.v < hi ? ld_elem(z, first.v) : 0.f;
        e.idx[lane] = first.v;
        e.prob[lane] = tm;
    }
    for (int k0 = lane; k0 < k4 && a.K > 64; k0 += 256) {    // four entries of a lane at a time, their loads in flight together
        int v[4];
        float t[4], zk[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = k0 + 64 * u;
            v[u] = k < 64 ? first.v : -1;
            t[u] = k < 64 ? first.t : -INFINITY;
            if (k >= 64 && k < a.K) {
                v[u] = class_at(a.top_idx, (int64_t)n * a.K + k, a.wide_index, a.V);
                t[u] = teacher_logit(a, (int64_t)n * a.K + k);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) zk[u] = v[u] >= lo && v[u] < hi ? ld_elem(z, v[u]) : 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = k0 + 64 * u;
            if (v[u] < 0) t[u] = -INFINITY;
            if (k < k4) {
                e.zk[k] = zk[u];
                e.idx[k] = v[u];
                e.prob[k] = t[u];
                tm = fmaxf(tm, t[u]);
            }
        }
    }
    tm = wave_max(tm);
    float ts = 0.f;
    for (int k = lane; k < k4; k += 64) {
        const float p = e.idx[k] >= 0 ? exp2_of((e.prob[k] - tm) * a.to_2T) : 0.f;
        e.prob[k] = p;
        ts += p;
    }
    ts = wave_sum(ts);
    for (int k = lane; k < k4; k += 64)
        if (e.idx[k] >= 0) e.prob[k] /= ts;
}

// The wave that has filled the entries in: T sum_k p_k (log p_k - log q_k), as sum_k p_k (T (log p_k + log sT) - (z_k - m)),
// in which no distance is divided by a small T; zk from `named` where given (the first 64 in `early`).
__device__ __forceinline__ float divergence(const LossArgs &a, const Entries &e, const float *named, float early, float m, float sT,
                                            int lane)
{
    float kd = 0.f;
    const float log_sT = logf(sT);
    for (int k = lane; k < a.K; k += 64) {
        const float p = e.prob[k], zk = !named ? e.zk[k] : k < 64 ? early : named[k];
        if (e.idx[k] >= 0 && !(p <= 0.f)) kd += p * (a.T * (logf(p) + log_sT) - (zk - m));
    }
    return wave_sum(kd);
}

// the classes in [lo, hi) that the targets name, whole
template <typename T, bool SOLO>
__device__ __forceinline__ void write_named(const RowTeam<SOLO> &team, const Entries &e, int K, T *dz, int label, float zl, int lo,
                                            int hi, const RowExps &x, float ck, float cl, float share, float gl)
{
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    for (int k = team.id; k <= K; k += team.size) {
        const int v = k < K ? e.idx[k] : label;
        if (v < lo || v >= hi) continue;
        float p = 0.f;
        bool first = true;
#pragma unroll 4
        for (int j = 0; j < K; j += 4) {
            const i32x4 i4 = *reinterpret_cast<const i32x4 *>(e.idx + j);
            const f32x4 p4 = *reinterpret_cast<const f32x4 *>(e.prob + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p += i4[i] == v ? p4[i] : 0.f;
                first &= i4[i] != v || j + i >= k;
            }
        }
        if (first) Vec<T>::put(dz, v, x.mix(k < K ? e.zk[k] : zl, ck, cl) - (share * p + (v == label ? gl : 0.f)));
    }
}

// Joins m, sT and s1 of `count` parts (three floats each at p) over the lanes of a wave; sums relative to the maximum of all.
__device__ __forceinline__ void join_parts(const LossArgs &a, const float *p, int count, int lane, float &m, float &sT, float &s1)
{
    m = -INFINITY;
    for (int i = lane; i < count; i += 64) m = fmaxf(m, p[3 * i]);
    m = wave_max(m);
    sT = s1 = 0.f;
    for (int i = lane; i < count; i += 64) {
        const float d = p[3 * i] - m;
        sT += p[3 * i + 1] * exp2_of(d * a.to_2T);
        s1 += p[3 * i + 2] * exp2_of(d * a.to_21);
    }
    sT = wave_sum(sT);
    s1 = wave_sum(s1);
}

// A wave's share of a row, relative to its own maximum (so no barrier stands between maximum and sums).  A share without any
// class has sums of 0.
template <typename T, int R>
__device__ __forceinline__ void share_sums(const LossArgs &a, typename Vec<T>::Raw (&raw)[R], bool temp, bool one, float &m, float &sT,
                                           float &s1)
{
    m = wave_max(row_max<T, R>(raw));
    const RowExps x(a, m == -INFINITY ? 0.f : m, temp, one);
    sT = s1 = 0.f;
    open_again(raw);
    x.template sums<T, R>(raw, sT, s1);
    sT = wave_sum(sT);
    s1 = wave_sum(s1);
    x.finish(sT, s1);
}

// ---------------------------------------------------------------------------
// Whole rows: loss (and statistics), and with GRAD the gradient
// ---------------------------------------------------------------------------
// The bound on the registers, for as many wavefronts as hide the reads, costs the instances with 8 vectors two registers (fp32
// with a gradient four) that go to memory and back.
template <typename T, int R, bool SOLO, bool GRAD>
__global__ __launch_bounds__(SOLO ? 256 : 1024, GRAD ? 8 : 6) void distill_rows(LossArgs a)
{
    extern __shared__ float lds[];
    __shared__ float shares[16 * 3];
    const RowTeam<SOLO> team;
    const int n = SOLO ? uniform((int)(blockIdx.x * 4 + (threadIdx.x >> 6))) : (int)blockIdx.x;
    if (SOLO && n >= a.N) return;
    const T *z = static_cast<const T *>(a.z) + n * a.z_stride;
    T *dz = static_cast<T *>(a.dz) + n * a.dz_stride;
    const int c0 = team.wave * a.run, cn = min(a.run, a.chunks - c0);
    const Targets targets(a, n, team.lane);
    typename Vec<T>::Raw raw[R];
    row_read<T, R>(raw, z, a.V, c0, cn, team.lane);
    const int label = targets.label;
    const bool has = targets.any(a, n, team.lane);
    if (!has && label < 0) {                              // nothing to learn from, whatever the logits are
        if (team.id == 0) a.loss[n] = 0.f;
        if (a.stats && team.id < 3) a.stats[(int64_t)n * 3 + team.id] = 0.f;
        if (GRAD) row_clear<T, R>(a, dz, c0, cn, team.lane);
        return;
    }
    const float zl = label >= 0 ? ld_elem(z, label) : 0.f;
    const Entries e = entries_at(lds + (SOLO ? (int)(threadIdx.x >> 6) * entry_floats(a.K) : 0), a.K);
    if (has && team.wave == 0) read_entries(a, e, targets, z, n, 0, a.V, team.lane);
    // statistics are asked for whole; without them a term without target needs no sum
    const bool temp = a.K > 0 && (has || a.stats), one = label >= 0 || a.stats;
    float m, sT, s1;
    share_sums<T, R>(a, raw, temp, one, m, sT, s1);
    if (!SOLO) {
        if (team.lane == 0) {
            shares[3 * team.wave] = m;
            shares[3 * team.wave + 1] = sT;
            shares[3 * team.wave + 2] = s1;
        }
        __syncthreads();                                  // also: the row is read, the entries are there
        join_parts(a, shares, team.waves, team.lane, m, sT, s1);
    } else {
        if (m == -INFINITY) sT = s1 = NAN;                // no class left
        team.sync();
    }
    if (!a.K) sT = s1;
    const RowExps x(a, m, has, label >= 0);
    float gk = 0.f, gl = 0.f, ck = 0.f, cl = 0.f;
    if (GRAD) {
        const float g = a.grad_scale * (a.grad ? a.grad[n] : 1.f);
        if (has) { gk = g * a.wk * a.T; ck = gk / sT; }
        if (label >= 0) { gl = g * a.wl; cl = gl / s1; }
        x.factors(ck, cl);
        open_again(raw);
        x.template write<T, R>(a, raw, dz, c0, cn, team.lane, ck, cl);
    }
    if (team.wave == 0) {
        const float kd = has ? divergence(a, e, nullptr, 0.f, m, sT, team.lane) : 0.f;
        if (team.lane == 0) {
            a.loss[n] = (has ? a.wk * a.T * kd : 0.f) + (label >= 0 ? a.wl * (logf(s1) - (zl - m)) : 0.f);
            if (a.stats) {
                a.stats[(int64_t)n * 3] = m;
                a.stats[(int64_t)n * 3 + 1] = sT;
                a.stats[(int64_t)n * 3 + 2] = s1;
            }
        }
    }
    if (GRAD) {
        team.sync();                                      // the softmax's share is written: the targets' classes may be again
        write_named(team, e, has ? a.K : 0, dz, label, zl, 0, a.V, x, ck, cl, gk, gl);
    }
}

// ---------------------------------------------------------------------------
// Parts of rows
// ---------------------------------------------------------------------------
// m, sT and s1 of a part; the first part's work-group also puts aside the logits that the targets name, as the gradient
// may take their place.
template <typename T, int R>
__global__ __launch_bounds__(256, 8) void distill_part_sums(LossArgs a)
{
    __shared__ float shares[4 * 3];
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
    float m, sT, s1;
    share_sums<T, R>(a, raw, a.K > 0, true, m, sT, s1);
    if (team.lane == 0) {
        shares[3 * team.wave] = m;
        shares[3 * team.wave + 1] = sT;
        shares[3 * team.wave + 2] = s1;
    }
    __syncthreads();
    if (team.wave > 0) return;
    join_parts(a, shares, team.waves, team.lane, m, sT, s1);
    if (m == -INFINITY && sT != sT) {                    // no class in the part (or a NaN in it, which the sums of a wave tell)
        bool nan = false;
        for (int i = team.lane; i < team.waves; i += 64) nan |= shares[3 * i + 2] != shares[3 * i + 2];
        if (!__any(nan)) sT = s1 = 0.f;
    }
    if (team.lane == 0) {
        float *p = a.part + (int64_t)blockIdx.x * 3;
        p[0] = m;
        p[1] = sT;
        p[2] = s1;
    }
}

// With dz in z's place another part's work-group may have written over what a part's moved-back last vector reads of that
// part; those values are dropped, and no other value is read that another work-group writes.
// Joins the parts (or takes the statistics given).  GRAD: a work-group writes its part's gradient, and the first part's
// also the row's loss where asked for; otherwise one work-group per row writes the loss.  The targets and the parts' maxima
// and sums, which come before the row, are three trips to memory one after the other.
template <typename T, int R, bool GRAD>
__global__ __launch_bounds__(256, 8) void distill_part_apply(LossArgs a)
{
    constexpr int V = Vec<T>::V;
    extern __shared__ float lds[];
    const RowTeam<false> team;
    const int n = GRAD ? fastdiv(blockIdx.x, a.div_parts) : (int)blockIdx.x, part = GRAD ? blockIdx.x - n * a.parts : 0;
    const T *z = static_cast<const T *>(a.z) + n * a.z_stride;
    T *dz = static_cast<T *>(a.dz) + n * a.dz_stride;
    const int first = part * a.part_chunks, last = min(first + a.part_chunks, a.chunks);
    const int c0 = first + team.wave * a.run, cn = min(a.run, last - c0);
    const bool lead = part == 0 && a.loss;
    const float *named = a.named + (int64_t)n * (a.K + 1);
    const Targets targets(a, n, team.lane);
    const float early = lead && team.lane < a.K ? named[team.lane] : 0.f, named_label = lead ? named[a.K] : 0.f;
    float m, sT, s1;
    if (a.row_stats) {
        m = a.row_stats[(int64_t)n * 3];
        sT = a.row_stats[(int64_t)n * 3 + 1];
        s1 = a.row_stats[(int64_t)n * 3 + 2];
    } else {
        join_parts(a, a.part + (int64_t)n * a.parts * 3, a.parts, team.lane, m, sT, s1);
        if (!a.K) sT = s1;
    }
    typename Vec<T>::Raw raw[R];
    if (GRAD) row_read<T, R>(raw, z, a.V, c0, cn, team.lane);
    // classes [lo, hi) are this work-group's to write
    const int lo = first * 64 * V, hi = (int)min((int64_t)last * 64 * V, (int64_t)a.V);
    const int label = targets.label;
    const bool has = targets.any(a, n, team.lane);
    if (!has && label < 0) {
        if (lead && team.id == 0) a.loss[n] = 0.f;
        if (lead && a.stats && team.id < 3) a.stats[(int64_t)n * 3 + team.id] = 0.f;
        if (GRAD) row_clear<T, R>(a, dz, c0, cn, team.lane);
        return;
    }
    const float zl = GRAD && label >= lo && label < hi ? ld_elem(z, label) : 0.f;
    const Entries e = entries_at(lds, a.K);
    if (has && team.wave == 0) read_entries(a, e, targets, z, n, GRAD ? lo : 0, GRAD ? hi : 0, team.lane);
    const RowExps x(a, m, has, label >= 0);
    float gk = 0.f, gl = 0.f, ck = 0.f, cl = 0.f;
    if (GRAD) {
        const float g = a.grad_scale * (a.grad ? a.grad[n] : 1.f);
        if (has) { gk = g * a.wk * a.T; ck = gk / sT; }
        if (label >= 0) { gl = g * a.wl; cl = gl / s1; }
        x.factors(ck, cl);
        __syncthreads();                                  // the logits that targets name are read: their places may be written
        x.template write<T, R>(a, raw, dz, c0, cn, team.lane, ck, cl);
    }
    if (lead && team.wave == 0) {
        const float kd = has ? divergence(a, e, named, early, m, sT, team.lane) : 0.f;
        if (team.lane == 0) {
            a.loss[n] = (has ? a.wk * a.T * kd : 0.f) + (label >= 0 ? a.wl * (logf(s1) - (named_label - m)) : 0.f);
            if (a.stats) {
                a.stats[(int64_t)n * 3] = m;
                a.stats[(int64_t)n * 3 + 1] = sT;
                a.stats[(int64_t)n * 3 + 2] = s1;
            }
        }
    }
    if (GRAD) {
        __syncthreads();                                  // the softmax's share is written: the targets' classes may be again
        write_named(team, e, has ? a.K : 0, dz, label, zl, lo, hi, x, ck, cl, gk, gl);
    }
}
