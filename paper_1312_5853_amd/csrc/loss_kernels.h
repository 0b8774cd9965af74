// Loss of a row of logits against a label and a teacher's top logits, and its gradient.
// Part of train_ops.hip: included there, inside its anonymous namespace.
//
//   m = max z, sT = sum exp((z - m) / T), s1 = sum exp(z - m); p = softmax(t / T) over the row's entries
//   loss = wk T^2 sum_k p_k (log p_k - (z_k - m) / T + log sT) + wl (log s1 - (z_label - m))
//   dz = g [wk T (exp((z - m) / T) / sT - p scattered) + wl (exp(z - m) / s1 - onehot)]
// A row's maximum is taken off before the division by T, so no finite logit overflows.

struct LossArgs {
    const void *z;
    void *dz;
    int64_t z_stride, dz_stride;
    const void *labels, *top_idx, *top_val;
    float *loss, *stats;
    const float *row_stats;          // backward: what the forward call left
    const float *grad;
    float grad_scale, T, inv_T, wk, wl;
    int N, V, K, wide_index, top_bf16;
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

__device__ __forceinline__ float block_max(float v, float *red)
{
    __syncthreads();
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// One work-group per row.  GRAD: dz too; the row's statistics are taken from the row, or from row_stats where given.
template <typename T, bool GRAD>
__global__ __launch_bounds__(256) void distill_rows_kernel(LossArgs a)
{
    __shared__ float red[256];
    __shared__ int idx[CONV_DISTILL_MAX_TOP];
    __shared__ float prob[CONV_DISTILL_MAX_TOP], zk[CONV_DISTILL_MAX_TOP];
    const int n = blockIdx.x, tid = threadIdx.x;
    const T *z = static_cast<const T *>(a.z) + n * a.z_stride;
    T *dz = static_cast<T *>(a.dz) + n * a.dz_stride;
    const int label = a.labels ? class_at(a.labels, n, a.wide_index, a.V) : -1;
    // the teacher's softmax over the entries that name a class
    float tm = -INFINITY, has = 0.f;
    for (int k = tid; k < a.K; k += 256) {
        const int64_t e = (int64_t)n * a.K + k;
        const int v = class_at(a.top_idx, e, a.wide_index, a.V);
        idx[k] = v;
        zk[k] = v >= 0 ? ld_elem(z, v) : 0.f;
        prob[k] = v >= 0 ? teacher_logit(a, e) : -INFINITY;
        if (v >= 0) { has = 1.f; tm = fmaxf(tm, prob[k]); }
    }
    has = block_max(has, red);
    tm = block_max(tm, red);
    const float zl = label >= 0 ? ld_elem(z, label) : 0.f;
    if (has == 0.f && label < 0) {                       // nothing to learn from: the logits are not looked at
        if (a.loss && tid == 0) a.loss[n] = 0.f;
        if (a.stats && tid < 3) a.stats[(int64_t)n * 3 + tid] = 0.f;
        if (GRAD)
            for (int v = tid; v < a.V; v += 256) st_elem(dz, v, 0.f);
        return;
    }
    float ts = 0.f;
    for (int k = tid; k < a.K; k += 256) {
        prob[k] = idx[k] >= 0 ? expf((prob[k] - tm) * a.inv_T) : 0.f;
        ts += prob[k];
    }
    ts = block_sum(ts, red);
    for (int k = tid; k < a.K; k += 256) prob[k] = idx[k] >= 0 ? prob[k] / ts : 0.f;

    float m, sT, s1;
    if (a.row_stats) {
        m = a.row_stats[(int64_t)n * 3];
        sT = a.row_stats[(int64_t)n * 3 + 1];
        s1 = a.row_stats[(int64_t)n * 3 + 2];
    } else {
        m = -INFINITY;
        for (int v = tid; v < a.V; v += 256) m = fmaxf(m, ld_elem(z, v));
        m = block_max(m, red);
        sT = s1 = 0.f;
        for (int v = tid; v < a.V; v += 256) {
            const float d = ld_elem(z, v) - m, e = expf(d);
            s1 += e;
            sT += a.K ? expf(d * a.inv_T) : e;
        }
        sT = block_sum(sT, red);
        s1 = block_sum(s1, red);
    }
    if (a.stats && tid == 0) {
        a.stats[(int64_t)n * 3] = m;
        a.stats[(int64_t)n * 3 + 1] = sT;
        a.stats[(int64_t)n * 3 + 2] = s1;
    }
    if (a.loss) {
        const float lT = logf(sT);
        float kd = 0.f;
        __syncthreads();
        for (int k = tid; k < a.K; k += 256)
            if (idx[k] >= 0 && !(prob[k] <= 0.f)) kd += prob[k] * (logf(prob[k]) - ((zk[k] - m) * a.inv_T - lT));
        kd = block_sum(kd, red);
        if (tid == 0)
            a.loss[n] = (has > 0.f ? a.wk * a.T * a.T * kd : 0.f) + (label >= 0 ? a.wl * (logf(s1) - (zl - m)) : 0.f);
    }
    if (GRAD) {
        const float g = a.grad_scale * (a.grad ? a.grad[n] : 1.f);
        const float gk = has > 0.f ? g * a.wk * a.T : 0.f, gl = label >= 0 ? g * a.wl : 0.f;
        const float ck = gk / sT, cl = gl / s1;
        auto soft = [&](float d) { return (gk != 0.f ? expf(d * a.inv_T) * ck : 0.f) + (gl != 0.f ? expf(d) * cl : 0.f); };
        for (int v = tid; v < a.V; v += 256) st_elem(dz, v, soft(ld_elem(z, v) - m));
        __syncthreads();
        // classes with a target are written again; the first entry that names a class writes it
        for (int k = tid; k <= a.K; k += 256) {
            const int v = k < a.K ? idx[k] : label;
            if (v < 0) continue;
            float p = 0.f;
            bool first = true;
            for (int j = 0; j < a.K; ++j)
                if (idx[j] == v) {
                    p += prob[j];
                    if (j < k) first = false;
                }
            if (!first) continue;
            st_elem(dz, v, soft((k < a.K ? zk[k] : zl) - m) - gk * p - (v == label ? gl : 0.f));
        }
    }
}
