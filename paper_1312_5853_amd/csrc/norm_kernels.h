// Group normalisation with an activation, forward and backward.
// Part of train_ops.hip: included there, inside its anonymous namespace.
//
//   mean = sum x / M, var = sum (x - mean)^2 / M, xh = (x - mean) rstd, z = gamma xh + beta, y = act(z)
//   dz = dy act'(z); per channel A = sum dz, B = sum dz xh; m1 = sum_c gamma A / M, m2 = sum_c gamma B / M
//   dx = rstd (gamma dz - m1 - xh m2); dbeta = sum_n A, dgamma = sum_n B

struct NormArgs {
    const void *x, *dy;
    void *out;                       // y or dx
    const float *gamma, *beta;       // nullptr: ones, zeros
    float *mean, *rstd;              // written by the forward kernels (nullptr: not), read by the backward ones
    float *part;                     // backward: [2][N][C], A and B of every sample and channel
    float *dgamma, *dbeta;
    int N, C, S, groups, cpg;
    float eps;
    int act, last;                   // last: channels last
};

__device__ __forceinline__ float act_fwd(float z, int act)
{
    if (act == kActRelu) return z > 0.f ? z : 0.f;
    if (act == kActSilu) return z / (1.f + __expf(-z));
    return z;
}

// dy * act'(z)
__device__ __forceinline__ float act_bwd(float dy, float z, int act)
{
    if (act == kActRelu) return z > 0.f ? dy : 0.f;
    if (act == kActSilu) {
        const float s = 1.f / (1.f + __expf(-z));
        return dy * (s * (1.f + z * (1.f - s)));
    }
    return dy;
}

// sum over a work-group of 256, in a fixed order; every thread gets it
__device__ __forceinline__ float block_sum(float v, float *red)
{
    __syncthreads();
    red[threadIdx.x] = v;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
        __syncthreads();
    }
    return red[0];
}

// element i of (sample n, group g), and its channel
__device__ __forceinline__ int64_t norm_elem(const NormArgs &a, int n, int g, int i, int &c)
{
    if (a.last) {
        c = g * a.cpg + i % a.cpg;
        return ((int64_t)n * a.S + i / a.cpg) * a.C + c;
    }
    c = g * a.cpg + i / a.S;
    return ((int64_t)n * a.C + g * a.cpg) * a.S + i;
}

// one work-group per sample and group, three passes over its values
template <typename T>
__global__ __launch_bounds__(256) void group_norm_fwd_kernel(NormArgs a)
{
    __shared__ float red[256];
    const int n = blockIdx.x / a.groups, g = blockIdx.x % a.groups, M = a.cpg * a.S;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.out);
    int c;
    float s = 0.f;
    for (int i = threadIdx.x; i < M; i += 256) s += ld_elem(x, norm_elem(a, n, g, i, c));
    const float mean = block_sum(s, red) / M;
    s = 0.f;
    for (int i = threadIdx.x; i < M; i += 256) {
        const float d = ld_elem(x, norm_elem(a, n, g, i, c)) - mean;
        s += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(s, red) / M + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
    for (int i = threadIdx.x; i < M; i += 256) {
        const int64_t e = norm_elem(a, n, g, i, c);
        const float z = (ld_elem(x, e) - mean) * rstd * (a.gamma ? a.gamma[c] : 1.f) + (a.beta ? a.beta[c] : 0.f);
        st_elem(y, e, act_fwd(z, a.act));
    }
}

// A and B of a sample's channel, one work-group each
template <typename T>
__global__ __launch_bounds__(256) void group_norm_bwd_sums(NormArgs a)
{
    __shared__ float red[256];
    const int n = blockIdx.x / a.C, c = blockIdx.x % a.C, g = c / a.cpg;
    const float mean = a.mean[(int64_t)n * a.groups + g], rstd = a.rstd[(int64_t)n * a.groups + g];
    const float gamma = a.gamma ? a.gamma[c] : 1.f, beta = a.beta ? a.beta[c] : 0.f;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    float A = 0.f, B = 0.f;
    for (int s = threadIdx.x; s < a.S; s += 256) {
        const int64_t e = a.last ? ((int64_t)n * a.S + s) * a.C + c : ((int64_t)n * a.C + c) * a.S + s;
        const float xh = (ld_elem(x, e) - mean) * rstd, dz = act_bwd(ld_elem(dy, e), gamma * xh + beta, a.act);
        A += dz;
        B += dz * xh;
    }
    A = block_sum(A, red);
    B = block_sum(B, red);
    if (threadIdx.x == 0) {
        a.part[blockIdx.x] = A;
        a.part[(int64_t)a.N * a.C + blockIdx.x] = B;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void group_norm_bwd_kernel(NormArgs a)
{
    __shared__ float red[256];
    const int n = blockIdx.x / a.groups, g = blockIdx.x % a.groups, M = a.cpg * a.S;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    T *dx = static_cast<T *>(a.out);
    const float mean = a.mean[blockIdx.x], rstd = a.rstd[blockIdx.x];
    float p = 0.f, q = 0.f;
    for (int j = threadIdx.x; j < a.cpg; j += 256) {
        const int c = g * a.cpg + j;
        const float gamma = a.gamma ? a.gamma[c] : 1.f;
        p += gamma * a.part[(int64_t)n * a.C + c];
        q += gamma * a.part[(int64_t)(a.N + n) * a.C + c];
    }
    const float m1 = block_sum(p, red) / M, m2 = block_sum(q, red) / M;
    int c;
    for (int i = threadIdx.x; i < M; i += 256) {
        const int64_t e = norm_elem(a, n, g, i, c);
        const float gamma = a.gamma ? a.gamma[c] : 1.f, beta = a.beta ? a.beta[c] : 0.f;
        const float xh = (ld_elem(x, e) - mean) * rstd, dz = act_bwd(ld_elem(dy, e), gamma * xh + beta, a.act);
        st_elem(dx, e, rstd * (gamma * dz - m1 - xh * m2));
    }
}

// sums over the samples, in order, a thread per channel
__global__ void group_norm_bwd_finish(NormArgs a)
{
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= a.C) return;
    float A = 0.f, B = 0.f;
    for (int n = 0; n < a.N; ++n) {
        A += a.part[(int64_t)n * a.C + c];
        B += a.part[(int64_t)(a.N + n) * a.C + c];
    }
    if (a.dbeta) a.dbeta[c] = A;
    if (a.dgamma) a.dgamma[c] = B;
}
