// HIP kernels (gfx950 / CDNA4) and C-ABI entry points of what a training step needs around the convolutions: group
// normalisation with an activation, and the loss against labels and a teacher's top logits.  Signatures and
// conventions are documented in include/convnet_hotpath.h.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>

#include "../../include/convnet_hotpath.h"
#include "host_status.h"

using namespace convnet;

namespace {

constexpr int kActNone = CONV_ACT_NONE, kActRelu = CONV_ACT_RELU, kActSilu = CONV_ACT_SILU;

#include "elements.h"
#include "norm_kernels.h"
#include "loss_kernels.h"

// ---------------------------------------------------------------------------
// Group normalisation
// ---------------------------------------------------------------------------
int norm_checks(int N, int C, int S, int groups, int layout, int dtype)
{
    if (N < 0 || C <= 0 || S <= 0 || groups <= 0 || C % groups) return kErrInvalidArg;
    if (layout != CONV_LAYOUT_PLANES && layout != CONV_LAYOUT_CHANNELS_LAST) return kErrInvalidArg;
    if (!glue_elem_bytes(dtype)) return kErrBadDtype;
    const int64_t limit = (int64_t)1 << 31;
    if ((int64_t)C * S >= limit || (int64_t)N * C >= limit) return kErrTooLarge;
    return kStatusOk;
}

size_t norm_workspace(int op, int N, int C, int S, int groups, int layout, int dtype)
{
    if (norm_checks(N, C, S, groups, layout, dtype) != kStatusOk) return 0;
    if (op != CONV_OP_BWD_DATA) return 0;
    return (size_t)2 * N * C * 4;
}

int norm_common(NormArgs &a, int op, int N, int C, int S, int groups, int act, int layout, int dtype, void *ws,
                size_t ws_bytes)
{
    const int rc = norm_checks(N, C, S, groups, layout, dtype);
    if (rc != kStatusOk) return rc;
    if (act != kActNone && act != kActRelu && act != kActSilu) return kErrInvalidArg;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(a.x, eb) || !aligned(a.dy, eb) || !aligned(a.out, eb)) return kErrMisaligned;
    if (!aligned(a.gamma, 4) || !aligned(a.beta, 4) || !aligned(a.mean, 4) || !aligned(a.rstd, 4) ||
        !aligned(a.dgamma, 4) || !aligned(a.dbeta, 4))
        return kErrMisaligned;
    const size_t need = norm_workspace(op, N, C, S, groups, layout, dtype);
    if (need) {
        if (!ws || ws_bytes < need) return kErrWorkspace;
        if (!aligned(ws, 256)) return kErrMisaligned;
    }
    a.part = static_cast<float *>(ws);
    a.N = N; a.C = C; a.S = S; a.groups = groups; a.cpg = C / groups;
    a.act = act; a.last = layout == CONV_LAYOUT_CHANNELS_LAST;
    return kStatusOk;
}

template <typename T>
int run_norm_fwd(const NormArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(group_norm_fwd_kernel<T>, dim3(a.N * a.groups), dim3(256), 0, st, a);
    return check_launch();
}

template <typename T>
int run_norm_bwd(const NormArgs &a, hipStream_t st)
{
    if (a.N > 0) {
        hipLaunchKernelGGL(group_norm_bwd_sums<T>, dim3(a.N * a.C), dim3(256), 0, st, a);
        hipLaunchKernelGGL(group_norm_bwd_kernel<T>, dim3(a.N * a.groups), dim3(256), 0, st, a);
        const int rc = check_launch();
        if (rc != kStatusOk) return rc;
    }
    if (!a.dgamma && !a.dbeta) return kStatusOk;
    hipLaunchKernelGGL(group_norm_bwd_finish, dim3((a.C + 63) / 64), dim3(64), 0, st, a);
    return check_launch();
}

// ---------------------------------------------------------------------------
// Loss
// ---------------------------------------------------------------------------
int loss_checks(int N, int V, int K, int dtype)
{
    if (N < 0 || V <= 0 || K < 0) return kErrInvalidArg;
    if (!glue_elem_bytes(dtype)) return kErrBadDtype;
    if (K > CONV_DISTILL_MAX_TOP) return kErrTooLarge;
    return kStatusOk;
}

// a: pointers, strides and scalars of the call are set; the rest is checked and filled in
int loss_common(LossArgs &a, bool dz, int N, int V, int K, float temperature, int index_bytes, int top_dtype, int dtype)
{
    if (N != 0 && (!a.z || (dz && !a.dz) || (!a.labels && K == 0) || (K > 0 && (!a.top_idx || !a.top_val))))
        return kErrInvalidArg;
    if (a.z_stride < V || (dz && a.dz_stride < V) || (index_bytes != 4 && index_bytes != 8)) return kErrInvalidArg;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(a.wk) || !isfinite(a.wl) || !isfinite(a.grad_scale))
        return kErrInvalidArg;
    if (N != 0 && dz && a.z == a.dz && a.z_stride != a.dz_stride) return kErrInvalidArg;
    const int rc = loss_checks(N, V, K, dtype);
    if (rc != kStatusOk) return rc;
    const int tb = K ? glue_elem_bytes(top_dtype) : 4;
    if (!tb) return kErrBadDtype;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(a.z, eb) || !aligned(a.dz, eb) || !aligned(a.labels, index_bytes) || !aligned(a.top_idx, index_bytes) ||
        !aligned(a.top_val, tb) || !aligned(a.loss, 4) || !aligned(a.stats, 4) || !aligned(a.row_stats, 4) ||
        !aligned(a.grad, 4))
        return kErrMisaligned;
    a.N = N; a.V = V; a.K = K;
    a.T = temperature; a.inv_T = 1.f / temperature;
    a.wide_index = index_bytes == 8; a.top_bf16 = tb == 2;
    if (a.wk == 0.f) a.K = 0;                            // a term of weight 0 is absent
    if (a.wl == 0.f) a.labels = nullptr;
    return kStatusOk;
}

template <bool GRAD>
int run_loss(const LossArgs &a, int dtype, void *stream)
{
    if (a.N == 0) return kStatusOk;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (glue_elem_bytes(dtype) == 4)
        hipLaunchKernelGGL((distill_rows_kernel<float, GRAD>), dim3(a.N), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((distill_rows_kernel<unsigned short, GRAD>), dim3(a.N), dim3(256), 0, st, a);
    return check_launch();
}

}  // namespace

extern "C" {

size_t group_norm_act_workspace_bytes(int op, int N, int C, int S, int groups, int layout, int dtype)
{
    return norm_workspace(op, N, C, S, groups, layout, dtype);
}

int group_norm_act_fwd(const void *x, const void *gamma, const void *beta, void *y, void *mean, void *rstd, int N, int C,
                       int S, int groups, float eps, int act, int layout, int dtype, void *ws, size_t ws_bytes,
                       void *stream)
{
    if ((N != 0 && (!x || !y || x == y)) || !(eps > 0.f) || !isfinite(eps)) return kErrInvalidArg;
    NormArgs a = {};
    a.x = x; a.out = y; a.eps = eps;
    a.gamma = static_cast<const float *>(gamma); a.beta = static_cast<const float *>(beta);
    a.mean = static_cast<float *>(mean); a.rstd = static_cast<float *>(rstd);
    const int rc = norm_common(a, CONV_OP_FWD, N, C, S, groups, act, layout, dtype, ws, ws_bytes);
    if (rc != kStatusOk) return rc;
    if (N == 0) return kStatusOk;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return glue_elem_bytes(dtype) == 4 ? run_norm_fwd<float>(a, st) : run_norm_fwd<unsigned short>(a, st);
}

int group_norm_act_bwd(const void *x, const void *dy, const void *gamma, const void *beta, const void *mean,
                       const void *rstd, void *dx, void *dgamma, void *dbeta, int N, int C, int S, int groups, int act,
                       int layout, int dtype, void *ws, size_t ws_bytes, void *stream)
{
    if (N != 0 && (!x || !dy || !mean || !rstd || !dx || x == dx || dy == dx)) return kErrInvalidArg;
    NormArgs a = {};
    a.x = x; a.dy = dy; a.out = dx;
    a.gamma = static_cast<const float *>(gamma); a.beta = static_cast<const float *>(beta);
    a.mean = static_cast<float *>(const_cast<void *>(mean)); a.rstd = static_cast<float *>(const_cast<void *>(rstd));
    a.dgamma = static_cast<float *>(dgamma); a.dbeta = static_cast<float *>(dbeta);
    const int rc = norm_common(a, CONV_OP_BWD_DATA, N, C, S, groups, act, layout, dtype, ws, ws_bytes);
    if (rc != kStatusOk) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return glue_elem_bytes(dtype) == 4 ? run_norm_bwd<float>(a, st) : run_norm_bwd<unsigned short>(a, st);
}

size_t distill_loss_workspace_bytes(int N, int V, int K, int dtype)
{
    (void)N; (void)V; (void)K; (void)dtype;
    return 0;
}

int distill_loss_fwd(const void *z, int64_t z_stride, const void *labels, const void *top_idx, const void *top_val,
                     void *loss, void *stats, int N, int V, int K, float temperature, float kd_weight,
                     float label_weight, int index_bytes, int top_dtype, int dtype, void *ws, size_t ws_bytes,
                     void *stream)
{
    (void)ws; (void)ws_bytes;
    if (N != 0 && !loss) return kErrInvalidArg;
    LossArgs a = {};
    a.z = z; a.z_stride = z_stride; a.labels = labels; a.top_idx = top_idx; a.top_val = top_val;
    a.loss = static_cast<float *>(loss); a.stats = static_cast<float *>(stats);
    a.wk = kd_weight; a.wl = label_weight;
    const int rc = loss_common(a, false, N, V, K, temperature, index_bytes, top_dtype, dtype);
    return rc != kStatusOk ? rc : run_loss<false>(a, dtype, stream);
}

int distill_loss_bwd(const void *z, int64_t z_stride, const void *labels, const void *top_idx, const void *top_val,
                     const void *stats, const void *grad, float grad_scale, void *dz, int64_t dz_stride, int N, int V,
                     int K, float temperature, float kd_weight, float label_weight, int index_bytes, int top_dtype,
                     int dtype, void *stream)
{
    if (N != 0 && !stats) return kErrInvalidArg;
    LossArgs a = {};
    a.z = z; a.z_stride = z_stride; a.labels = labels; a.top_idx = top_idx; a.top_val = top_val;
    a.dz = dz; a.dz_stride = dz_stride; a.row_stats = static_cast<const float *>(stats);
    a.grad = static_cast<const float *>(grad); a.grad_scale = grad_scale;
    a.wk = kd_weight; a.wl = label_weight;
    const int rc = loss_common(a, true, N, V, K, temperature, index_bytes, top_dtype, dtype);
    return rc != kStatusOk ? rc : run_loss<true>(a, dtype, stream);
}

int distill_loss_fwd_bwd(const void *z, int64_t z_stride, const void *labels, const void *top_idx, const void *top_val,
                         const void *grad, float grad_scale, void *loss, void *dz, int64_t dz_stride, int N, int V,
                         int K, float temperature, float kd_weight, float label_weight, int index_bytes, int top_dtype,
                         int dtype, void *ws, size_t ws_bytes, void *stream)
{
    (void)ws; (void)ws_bytes;
    if (N != 0 && !loss) return kErrInvalidArg;
    LossArgs a = {};
    a.z = z; a.z_stride = z_stride; a.labels = labels; a.top_idx = top_idx; a.top_val = top_val;
    a.dz = dz; a.dz_stride = dz_stride; a.loss = static_cast<float *>(loss);
    a.grad = static_cast<const float *>(grad); a.grad_scale = grad_scale;
    a.wk = kd_weight; a.wl = label_weight;
    const int rc = loss_common(a, true, N, V, K, temperature, index_bytes, top_dtype, dtype);
    return rc != kStatusOk ? rc : run_loss<true>(a, dtype, stream);
}

}  // extern "C"
