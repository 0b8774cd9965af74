// HIP kernels (gfx950 / CDNA4) and C-ABI entry points of the fully connected part of a network: layer normalisation, tensors
// held in blocks of 8 or 4 bits with a shared power of two, the filter gradient from 8 bits and the forward pass in 4 bits.
// Signatures and conventions are documented in include/convnet_hotpath.h.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "../../include/convnet_hotpath.h"
#include "host_status.h"

using namespace convnet;

namespace {

#include "elements.h"
#include "vectors.h"
#include "block_plan.h"
#include "block_formats.h"
#include "layer_norm_kernels.h"
#include "block_kernels.h"
#include "fc_kept_kernels.h"
#include "fc_q4_kernels.h"

typedef unsigned short Bf16;

// codes are read and written 16 bytes at a time, exponents four
bool blocks_aligned(const void *codes, const void *scales) { return aligned(codes, 16) && aligned(scales, 4); }

template <typename Kern, typename Args>
void launch(Kern kern, int64_t blocks, int threads, size_t lds, hipStream_t st, const Args &a)
{
    if (lds > 64 * 1024)                                 // more dynamic LDS than that has to be allowed per kernel
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(threads), lds, st, a);
}

// ---------------------------------------------------------------------------
// Blocks
// ---------------------------------------------------------------------------
int blocks_common(BlockArgs &a, int N, int C, int form, int dtype, const void *values, const void *codes)
{
    if (N < 0 || C <= 0 || a.stride < C || (form != kE4M3 && form != kE2M1)) return kErrInvalidArg;
    if (N != 0 && (!values || !codes || !a.scales || values == codes || values == a.scales || codes == a.scales)) return kErrInvalidArg;
    const int eb = glue_elem_bytes(dtype);
    if (!eb) return kErrBadDtype;
    if (C > (1 << 30) || N * pitch_of(C) > (int64_t)1 << 34) return kErrTooLarge;       // a thread to eight values
    if (!aligned(values, eb) || !blocks_aligned(codes, a.scales)) return kErrMisaligned;
    a.C = C;
    a.per_row = (int)(pitch_of(C) / 8);
    a.total = (int64_t)N * a.per_row;
    a.div = make_fastdiv(a.per_row);
    return kStatusOk;
}

template <typename T>
void run_quantize(const BlockArgs &a, int form, hipStream_t st)
{
    const int64_t blocks = (a.total + 255) / 256;
    if (form == kE4M3) launch(quantize_blocks_kernel<T, kE4M3>, blocks, 256, 0, st, a);
    else launch(quantize_blocks_kernel<T, kE2M1>, blocks, 256, 0, st, a);
}

template <typename T>
void run_dequantize(const BlockArgs &a, int form, hipStream_t st)
{
    const int64_t blocks = (a.total + 255) / 256;
    if (form == kE4M3) launch(dequantize_blocks_kernel<T, kE4M3>, blocks, 256, 0, st, a);
    else launch(dequantize_blocks_kernel<T, kE2M1>, blocks, 256, 0, st, a);
}

// ---------------------------------------------------------------------------
// Layer normalisation
// ---------------------------------------------------------------------------
template <typename T>
int run_layer_norm_fwd(const LayerNormPlan &p, hipStream_t st)
{
    if (p.wide) launch(layer_norm_fwd_wide<T>, p.blocks, p.threads, 0, st, p.a);
    else if (p.regs == 1) launch(layer_norm_fwd_rows<T, 1>, p.blocks, p.threads, 0, st, p.a);
    else if (p.regs == 2) launch(layer_norm_fwd_rows<T, 2>, p.blocks, p.threads, 0, st, p.a);
    else if (p.regs == 4) launch(layer_norm_fwd_rows<T, 4>, p.blocks, p.threads, 0, st, p.a);
    else if constexpr (sizeof(T) == 4) launch(layer_norm_fwd_rows<T, 8>, p.blocks, p.threads, 0, st, p.a);
    return check_launch();
}

template <typename T, bool HELD, bool SUMS>
void launch_layer_norm_bwd(const LayerNormPlan &p, int64_t blocks, hipStream_t st)
{
    constexpr int few = 8 * (int)sizeof(T) / 16;         // vectors of eight values
    if (few > 1 && p.regs == 1) return launch(layer_norm_bwd_rows<T, HELD, 1, SUMS, 1>, blocks, p.threads, p.lds, st, p.a);
    // Two rows at a time in more than eight wavefronts of bfloat16 rows (4097 to 8192 values), whose loads cover more of the memory's
    // latency, where a work-group has sixteen rows or more.  us, two and one at a time: 6001 x 5003 53.2 and 53.9, from 8 bits 48.1 and
    // 52.7; 4096 x 7001 46.7 and 50.9, 41.8 and 48.6; 12000 x 4100 81.9 and 86.2, 71.2 and 86.0; 12000 x 8192 120.6 and 116.0, 99.0 and
    // 96.6; but 700 x 8192 17.7 and 16.4, 19.0 and 17.4; 2600 x 6144 27.6 and 25.4, 25.1 and 24.0
    if constexpr (SUMS && few == 1)
        if (p.regs == few && p.a.waves > 8 && p.a.N >= 4096) return launch(layer_norm_bwd_rows<T, HELD, few, true, 2>, blocks, p.threads, p.lds, st, p.a);
    if (p.regs == few) return launch(layer_norm_bwd_rows<T, HELD, few, SUMS, 1>, blocks, p.threads, p.lds, st, p.a);
    if (p.regs == 2 * few) return launch(layer_norm_bwd_rows<T, HELD, 2 * few, SUMS, 1>, blocks, p.threads, p.lds, st, p.a);
    if constexpr (!SUMS) launch(layer_norm_bwd_rows<T, HELD, 3 * few, SUMS, 1>, blocks, p.threads, p.lds, st, p.a);
}

template <typename T, bool HELD>
int run_layer_norm_bwd(LayerNormPlan &p, hipStream_t st)
{
    const LayerNormArgs &a = p.a;
    const bool sums = a.dgamma || a.dbeta;
    const int tiles = (a.C + 63) / 64;
    if (a.N > 0) {
        if (p.wide) {
            launch(layer_norm_bwd_wide<T, HELD>, p.blocks, p.threads, 0, st, a);
        } else if (a.part && !p.apart) {
            launch_layer_norm_bwd<T, HELD, true>(p, p.blocks, st);
        } else {
            launch_layer_norm_bwd<T, HELD, false>(p, p.blocks + (p.columns && sums ? tiles : 0), st);
        }
        if (a.part && p.apart) launch(layer_norm_columns<T, HELD>, (int64_t)a.part_rows * tiles, 1024, 0, st, a);
    }
    if (sums && (a.N == 0 || !p.columns)) launch(layer_norm_join, p.join_blocks, 1024, 0, st, a);
    return check_launch();
}

// a: the call's pointers and strides
int layer_norm_bwd_common(const LayerNormArgs &given, bool held, int N, int C, int dtype, void *ws, size_t ws_bytes, void *stream)
{
    const LayerNormArgs &g = given;
    if (g.dy_stride < C || g.out_stride < C || (!held && g.x_stride < C)) return kErrInvalidArg;
    LayerNormPlan p;
    const int rc = plan_layer_norm(p, CONV_OP_BWD_DATA, N, C, dtype);
    if (rc != kStatusOk) return rc;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(g.x, eb) || !aligned(g.dy, eb) || !aligned(g.out, eb) || !blocks_aligned(g.codes, g.scales) || !aligned(g.gamma, 4) ||
        !aligned(g.mean, 4) || !aligned(g.rstd, 4) || !aligned(g.dgamma, 4) || !aligned(g.dbeta, 4))
        return kErrMisaligned;
    const bool sums = g.dgamma || g.dbeta;
    if (sums && p.part_bytes) {
        if (!ws || ws_bytes < p.part_bytes) return kErrWorkspace;
        if (!aligned(ws, 256)) return kErrMisaligned;
    }
    LayerNormArgs &a = p.a;
    a.x = g.x; a.codes = g.codes; a.scales = g.scales; a.dy = g.dy; a.out = g.out;
    a.gamma = g.gamma; a.mean = g.mean; a.rstd = g.rstd; a.dgamma = g.dgamma; a.dbeta = g.dbeta;
    a.x_stride = g.x_stride; a.dy_stride = g.dy_stride; a.out_stride = g.out_stride;
    a.part = sums && !p.columns ? static_cast<float *>(ws) : nullptr;
    if (N == 0) a.part_rows = 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (held) return eb == 4 ? run_layer_norm_bwd<float, true>(p, st) : run_layer_norm_bwd<Bf16, true>(p, st);
    return eb == 4 ? run_layer_norm_bwd<float, false>(p, st) : run_layer_norm_bwd<Bf16, false>(p, st);
}

// ---------------------------------------------------------------------------
// Fully connected layers
// ---------------------------------------------------------------------------
template <typename T, int TILES, int KS, int OCC>
void launch_kept_grad(const KeptGradPlan &p, hipStream_t st)
{
    launch(fc_grad_kept_kernel<T, TILES, TILES, KS, OCC>, p.blocks, 256, grad_lds<T, TILES, TILES, KS>(), st, p.a);
}

template <typename T, int SLICES, int OCC>
void launch_few_grad(const KeptGradPlan &p, hipStream_t st)
{
    KeptGradArgs a = p.a;
    for (int o = 0;; o += p.outputs) {
        a.O = std::min(p.outputs, p.a.O - o);
        launch(fc_grad_few_kernel<T, SLICES, OCC>, (int64_t)ceil_div(a.O, 128) * a.itiles, 256, 0, st, a);
        if (a.O == p.a.O - o) return;
        a.dy = static_cast<const T *>(a.dy) + a.O;
        a.dw += (int64_t)a.O * a.I;
    }
}

template <typename T>
void run_kept_grad(const KeptGradPlan &p, hipStream_t st)
{
    if (p.slices == 1) return launch_few_grad<T, 1, 3>(p, st);
    if (p.slices == 2) return launch_few_grad<T, 2, 3>(p, st);
    if (p.slices == 4) return launch_few_grad<T, 4, 3>(p, st);
    if (p.slices == 8) return launch_few_grad<T, 8, 3>(p, st);
    if constexpr (sizeof(T) == 4) {
        if (p.tile == 256) launch_kept_grad<T, 4, 32, 1>(p, st);
        else if (p.step == 32) launch_kept_grad<T, 2, 32, 2>(p, st);
        else launch_kept_grad<T, 2, 16, 2>(p, st);
    } else {
        if (p.tile == 256) launch_kept_grad<T, 4, 64, 1>(p, st);
        else launch_kept_grad<T, 2, 64, 2>(p, st);
    }
}

template <typename T>
void run_q4_prepare(const Q4PrepArgs &p, hipStream_t st)
{
    launch(q4_prepare<T>, (int64_t)p.x_blocks + (int64_t)p.s_tiles * ceil_div(p.O, 32), 256, 0, st, p);
}

template <typename T>
void run_q4_tiles(Q4TileArgs &a, int tile, hipStream_t st)
{
    a.ntiles = ceil_div(a.N, tile); a.otiles = ceil_div(a.O, tile);
    a.per_xcd = ceil_div(a.ntiles * a.otiles, 8);
    const size_t lds = (size_t)kQ4Stages * 2 * tile * 68 + tile * 4;
    if (tile == 256) launch(fc_q4_tiles<T, 4, 4, 2, 2, 1>, (int64_t)8 * a.per_xcd, 256, lds, st, a);
    else launch(fc_q4_tiles<T, 2, 2, 2, 2, 2>, (int64_t)8 * a.per_xcd, 256, lds, st, a);
}

template <typename TX, typename TY>
void run_q4_rows(Q4RowsArgs &a, const Q4Plan &plan, hipStream_t st)
{
    // LDS: x's codes and exponents, if they are made there, and the rings; the sums of the wavefronts take their place
    auto go = [&](auto kern, int AO, int J, int waves, int stages) {
        a.ntiles = ceil_div(a.N, 16 * J);
        a.units = a.ntiles * ceil_div(a.O, 16 * AO);
        a.per_xcd = ceil_div(a.units, 8);
        a.held = plan.fused ? round_up(a.N * a.steps * 68, 256) : 0;
        const size_t rings = (size_t)a.held + waves * stages * q4_rows_stage(AO, J, plan.fused);
        launch(kern, (int64_t)8 * a.per_xcd, waves * 64, std::max(rings, (size_t)waves * AO * J * 1024), st, a);
    };
    if (plan.fused) go(fc_q4_rows<TX, TY, 1, 1, true, 8, 3>, 1, 1, 8, 3);
    else if (plan.wide == 1) go(fc_q4_rows<float, TY, 1, 1, false, 8, 3>, 1, 1, 8, 3);
    else if (plan.wide == 2) go(fc_q4_rows<float, TY, 1, 2, false, 8, 3>, 1, 2, 8, 3);
    else go(fc_q4_rows<float, TY, 2, 4, false, 4, 3>, 2, 4, 4, 3);
}

}  // namespace

extern "C" {

int quantize_blocks(const void *x, int64_t x_stride, void *codes, void *scales, int N, int C, int format, int dtype, void *stream)
{
    BlockArgs a = {};
    a.in = x; a.out = codes; a.scales = static_cast<unsigned char *>(scales); a.stride = x_stride;
    const int rc = blocks_common(a, N, C, format, dtype, x, codes);
    if (rc != kStatusOk || N == 0) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (glue_elem_bytes(dtype) == 4) run_quantize<float>(a, format, st);
    else run_quantize<Bf16>(a, format, st);
    return check_launch();
}

int dequantize_blocks(const void *codes, const void *scales, void *x, int64_t x_stride, int N, int C, int format, int dtype,
                      void *stream)
{
    BlockArgs a = {};
    a.in = codes; a.out = x; a.scales = static_cast<unsigned char *>(const_cast<void *>(scales)); a.stride = x_stride;
    const int rc = blocks_common(a, N, C, format, dtype, x, codes);
    if (rc != kStatusOk || N == 0) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (glue_elem_bytes(dtype) == 4) run_dequantize<float>(a, format, st);
    else run_dequantize<Bf16>(a, format, st);
    return check_launch();
}

size_t layer_norm_workspace_bytes(int op, int N, int C, int dtype)
{
    LayerNormPlan p;
    return plan_layer_norm(p, op, N, C, dtype) == kStatusOk ? p.part_bytes : 0;
}

int layer_norm_fwd(const void *x, int64_t x_stride, const void *gamma, const void *beta, void *y, int64_t y_stride, void *mean,
                   void *rstd, int N, int C, float eps, int dtype, void *stream)
{
    if ((N != 0 && (!x || !y || x == y)) || !(eps > 0.f) || !isfinite(eps) || x_stride < C || y_stride < C) return kErrInvalidArg;
    LayerNormPlan p;
    const int rc = plan_layer_norm(p, CONV_OP_FWD, N, C, dtype);
    if (rc != kStatusOk) return rc;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(x, eb) || !aligned(y, eb) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return kErrMisaligned;
    if (N == 0) return kStatusOk;
    LayerNormArgs &a = p.a;
    a.x = x; a.x_stride = x_stride; a.out = y; a.out_stride = y_stride; a.eps = eps;
    a.gamma = static_cast<const float *>(gamma); a.beta = static_cast<const float *>(beta);
    a.mean = static_cast<float *>(mean); a.rstd = static_cast<float *>(rstd);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return eb == 4 ? run_layer_norm_fwd<float>(p, st) : run_layer_norm_fwd<Bf16>(p, st);
}

int layer_norm_bwd(const void *x, int64_t x_stride, const void *dy, int64_t dy_stride, const void *gamma, const void *mean,
                   const void *rstd, void *dx, int64_t dx_stride, void *dgamma, void *dbeta, int N, int C, int dtype, void *ws,
                   size_t ws_bytes, void *stream)
{
    if (N != 0 && (!x || !dy || !mean || !rstd || !dx || x == dx || dy == dx)) return kErrInvalidArg;
    LayerNormArgs a = {};
    a.x = x; a.x_stride = x_stride; a.dy = dy; a.dy_stride = dy_stride; a.out = dx; a.out_stride = dx_stride;
    a.gamma = static_cast<const float *>(gamma);
    a.mean = static_cast<float *>(const_cast<void *>(mean)); a.rstd = static_cast<float *>(const_cast<void *>(rstd));
    a.dgamma = static_cast<float *>(dgamma); a.dbeta = static_cast<float *>(dbeta);
    return layer_norm_bwd_common(a, false, N, C, dtype, ws, ws_bytes, stream);
}

int layer_norm_bwd_kept(const void *codes, const void *scales, const void *dy, int64_t dy_stride, const void *gamma,
                        const void *mean, const void *rstd, void *dx, int64_t dx_stride, void *dgamma, void *dbeta, int N, int C,
                        int dtype, void *ws, size_t ws_bytes, void *stream)
{
    if (N != 0 && (!codes || !scales || !dy || !mean || !rstd || !dx || dy == dx || codes == dx || scales == dx)) return kErrInvalidArg;
    LayerNormArgs a = {};
    a.codes = static_cast<const unsigned char *>(codes); a.scales = static_cast<const unsigned char *>(scales);
    a.dy = dy; a.dy_stride = dy_stride; a.out = dx; a.out_stride = dx_stride;
    a.gamma = static_cast<const float *>(gamma);
    a.mean = static_cast<float *>(const_cast<void *>(mean)); a.rstd = static_cast<float *>(const_cast<void *>(rstd));
    a.dgamma = static_cast<float *>(dgamma); a.dbeta = static_cast<float *>(dbeta);
    return layer_norm_bwd_common(a, true, N, C, dtype, ws, ws_bytes, stream);
}

size_t fc_kept_workspace_bytes(int N, int I, int O, int dtype)
{
    KeptGradPlan p;
    return plan_kept_grad(p, N, I, O, dtype) == kStatusOk ? p.part_bytes : 0;
}

int fc_bwd_filter_kept(const void *codes, const void *scales, const void *dy, void *dw, int N, int I, int O, int dtype, void *ws,
                       size_t ws_bytes, void *stream)
{
    if (!dw || (N != 0 && (!codes || !scales || !dy || dw == dy || dw == codes || dw == scales))) return kErrInvalidArg;
    KeptGradPlan p;
    const int rc = plan_kept_grad(p, N, I, O, dtype);
    if (rc != kStatusOk) return rc;
    const size_t eb = glue_elem_bytes(dtype);
    if (!blocks_aligned(codes, scales) || !aligned(dy, eb) || !aligned(dw, 4)) return kErrMisaligned;
    if (p.part_bytes) {
        if (!ws || ws_bytes < p.part_bytes) return kErrWorkspace;
        if (!aligned(ws, 256)) return kErrMisaligned;
    }
    KeptGradArgs &a = p.a;
    a.codes = static_cast<const unsigned char *>(codes); a.scales = static_cast<const unsigned char *>(scales);
    a.dy = dy;
    a.dw = static_cast<float *>(a.splits > 1 ? ws : dw);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (N > 0 && eb == 4) run_kept_grad<float>(p, st);
    else if (N > 0) run_kept_grad<Bf16>(p, st);
    if (N == 0 || a.splits > 1) {
        const int64_t count = (int64_t)I * O;
        hipLaunchKernelGGL(fc_grad_join, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, a.dw, static_cast<float *>(dw),
                           count, N == 0 ? 0 : a.splits);
    }
    return check_launch();
}

size_t fc_q4_workspace_bytes(int N, int I, int O, int dtype)
{
    return check_q4(N, I, O, dtype) == kStatusOk ? plan_q4(N, I, O).total : 0;
}

int fc_fwd_q4(const void *x, const void *w_codes, const void *w_scales, const void *bias, void *y, int N, int I, int O, int relu,
              int dtype, void *ws, size_t ws_bytes, void *stream)
{
    if (N != 0 && (!x || !w_codes || !w_scales || !y || x == y || w_codes == y || w_scales == y)) return kErrInvalidArg;
    const int rc = check_q4(N, I, O, dtype);
    if (rc != kStatusOk) return rc;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(x, eb) || !blocks_aligned(w_codes, w_scales) || !aligned(bias, 4) || !aligned(y, dtype == kDtypeBf16OutBf16 ? 2 : 4))
        return kErrMisaligned;
    if (N == 0) return kStatusOk;
    const Q4Plan plan = plan_q4(N, I, O);
    if (plan.total) {
        if (!ws || ws_bytes < plan.total) return kErrWorkspace;
        if (!aligned(ws, 256)) return kErrMisaligned;
    }
    unsigned char *const scratch = static_cast<unsigned char *>(ws);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (!plan.fused) {
        Q4PrepArgs p = {};
        p.x.in = x; p.x.out = scratch; p.x.stride = I; p.x.C = I;
        p.x.per_row = plan.steps * 16;
        p.x.total = (int64_t)N * p.x.per_row;
        p.x.div = make_fastdiv(p.x.per_row);
        p.w_scales = static_cast<const unsigned *>(w_scales);
        p.xs = reinterpret_cast<unsigned *>(scratch + plan.xs); p.ws = reinterpret_cast<unsigned *>(scratch + plan.ws);
        p.O = O; p.steps = plan.steps; p.nrows = plan.nrows; p.orows = plan.orows;
        p.x_blocks = (int)((p.x.total + 255) / 256);
        p.s_tiles = ceil_div(plan.steps, 32);
        if (eb == 4) run_q4_prepare<float>(p, st);
        else run_q4_prepare<Bf16>(p, st);
    }
    if (plan.tile) {
        Q4TileArgs a = {};
        a.xc = scratch; a.xs = scratch + plan.xs;
        a.wc = static_cast<const unsigned char *>(w_codes); a.ws = scratch + plan.ws;
        a.bias = static_cast<const float *>(bias);
        a.y = y;
        a.N = N; a.O = O; a.steps = plan.steps; a.relu = relu;
        a.nrows = plan.nrows; a.orows = plan.orows;
        if (dtype == kDtypeBf16OutBf16) run_q4_tiles<Bf16>(a, plan.tile, st);
        else run_q4_tiles<float>(a, plan.tile, st);
        return check_launch();
    }
    Q4RowsArgs a = {};
    a.x = x; a.xc = scratch; a.xs = scratch + plan.xs;
    a.wc = static_cast<const unsigned char *>(w_codes);
    a.ws = plan.fused ? static_cast<const unsigned char *>(w_scales) : scratch + plan.ws;
    a.bias = static_cast<const float *>(bias);
    a.y = y;
    a.N = N; a.I = I; a.O = O; a.steps = plan.steps; a.relu = relu;
    a.nrows = plan.nrows; a.orows = plan.orows;
    a.div_row = make_fastdiv(plan.steps * 16);
    if (dtype == kDtypeBf16OutBf16) run_q4_rows<Bf16, Bf16>(a, plan, st);
    else if (eb == 2) run_q4_rows<Bf16, float>(a, plan, st);
    else run_q4_rows<float, float>(a, plan, st);
    return check_launch();
}

}  // extern "C"
