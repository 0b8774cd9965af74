// The plans of layer normalisation and of the fully connected passes on tensors held in blocks, for tests that have to reach one of
// their kernels (built by conftest.py as a shared library; host code only).
#include <math.h>

#include "../include/convnet_hotpath.h"
#include "../paper_1312_5853_amd/csrc/plan.h"

using namespace convnet;

namespace {
#include "../paper_1312_5853_amd/csrc/block_plan.h"
}

// Each writes what conftest.py names, in that order, or returns a status.
extern "C" int layer_norm_plan(int op, int N, int C, int dtype, long long *out)
{
    LayerNormPlan p;
    const int rc = plan_layer_norm(p, op, N, C, dtype);
    if (rc != kStatusOk) return rc;
    const long long v[] = {p.wide, p.columns, p.apart, p.regs, p.threads, p.blocks, (long long)p.lds, p.a.waves, p.a.groups,
                           p.a.rows_per_part, p.a.part_rows, p.a.row_blocks, p.join_blocks, (long long)p.part_bytes};
    std::copy(v, v + sizeof(v) / sizeof(v[0]), out);
    return kStatusOk;
}

extern "C" int kept_grad_plan(int N, int I, int O, int dtype, long long *out)
{
    KeptGradPlan p;
    const int rc = plan_kept_grad(p, N, I, O, dtype);
    if (rc != kStatusOk) return rc;
    const long long v[] = {p.slices, p.tile, p.step, p.outputs, p.a.itiles, p.a.otiles, p.a.splits, p.a.rows_per_split, p.blocks,
                           (long long)p.part_bytes};
    std::copy(v, v + sizeof(v) / sizeof(v[0]), out);
    return kStatusOk;
}

extern "C" int q4_plan(int N, int I, int O, long long *out)
{
    const int rc = check_q4(N, I, O, kDtypeF32);
    if (rc != kStatusOk) return rc;
    const Q4Plan p = plan_q4(N, I, O);
    const long long v[] = {p.fused, p.tile, p.steps, p.wide, p.nrows, p.orows, (long long)p.total};
    std::copy(v, v + sizeof(v) / sizeof(v[0]), out);
    return kStatusOk;
}
