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
#include "vectors.h"
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
    // more than the card holds; keeps the numbers of tiles and rows of sums in their 32 bits
    if ((int64_t)N * C * S >= (int64_t)1 << 40) return kErrTooLarge;
    return kStatusOk;
}

int pow2_up(int v)
{
    int p = 1;
    while (p < v) p <<= 1;
    return p;
}
int pow2_down(int v)
{
    int p = 1;
    while (2 * p <= v) p <<= 1;
    return p;
}

// a launch has fewer than 2^32 threads
bool launchable(int64_t blocks, int threads) { return blocks * threads < (int64_t)1 << 32; }

constexpr size_t kMaxLds = 160 * 1024;
int pitch_of(int threads) { return threads + 9; }        // words between a thread's sums, channels last

constexpr int kMaxWaves = 16, kSplitWaves = 8, kSplitRun = 4;

// How a call runs: which kernels, on what tiles, with how much scratch.
struct NormPlan {
    bool planes, wide, split, solo, one;
    int threads, join_threads, regs;  // regs: vectors a lane keeps (of each input): the kernel's template argument
    int64_t blocks;
    size_t lds, part_bytes, sums_bytes, total;
    NormArgs a;
};

int regs_for(int run, int most)
{
    return std::min(pow2_up(run), most);
}

void plan_planes(NormPlan &p, bool bwd, int V)
{
    NormArgs &a = p.a;
    a.vectors = (a.S - 1) / V + 1;
    a.chunks = (a.vectors + 63) / 64;
    // flat where a plane of its own would leave a sixth of the lanes idle: backward on 256 x 384 planes of 169 bfloat16 (22
    // vectors) 28 us, and 50 with a unit to a plane; on 128 x 256 planes of 729 (92) 36.4 and 37.3.  Longer planes gain
    // nothing by it: 128 x 256 planes of 729 fp32 (183 of 192) backward 56.6 us, and 58.6 flat
    a.flat = a.vectors < 0.85 * 64 * a.chunks;
    const int64_t units = a.flat ? ((int64_t)a.cpg * a.vectors + 63) / 64 : (int64_t)a.cpg * a.chunks;
    const int most = 8;
    const int64_t groups = (int64_t)a.N * a.groups;
    a.tiles = 1;
    a.span = a.cpg;
    int64_t slots = a.flat ? (int64_t)a.cpg * a.vectors : 4 * units;
    if (units <= (int64_t)kMaxWaves * most && a.cpg <= 4096) {
        a.units = (int)units;
        // a wave to a group, four to a work-group and no barrier, for many small groups: 1024 x 64 planes of 16 fp32 in 64
        // groups 16.4 us forward and 28.7 backward, 18.9 and 29.9 with a work-group to each; at 4 units it loses (bfloat16
        // backward on 512 x 256 planes of 196 in 32 groups: 44 us, and 38)
        p.solo = units <= 2 && groups >= 1024;
        // units to a wave, of one tensor or of two: 2, 4, 8 units of it measured (forward 58, 58, 60 us on 128 x 96 planes of
        // 3025 fp32, backward 52, 53, 61 us on 128 x 256 planes of 729); few groups take a wave to a unit (one sample of 256
        // planes of 169 fp32, which 32 work-groups of a wave or eleven take: latency alone)
        const int want = groups < 1024 ? 1 : bwd ? 2 : 4;
        const int waves = p.solo ? 1 : std::min(kMaxWaves, ceil_div(a.units, want));
        a.run = ceil_div(a.units, waves);
        p.threads = p.solo ? 256 : 64 * ceil_div(a.units, a.run);
        p.blocks = p.solo ? (groups + 3) / 4 : groups;
        p.regs = regs_for(a.run, most);
    } else {
        p.split = true;
        const int per = kSplitWaves * kSplitRun;
        if (a.chunks > per) {                              // parts of a plane (flat planes are shorter)
            a.flat = 0;
            a.parts = ceil_div(a.chunks, per);
            a.span = ceil_div(a.chunks, a.parts);
            a.parts = ceil_div(a.chunks, a.span);
            a.tiles = a.cpg * a.parts;
            slots = 4 * a.span;
        } else {                                           // whole planes
            a.span = std::min(a.cpg, std::max(1, a.flat ? per * 64 / a.vectors : per / a.chunks));
            a.tiles = ceil_div(a.cpg, a.span);
            slots = a.flat ? (int64_t)a.span * a.vectors : 4 * (int64_t)a.span * a.chunks;
        }
        p.threads = 64 * kSplitWaves;
        a.run = kSplitRun;
        p.regs = kSplitRun;
        p.blocks = groups * a.tiles;
    }
    a.rows_per_sample = a.parts ? a.parts : 1;
    p.lds = bwd ? (size_t)((p.solo ? 4 : 1) * 2 * (slots + (a.parts ? 1 : a.span)) * 4) : 0;
    a.div_chunks = make_fastdiv(a.chunks);
    a.inv_vectors = (float)(1.0 / a.vectors);
    a.half_vectors = (float)(0.5 / a.vectors);
}

void plan_last(NormPlan &p, bool bwd, int V, int eb)
{
    NormArgs &a = p.a;
    const int most = !bwd ? 16 : eb == 4 ? 10 : 8;
    int best = 0;
    double best_score = 0.0;
    p.one = a.cpg % V == 0;
    auto lds_of = [&](int threads, int64_t slab_groups) {
        const int64_t of_channels = bwd ? 2 * slab_groups * a.cpg : 0;
        return (size_t)(2 * (p.one && !bwd ? 1 : V) * pitch_of(threads) + 2 * slab_groups + of_channels) * 4;
    };
    auto lanes_of = [&](int slab_groups) { return (int)(((int64_t)slab_groups * a.cpg + V - 1) / V); };
    for (int j = 1; j <= a.groups; ++j) {
        if (a.groups % j) continue;
        const int64_t lanes64 = ((int64_t)j * a.cpg + V - 1) / V;
        if (lanes64 > 1024 || lds_of(1024, j) > kMaxLds) break;
        const int rows = 1024 / (int)lanes64;
        if (ceil_div(a.S, rows) > most) continue;
        const double seg = (double)j * a.cpg * eb;
        // Columns of fewer bytes cost more lines than tiles and their joins cost launches: backward 64 x 96 x 55 x 55 fp32 74 us
        // in one pass of 48-byte columns, and 93 in tiles; forward in columns of 16 or 24 bytes 4 x 256 x 112 x 112 bf16 34 us
        // and 32 x 64 x 112 x 112 bf16 57, in tiles 23 and 44.  At 48 bytes forward goes either way (64 x 192 x 48 x 48 bf16 48
        // us in one pass of 48 bytes, 45 in tiles, and 37 in the 96 bytes that it takes; 32 x 96 x 55 x 55 bf16 20 and 25).
        if (seg < (bwd ? 48 : 64) && j != a.groups) continue;
        // lines that a slab shares with its neighbours are read by both; few work-groups leave the card idle
        const double wgs = (double)a.N * (a.groups / j);
        const double score = seg / (seg + 64) * std::min(1.0, wgs / 512);
        if (score > best_score) { best_score = score; best = j; }
    }
    int threads;
    if (best) {
        a.slab_groups = best;
        a.lanes = lanes_of(best);
        // rows to a thread.  Forward 4, 8, 16: 25.8, 22.1, 24.3 us on 128 x 256 x 27 x 27 bf16, 25.6, 19.9, 19.5 us on
        // 256 x 384 x 13 x 13; backward 4 to 10 are within 3 %, and 6 leaves more work-groups to a CU than 10
        const int want = bwd ? 6 : 8;
        threads = std::min<int64_t>(1024, round_up64((int64_t)a.lanes * ceil_div(a.S, want), 64));
        a.rows = threads / a.lanes;
        a.tile_rows = a.S;
        a.tiles = 1;
    } else {
        p.split = true;
        int j = 1;
        for (int k = 1; k <= a.groups; ++k)
            if (a.groups % k == 0 && lanes_of(k) <= 512) j = k;
        a.slab_groups = j;
        a.lanes = lanes_of(j);
        threads = std::max(512, round_up(a.lanes, 64));
        a.rows = threads / a.lanes;
        const int64_t N_slabs = (int64_t)a.N * (a.groups / j);
        // as many rows to a thread as leave 512 work-groups, 32 at most: forward 4 x 256 x 112 x 112 bf16 23.0 us, 28.5 with
        // 128 work-groups and 22.5 with 2048; 32 x 64 x 112 x 112 bf16 44, 40 and 52 us.  (A thread holds kSplitRun of them at
        // a time: 6 rows, say, are a full and a half-empty trip to memory.)
        const int most_rows = (int)std::max<int64_t>(4, std::min<int64_t>(32, (int64_t)N_slabs * ceil_div(a.S, a.rows) / 512));
        a.tile_rows = std::min(a.S, a.rows * most_rows);
        a.tiles = ceil_div(a.S, a.tile_rows);
        a.tile_rows = ceil_div(a.S, a.tiles);
    }
    a.cw = a.slab_groups * a.cpg;
    a.slabs = a.groups / a.slab_groups;
    p.threads = threads;
    p.regs = ceil_div(a.tile_rows, a.rows);
    a.pitch = pitch_of(threads);
    a.group_lanes = std::min(64, pow2_down(std::max(1, threads / a.slab_groups)));
    a.channel_lanes = std::min(64, pow2_down(std::max(1, threads / a.cw)));
    a.work = a.N * a.tiles * a.slabs;
    a.units_per_xcd = ceil_div(a.work, 8);
    p.blocks = 8 * (int64_t)a.units_per_xcd;
    a.div_width = make_fastdiv(p.one ? a.cpg / V : a.cpg);
    p.lds = lds_of(threads, a.slab_groups);
    a.rows_per_sample = a.tiles;
    a.div_lanes = make_fastdiv(a.lanes);
    a.div_slabs = make_fastdiv(a.slabs);
}

int plan_norm(NormPlan &p, int op, int N, int C, int S, int groups, int layout, int dtype)
{
    p = {};
    const int rc = norm_checks(N, C, S, groups, layout, dtype);
    if (rc != kStatusOk) return rc;
    if (op != CONV_OP_FWD && op != CONV_OP_BWD_DATA) return kErrInvalidArg;
    const bool bwd = op == CONV_OP_BWD_DATA;
    const int eb = glue_elem_bytes(dtype), V = 16 / eb;
    NormArgs &a = p.a;
    a.N = N; a.C = C; a.S = S; a.groups = groups; a.cpg = C / groups;
    a.inv_m64 = 1.0 / ((double)a.cpg * S);
    a.inv_m = (float)a.inv_m64;
    a.div_groups = make_fastdiv(groups);
    a.div_cpg = make_fastdiv(a.cpg);
    // one channel, or one position: the same memory either way
    p.planes = layout == CONV_LAYOUT_PLANES ? S > 1 : C == 1;
    p.wide = !p.planes && a.cpg > 1024 * V;
    if (p.wide) {
        p.threads = 1024;
        p.blocks = (int64_t)N * groups;
        a.tiles = a.rows_per_sample = 1;
    } else if (p.planes) {
        plan_planes(p, bwd, V);
    } else {
        plan_last(p, bwd, V, eb);
    }
    a.div_tiles = make_fastdiv(a.tiles);
    // forward: every work-group joins its group's tiles itself where these are few, which saves a launch of 4 us; past that
    // the joins' reads (12 bytes to a tile and work-group) would come to a part of the tensor's own
    a.join = (int64_t)a.tiles * (p.planes ? 1 : a.slab_groups) <= 2048;
    if ((int64_t)N * a.rows_per_sample >= ((int64_t)1 << 31) || !launchable(p.blocks, p.threads)) return kErrTooLarge;
    a.part_rows = N * a.rows_per_sample;
    const int64_t ng = (int64_t)N * groups;
    if (p.split) {
        // threads that join a group's sums, a channel of a row to each: 128 x 96 x 55 x 55 bf16 in 32 groups, channels last,
        // 4.8 us, 8.0 with 256 threads at least and 32 with 1024; 8 x 512 x 56 x 56 bf16 in one group 15.5 us, 38 with 256
        const int64_t loads = (int64_t)a.cpg * a.rows_per_sample;
        p.join_threads = std::min(1024, std::max(64, pow2_up((int)std::min<int64_t>(loads, 1024))));
        a.join_lanes = std::min(pow2_up(std::min(a.cpg, p.join_threads)), p.join_threads / pow2_up(std::min(16, a.rows_per_sample)));
        if (!launchable(ng, p.join_threads)) return kErrTooLarge;
    }
    if (bwd) p.part_bytes = (size_t)2 * a.part_rows * C * 4;
    else if (p.split) p.part_bytes = (size_t)ng * a.tiles * 3 * 4;
    if (p.split) p.sums_bytes = (size_t)(ng * 2 + (bwd ? 2 * (int64_t)N * C : 0)) * 4;
    p.part_bytes = (size_t)round_up64(p.part_bytes, 256);
    p.total = p.part_bytes + (size_t)round_up64(p.sums_bytes, 256);
    return kStatusOk;
}

// a holds the call's pointers, act and eps; takes the plan's figures over
int norm_common(NormPlan &p, const NormArgs &given, int op, int N, int C, int S, int groups, int layout, int dtype, void *ws,
                size_t ws_bytes)
{
    const int rc = plan_norm(p, op, N, C, S, groups, layout, dtype);
    if (rc != kStatusOk) return rc;
    const NormArgs &a = given;
    if (a.act != kActNone && a.act != kActRelu && a.act != kActSilu) return kErrInvalidArg;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(a.x, eb) || !aligned(a.dy, eb) || !aligned(a.out, eb)) return kErrMisaligned;
    if (!aligned(a.gamma, 4) || !aligned(a.beta, 4) || !aligned(a.mean, 4) || !aligned(a.rstd, 4) ||
        !aligned(a.dgamma, 4) || !aligned(a.dbeta, 4))
        return kErrMisaligned;
    if (p.total) {
        if (!ws || ws_bytes < p.total) return kErrWorkspace;
        if (!aligned(ws, 256)) return kErrMisaligned;
    }
    p.a.x = a.x; p.a.dy = a.dy; p.a.out = a.out; p.a.gamma = a.gamma; p.a.beta = a.beta;
    p.a.mean = a.mean; p.a.rstd = a.rstd; p.a.dgamma = a.dgamma; p.a.dbeta = a.dbeta;
    p.a.act = a.act; p.a.eps = a.eps;
    p.a.part = static_cast<float *>(ws);
    p.a.group_sums = reinterpret_cast<float *>(static_cast<char *>(ws) + p.part_bytes);
    p.a.joined = p.a.group_sums;
    p.a.sample_sums = p.split ? p.a.group_sums + (int64_t)2 * N * groups : p.a.part;
    return kStatusOk;
}

template <typename Kern>
void launch_norm(Kern kern, const NormPlan &p, size_t lds, hipStream_t st)
{
    if (lds > 64 * 1024)                             // more dynamic LDS than that has to be allowed per kernel
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLds);
    hipLaunchKernelGGL(kern, dim3((unsigned)p.blocks), dim3(p.threads), lds, st, p.a);
}

template <typename T, int MODE>
void launch_norm_fwd(const NormPlan &p, hipStream_t st)
{
    if (p.planes) {
        if constexpr (MODE != kWhole) launch_norm(group_norm_planes_fwd<T, kSplitRun, false, MODE>, p, 0, st);
        else if (p.solo && p.regs == 1) launch_norm(group_norm_planes_fwd<T, 1, true, MODE>, p, 0, st);
        else if (p.solo) launch_norm(group_norm_planes_fwd<T, 2, true, MODE>, p, 0, st);
        else if (p.regs == 1) launch_norm(group_norm_planes_fwd<T, 1, false, MODE>, p, 0, st);
        else if (p.regs == 2) launch_norm(group_norm_planes_fwd<T, 2, false, MODE>, p, 0, st);
        else if (p.regs == 4) launch_norm(group_norm_planes_fwd<T, 4, false, MODE>, p, 0, st);
        else launch_norm(group_norm_planes_fwd<T, 8, false, MODE>, p, 0, st);
        return;
    }
    auto go = [&](auto of_one, auto of_several) { launch_norm(p.one ? of_one : of_several, p, p.lds, st); };
    if constexpr (MODE != kWhole) go(group_norm_last_fwd<T, kSplitRun, MODE, true>, group_norm_last_fwd<T, kSplitRun, MODE, false>);
    else if (p.regs <= 4) go(group_norm_last_fwd<T, 4, MODE, true>, group_norm_last_fwd<T, 4, MODE, false>);
    else if (p.regs <= 8) go(group_norm_last_fwd<T, 8, MODE, true>, group_norm_last_fwd<T, 8, MODE, false>);
    else go(group_norm_last_fwd<T, 16, MODE, true>, group_norm_last_fwd<T, 16, MODE, false>);
}

template <typename T, int MODE>
void launch_norm_bwd(const NormPlan &p, hipStream_t st)
{
    const size_t lds = MODE == kApply ? 0 : p.lds;
    if (p.planes) {
        if constexpr (MODE != kWhole) launch_norm(group_norm_planes_bwd<T, kSplitRun, false, MODE>, p, lds, st);
        else if (p.solo && p.regs == 1) launch_norm(group_norm_planes_bwd<T, 1, true, MODE>, p, lds, st);
        else if (p.solo) launch_norm(group_norm_planes_bwd<T, 2, true, MODE>, p, lds, st);
        else if (p.regs == 1) launch_norm(group_norm_planes_bwd<T, 1, false, MODE>, p, lds, st);
        else if (p.regs == 2) launch_norm(group_norm_planes_bwd<T, 2, false, MODE>, p, lds, st);
        else if (p.regs == 4) launch_norm(group_norm_planes_bwd<T, 4, false, MODE>, p, lds, st);
        else launch_norm(group_norm_planes_bwd<T, 8, false, MODE>, p, lds, st);
        return;
    }
    auto go = [&](auto of_one, auto of_several) { launch_norm(p.one ? of_one : of_several, p, lds, st); };
    if constexpr (MODE != kWhole) go(group_norm_last_bwd<T, kSplitRun, MODE, true>, group_norm_last_bwd<T, kSplitRun, MODE, false>);
    else if (p.regs <= 4) go(group_norm_last_bwd<T, 4, MODE, true>, group_norm_last_bwd<T, 4, MODE, false>);
    else if (p.regs <= 6) go(group_norm_last_bwd<T, 6, MODE, true>, group_norm_last_bwd<T, 6, MODE, false>);
    else if (p.regs <= 8) go(group_norm_last_bwd<T, 8, MODE, true>, group_norm_last_bwd<T, 8, MODE, false>);
    else if constexpr (sizeof(T) == 4) go(group_norm_last_bwd<T, 10, MODE, true>, group_norm_last_bwd<T, 10, MODE, false>);
}

template <typename T>
int run_norm_fwd(NormPlan &p, hipStream_t st)
{
    if (p.wide) {
        launch_norm(group_norm_wide_fwd<T>, p, 0, st);
    } else if (!p.split) {
        launch_norm_fwd<T, kWhole>(p, st);
    } else {
        launch_norm_fwd<T, kSums>(p, st);
        const int total = p.a.N * p.a.groups;
        if (!p.a.join)
            hipLaunchKernelGGL(group_norm_join_stats, dim3((total + 3) / 4), dim3(256), 0, st, p.a);
        launch_norm_fwd<T, kApply>(p, st);
    }
    return check_launch();
}

template <typename T>
int run_norm_bwd(NormPlan &p, hipStream_t st)
{
    if (p.a.N > 0) {
        if (p.wide) {
            launch_norm(group_norm_wide_bwd<T>, p, 0, st);
        } else if (!p.split) {
            launch_norm_bwd<T, kWhole>(p, st);
        } else {
            launch_norm_bwd<T, kSums>(p, st);
            hipLaunchKernelGGL(group_norm_join_groups, dim3(p.a.N * p.a.groups), dim3(p.join_threads), 0, st, p.a);
            launch_norm_bwd<T, kApply>(p, st);
        }
    }
    if (p.a.dgamma || p.a.dbeta)
        hipLaunchKernelGGL(group_norm_join_channels, dim3((p.a.C + 15) / 16), dim3(256), 0, st, p.a);
    return check_launch();
}

// ---------------------------------------------------------------------------
// Loss
// ---------------------------------------------------------------------------
// How a call runs: a wave or a work-group to a row, or several work-groups.
struct LossPlan {
    bool solo;
    int chunks, run, parts, part_chunks, threads, regs;
    int64_t blocks;
    size_t part_bytes, total;
};

// A part of a row: four waves of four vectors a lane, or of two where that gives few work-groups (33 x 50021 fp32, both:
// 12.1 and 11.9 us; 2048 x 65536 bf16, gradient alone: 103 and 115 us; eight waves of four: 12.3 and 105 us).
constexpr int kPartWaves = 4, kPartRun = 4, kPartFew = 1024;

int part_run(int64_t rows, int chunks)
{
    return rows * ceil_div(chunks, kPartWaves * kPartRun) >= kPartFew ? kPartRun : kPartRun / 2;
}

int plan_loss(LossPlan &p, int N, int V, int K, int dtype, bool from_stats)
{
    p = {};
    if (N < 0 || V <= 0 || K < 0) return kErrInvalidArg;
    const int eb = glue_elem_bytes(dtype);
    if (!eb) return kErrBadDtype;
    if (K > CONV_DISTILL_MAX_TOP || V > (1 << 30)) return kErrTooLarge;
    const int vec = 16 / eb, nv = (V + vec - 1) / vec;
    p.chunks = ceil_div(nv, 64);
    p.parts = 1;
    const int part = kPartWaves * part_run(N, p.chunks);
    // a thread to each entry and to the label, which go through all the others: gradient of 689 x 256 fp32 with 110 entries
    // 8.4 us, 10.8 with a thread to two
    const int for_entries = round_up(K + 1, 64);
    if (from_stats) {                                      // nothing to join: parts of a row are work of their own
        p.part_chunks = std::min(p.chunks, part);
        p.run = ceil_div(p.part_chunks, kPartWaves);
        p.threads = std::max(64 * ceil_div(p.part_chunks, p.run), std::min(256, for_entries));
        p.parts = ceil_div(p.chunks, p.part_chunks);
        p.blocks = (int64_t)N * p.parts;
        return launchable(p.blocks, p.threads) ? kStatusOk : kErrTooLarge;
    }
    // a wave to a row: 4096 x 1000 bf16, loss 7.2 us, both 11.1; with a work-group to a row 9.2 and 13.1
    p.solo = p.chunks <= 4 && N >= 1024;
    if (p.solo) {
        p.run = p.chunks;
        p.threads = 256;
        p.blocks = ((int64_t)N + 3) / 4;
    } else if (p.chunks <= 16 * 4 || (p.chunks <= 16 * 8 && N >= 128)) {
        // A work-group to a row.  Few rows, both: 64 x 10007 fp32 7.5 us this way, 10.0 in parts, 1 x 16000 6.3 and 8.2; up to
        // twice as long ones where they occupy half of the card: 128 x 32003 fp32 13.1 us, 15.3 in parts, 33 x 32003 10.4 and 9.9.
        // Vectors of a lane: many rows 2048 x 5000 fp32 20.7 us with four, 28.5 with one; few 128 x 1000 6.3 and 5.5.
        const int want = N >= 512 ? 4 : 1;
        p.run = ceil_div(p.chunks, std::min(16, ceil_div(p.chunks, want)));
        p.threads = std::max(64 * ceil_div(p.chunks, p.run), std::min(1024, for_entries));
        p.blocks = N;
    } else {
        p.parts = ceil_div(p.chunks, part);
        p.part_chunks = ceil_div(p.chunks, p.parts);
        p.parts = ceil_div(p.chunks, p.part_chunks);
        p.run = ceil_div(p.part_chunks, kPartWaves);
        p.threads = std::max(64 * ceil_div(p.part_chunks, p.run), std::min(256, for_entries));
        p.blocks = (int64_t)N * p.parts;
        p.part_bytes = (size_t)round_up64(p.blocks * 3 * 4, 256);
        p.total = p.part_bytes + (size_t)round_up64((int64_t)N * (K + 1) * 4, 256);
    }
    p.regs = std::min(pow2_up(p.run), 8);
    return launchable(p.blocks, p.threads) ? kStatusOk : kErrTooLarge;
}

// a: pointers, strides and scalars of the call are set; the rest is checked and filled in
int loss_common(LossArgs &a, LossPlan &p, bool dz, int N, int V, int K, float temperature, int index_bytes, int top_dtype,
                int dtype, void *ws, size_t ws_bytes)
{
    if (N != 0 && (!a.z || (dz && !a.dz) || (!a.labels && K == 0) || (K > 0 && (!a.top_idx || !a.top_val))))
        return kErrInvalidArg;
    if (a.z_stride < V || (dz && a.dz_stride < V) || (index_bytes != 4 && index_bytes != 8)) return kErrInvalidArg;
    const float log2e = 1.44269504088896340736f;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(log2e / temperature) || !isfinite(a.wk) ||
        !isfinite(a.wl) || !isfinite(a.grad_scale))
        return kErrInvalidArg;
    if (N != 0 && dz && a.z == a.dz && a.z_stride != a.dz_stride) return kErrInvalidArg;
    const int rc = plan_loss(p, N, V, K, dtype, a.row_stats != nullptr);
    if (rc != kStatusOk) return rc;
    const int tb = K ? glue_elem_bytes(top_dtype) : 4;
    if (!tb) return kErrBadDtype;
    const size_t eb = glue_elem_bytes(dtype);
    if (!aligned(a.z, eb) || !aligned(a.dz, eb) || !aligned(a.labels, index_bytes) || !aligned(a.top_idx, index_bytes) ||
        !aligned(a.top_val, tb) || !aligned(a.loss, 4) || !aligned(a.stats, 4) || !aligned(a.row_stats, 4) ||
        !aligned(a.grad, 4))
        return kErrMisaligned;
    if (p.total) {
        if (!ws || ws_bytes < p.total) return kErrWorkspace;
        if (!aligned(ws, 256)) return kErrMisaligned;
    }
    a.N = N; a.V = V; a.K = K;
    a.T = temperature;
    a.to_21 = log2e; a.to_2T = log2e / temperature;
    a.wide_index = index_bytes == 8; a.top_bf16 = tb == 2;
    if (a.wk == 0.f) a.K = 0;                            // a term of weight 0 is absent
    if (a.wl == 0.f) a.labels = nullptr;
    a.chunks = p.chunks; a.run = p.run; a.parts = p.parts; a.part_chunks = p.part_chunks;
    a.div_parts = make_fastdiv(p.parts);
    a.part = static_cast<float *>(ws);
    a.named = reinterpret_cast<float *>(static_cast<char *>(ws) + p.part_bytes);
    return kStatusOk;
}

template <typename Kern>
void launch_loss(Kern kern, const LossArgs &a, int64_t blocks, int threads, size_t lds, hipStream_t st)
{
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(threads), lds, st, a);
}

template <typename T, bool GRAD>
int run_loss_typed(const LossArgs &a, const LossPlan &p, hipStream_t st)
{
    const size_t lds = (size_t)(p.solo ? 4 : 1) * 3 * round_up(a.K, 4) * 4;
    if constexpr (GRAD)
        if (a.row_stats) {
            if (p.run <= 2) launch_loss(distill_part_apply<T, 2, true>, a, p.blocks, p.threads, lds, st);
            else launch_loss(distill_part_apply<T, 4, true>, a, p.blocks, p.threads, lds, st);
            return check_launch();
        }
    if (p.parts > 1) {
        const int64_t blocks = GRAD ? p.blocks : a.N;        // the loss alone: a work-group to a row
        const int threads = GRAD ? p.threads : 256;
        if (p.run <= 2) {
            launch_loss(distill_part_sums<T, 2>, a, p.blocks, p.threads, 0, st);
            launch_loss(distill_part_apply<T, 2, GRAD>, a, blocks, threads, lds, st);
        } else {
            launch_loss(distill_part_sums<T, 4>, a, p.blocks, p.threads, 0, st);
            launch_loss(distill_part_apply<T, 4, GRAD>, a, blocks, threads, lds, st);
        }
    } else if (p.solo && p.regs == 1) {
        launch_loss(distill_rows<T, 1, true, GRAD>, a, p.blocks, p.threads, lds, st);
    } else if (p.solo && p.regs == 2) {
        launch_loss(distill_rows<T, 2, true, GRAD>, a, p.blocks, p.threads, lds, st);
    } else if (p.solo) {
        launch_loss(distill_rows<T, 4, true, GRAD>, a, p.blocks, p.threads, lds, st);
    } else if (p.regs == 1) {
        launch_loss(distill_rows<T, 1, false, GRAD>, a, p.blocks, p.threads, lds, st);
    } else if (p.regs <= 4) {
        launch_loss(distill_rows<T, 4, false, GRAD>, a, p.blocks, p.threads, lds, st);
    } else {
        launch_loss(distill_rows<T, 8, false, GRAD>, a, p.blocks, p.threads, lds, st);
    }
    return check_launch();
}

template <bool GRAD>
int run_loss(const LossArgs &a, const LossPlan &p, int dtype, void *stream)
{
    if (a.N == 0) return kStatusOk;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return glue_elem_bytes(dtype) == 4 ? run_loss_typed<float, GRAD>(a, p, st)
                                       : run_loss_typed<unsigned short, GRAD>(a, p, st);
}

}  // namespace

extern "C" {

size_t group_norm_act_workspace_bytes(int op, int N, int C, int S, int groups, int layout, int dtype)
{
    NormPlan p;
    return plan_norm(p, op, N, C, S, groups, layout, dtype) == kStatusOk ? p.total : 0;
}

int group_norm_act_fwd(const void *x, const void *gamma, const void *beta, void *y, void *mean, void *rstd, int N, int C,
                       int S, int groups, float eps, int act, int layout, int dtype, void *ws, size_t ws_bytes,
                       void *stream)
{
    if ((N != 0 && (!x || !y || x == y)) || !(eps > 0.f) || !isfinite(eps)) return kErrInvalidArg;
    NormArgs a = {};
    a.x = x; a.out = y; a.eps = eps; a.act = act;
    a.gamma = static_cast<const float *>(gamma); a.beta = static_cast<const float *>(beta);
    a.mean = static_cast<float *>(mean); a.rstd = static_cast<float *>(rstd);
    NormPlan p;
    const int rc = norm_common(p, a, CONV_OP_FWD, N, C, S, groups, layout, dtype, ws, ws_bytes);
    if (rc != kStatusOk) return rc;
    if (N == 0) return kStatusOk;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return glue_elem_bytes(dtype) == 4 ? run_norm_fwd<float>(p, st) : run_norm_fwd<unsigned short>(p, st);
}

int group_norm_act_bwd(const void *x, const void *dy, const void *gamma, const void *beta, const void *mean,
                       const void *rstd, void *dx, void *dgamma, void *dbeta, int N, int C, int S, int groups, int act,
                       int layout, int dtype, void *ws, size_t ws_bytes, void *stream)
{
    if (N != 0 && (!x || !dy || !mean || !rstd || !dx || x == dx || dy == dx)) return kErrInvalidArg;
    NormArgs a = {};
    a.x = x; a.dy = dy; a.out = dx; a.act = act;
    a.gamma = static_cast<const float *>(gamma); a.beta = static_cast<const float *>(beta);
    a.mean = static_cast<float *>(const_cast<void *>(mean)); a.rstd = static_cast<float *>(const_cast<void *>(rstd));
    a.dgamma = static_cast<float *>(dgamma); a.dbeta = static_cast<float *>(dbeta);
    NormPlan p;
    const int rc = norm_common(p, a, CONV_OP_BWD_DATA, N, C, S, groups, layout, dtype, ws, ws_bytes);
    if (rc != kStatusOk) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return glue_elem_bytes(dtype) == 4 ? run_norm_bwd<float>(p, st) : run_norm_bwd<unsigned short>(p, st);
}

size_t distill_loss_workspace_bytes(int N, int V, int K, int dtype)
{
    LossPlan p;
    return plan_loss(p, N, V, K, dtype, false) == kStatusOk ? p.total : 0;
}

int distill_loss_fwd(const void *z, int64_t z_stride, const void *labels, const void *top_idx, const void *top_val,
                     void *loss, void *stats, int N, int V, int K, float temperature, float kd_weight,
                     float label_weight, int index_bytes, int top_dtype, int dtype, void *ws, size_t ws_bytes,
                     void *stream)
{
    if (N != 0 && !loss) return kErrInvalidArg;
    LossArgs a = {};
    a.z = z; a.z_stride = z_stride; a.labels = labels; a.top_idx = top_idx; a.top_val = top_val;
    a.loss = static_cast<float *>(loss); a.stats = static_cast<float *>(stats);
    a.wk = kd_weight; a.wl = label_weight;
    LossPlan p;
    const int rc = loss_common(a, p, false, N, V, K, temperature, index_bytes, top_dtype, dtype, ws, ws_bytes);
    return rc != kStatusOk ? rc : run_loss<false>(a, p, dtype, stream);
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
    LossPlan p;
    const int rc = loss_common(a, p, true, N, V, K, temperature, index_bytes, top_dtype, dtype, nullptr, 0);
    return rc != kStatusOk ? rc : run_loss<true>(a, p, dtype, stream);
}

int distill_loss_fwd_bwd(const void *z, int64_t z_stride, const void *labels, const void *top_idx, const void *top_val,
                         const void *grad, float grad_scale, void *loss, void *dz, int64_t dz_stride, int N, int V,
                         int K, float temperature, float kd_weight, float label_weight, int index_bytes, int top_dtype,
                         int dtype, void *ws, size_t ws_bytes, void *stream)
{
    if (N != 0 && !loss) return kErrInvalidArg;
    LossArgs a = {};
    a.z = z; a.z_stride = z_stride; a.labels = labels; a.top_idx = top_idx; a.top_val = top_val;
    a.dz = dz; a.dz_stride = dz_stride; a.loss = static_cast<float *>(loss);
    a.grad = static_cast<const float *>(grad); a.grad_scale = grad_scale;
    a.wk = kd_weight; a.wl = label_weight;
    LossPlan p;
    const int rc = loss_common(a, p, true, N, V, K, temperature, index_bytes, top_dtype, dtype, ws, ws_bytes);
    return rc != kStatusOk ? rc : run_loss<true>(a, p, dtype, stream);
}

}  // extern "C"
