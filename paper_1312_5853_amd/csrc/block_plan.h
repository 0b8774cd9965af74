// Host-side planning of layer normalisation and of the fully connected passes on tensors held in blocks: argument checks, which kernel
// takes which sizes, its grid, its scratch, and the arguments of layer norm's kernels and the filter gradient's.  Included inside an anonymous
// namespace after plan.h and the public header; plain C++ with no HIP dependency, so the same header compiles into a CPU-only query.

constexpr int kRowFill = 128;         // a row's codes are filled up with zeros to a multiple of this many values

inline int pow2_up(int v)
{
    int p = 1;
    while (p < v) p <<= 1;
    return p;
}

constexpr int64_t kMaxElements = (int64_t)1 << 31;       // of a fully connected layer's tensors

// of rows or columns, whose number may be any that an int holds
inline int parts_of(int n, int m) { return (n - 1) / m + 1; }

inline int64_t pitch_of(int C) { return round_up64(C, kRowFill); }

// ---------------------------------------------------------------------------
// Layer normalisation
// ---------------------------------------------------------------------------
constexpr int kWideThreads = 1024;    // to a row longer than a work-group keeps
constexpr int layer_norm_bwd_waves(int values) { return values <= 8 ? 16 : 12; }        // most to a row, by values to a thread

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
    int row_blocks;                          // backward: work-groups that take rows; those after them take columns
    float inv_c, eps;
};

struct LayerNormPlan {
    bool wide;                    // rows longer than a work-group keeps
    bool columns, apart;          // backward: columns' sums by work-groups of their own, in the same launch or in one of their own
    int regs, threads;
    int64_t blocks, join_blocks;  // grids: of the kernel that takes rows, and of the one that joins the columns' sums
    size_t lds, part_bytes;
    LayerNormArgs a;
};

inline int plan_layer_norm(LayerNormPlan &p, int op, int N, int C, int dtype)
{
    p = {};
    if (N < 0 || C <= 0 || (op != CONV_OP_FWD && op != CONV_OP_BWD_DATA)) return kErrInvalidArg;
    const int eb = glue_elem_bytes(dtype);
    if (!eb) return kErrBadDtype;
    if (C > (1 << 27) || (int64_t)N * C >= (int64_t)1 << 40) return kErrTooLarge;
    const bool bwd = op == CONV_OP_BWD_DATA;
    const int V = 16 / eb;
    LayerNormArgs &a = p.a;
    a.N = N; a.C = C;
    a.vectors = (C - 1) / V + 1;
    a.pitch = pitch_of(C);
    a.inv_c = (float)(1.0 / C);
    // values to a thread: forward 16, 32 where a work-group of 1024 threads needs them; backward 8, and 16 or 24 in up to 768 threads,
    // which have registers for their sums too
    const int chunks = (a.vectors + 63) / 64;
    const int few = (bwd ? 8 : 16) / V, most_waves = bwd && chunks > 16 * few ? layer_norm_bwd_waves(16) : 16;
    p.wide = chunks > most_waves * (bwd ? 3 : 2) * few;
    if (p.wide) {
        a.waves = 16; a.groups = 1;
        p.threads = kWideThreads;
        p.blocks = std::min(N, 1 << 16);
        p.apart = bwd;
    } else {
        a.waves = std::min(most_waves, ceil_div(chunks, few));
        const int runs = ceil_div(chunks, a.waves);
        p.regs = runs <= 2 * few ? pow2_up(runs) : 3 * few;
        // dgamma and dbeta by work-groups of their own, over few rows in the same launch (us: 512 x 1024 fp32 9.2 and 10.9, 512 x 9216
        // 22.2 and 22.1, bfloat16 14.4 and 20.1, 768 x 1024 fp32 11.9 and 10.5), and where a thread has no registers left for sums (24 values; 3000 x 16384 fp32
        // with them, spilt, 368 us)
        p.columns = bwd && N <= 640;
        p.apart = bwd && !p.columns && p.regs == 3 * few;
        // rows side by side in a work-group (backward their columns' sums are joined in LDS), as many as few rows leave for all CUs
        const int beside = (bwd ? 16 : 8) / a.waves;
        a.groups = std::max(1, p.columns ? beside : std::min(beside, parts_of(N, 256)));
        p.threads = a.waves * a.groups * 64;
        const int rounds = parts_of(N, a.groups), width = a.vectors * V;
        if (bwd) {
            // One to a CU, as every one's sums are written and read again (a call of 6001 x 5003 bfloat16 from 8 bits 48.1 us, 52.2 with
            // two, 8192 x 4096 fp32 82.0 and 84.9); but a column's sum in a thread runs over at most 256 rows.
            a.row_blocks = std::min(rounds, std::max(256, parts_of(rounds, 256)));
            p.blocks = a.row_blocks;
            a.part_rows = p.columns ? 0 : a.row_blocks;
            p.lds = (size_t)std::max(width * (a.groups > 1 && !p.columns && !p.apart ? 2 * a.groups : 1), p.columns ? 2 * p.threads : 0) * 4;
        } else {
            p.blocks = std::min(rounds, p.regs * V <= 8 ? 1024 : 512);
        }
    }
    if (p.apart) {
        const int tiles = (C + 63) / 64;
        a.part_rows = std::max(1, std::min(parts_of(N, 256), 2048 / tiles));
        a.rows_per_part = std::max(1, parts_of(N, a.part_rows));
        a.part_rows = parts_of(N, a.rows_per_part);
    }
    if (bwd) p.join_blocks = std::min(2 * ((C + 63) / 64), 1 << 21);         // (a launch has fewer than 2^32 threads)
    if (bwd) p.part_bytes = (size_t)round_up64((int64_t)a.part_rows * 2 * C * 4, 256);
    return kStatusOk;
}

// ---------------------------------------------------------------------------
// Fully connected layers
// ---------------------------------------------------------------------------
constexpr int kFewInputs = 64;        // of a step of the filter gradient over few samples

struct KeptGradArgs {
    const unsigned char *codes, *scales;
    const void *dy;
    float *dw;                   // [O][I], or one such for every split
    int64_t pitch, dy_stride;
    int N, I, O;
    int itiles, otiles, splits, rows_per_split;
    int units, per_xcd;
};

struct KeptGradPlan {
    KeptGradArgs a;
    int slices;                   // few samples: sixteens of them; 0: tiles, or no samples
    int outputs;                  // to a launch
    int tile, step;               // outputs, and inputs, of a tile; rows of a step
    int64_t blocks;               // the grid
    size_t part_bytes;
};

inline int plan_kept_grad(KeptGradPlan &p, int N, int I, int O, int dtype)
{
    p = {};
    if (N < 0 || I <= 0 || O <= 0) return kErrInvalidArg;
    if (!glue_elem_bytes(dtype)) return kErrBadDtype;
    if (N * pitch_of(I) >= kMaxElements || (int64_t)N * O >= kMaxElements || (int64_t)I * O >= kMaxElements) return kErrTooLarge;
    KeptGradArgs &a = p.a;
    a.N = N; a.I = I; a.O = O;
    a.pitch = pitch_of(I);
    a.dy_stride = O;
    a.splits = 1;
    p.outputs = O;
    if (N == 0) return kStatusOk;                            // dw is filled
    // The gradients stay in registers, and a work-group goes through its share of the inputs (9216 -> 4096, three states in turn): 128
    // rows fp32 37 us, 52 in tiles, bfloat16 34 and 40; one row 32 and 33, 32 and 38.
    if (N <= 128) {
        p.slices = N <= 16 ? 1 : N <= 32 ? 2 : N <= 64 ? 4 : 8;
        p.outputs = std::min(O, 1 << 30);                    // (a launch has fewer than 2^32 threads)
        a.otiles = parts_of(p.outputs, 128);
        const int inputs = parts_of(I, kFewInputs), shares = std::max(1, std::min(inputs, 768 / a.otiles));
        a.rows_per_split = ceil_div(inputs, shares);
        a.itiles = ceil_div(inputs, a.rows_per_split);
        p.blocks = (int64_t)a.otiles * a.itiles;
        return kStatusOk;
    }
    // Large tiles, one work-group to a CU, feed the matrix units with half the traffic, where they fill the rounds of 256 that they
    // run in: 8192 rows 4096 -> 4096 bfloat16 220 us, 288 in tiles of 128, fp32 635 and 767; 9216 -> 4096 (576 tiles, three rounds)
    // 643 and 642, fp32 1716 and 1714
    const int64_t large = (int64_t)ceil_div(I, 256) * ceil_div(O, 256);
    p.tile = N >= 1024 && large >= 0.77 * round_up64(large, 256) ? 256 : 128;
    // fp32 over few rows: shorter steps leave room for more work-groups, one of which stores while others multiply (130 rows
    // 9216 -> 4096 55 us, and 66; 256 rows 75 and 78); over many the longer ones are faster (1024 rows 4096 -> 4096 100 and 106)
    p.step = glue_elem_bytes(dtype) == 2 ? 64 : p.tile == 128 && N <= 256 ? 16 : 32;
    a.itiles = ceil_div(I, p.tile);
    a.otiles = ceil_div(O, p.tile);
    const int64_t tiles = (int64_t)a.itiles * a.otiles;
    const int steps = std::max(1, ceil_div(N, p.step));
    // as many parts of the sum as fill the card, of 256 rows at least: each is written and read again
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>((p.tile == 256 ? 256 : 512) / tiles, N / 256));
    const int per = ceil_div(steps, a.splits);
    a.rows_per_split = per * p.step;
    a.splits = ceil_div(steps, per);
    a.units = (int)(tiles * a.splits);
    a.per_xcd = ceil_div(a.units, 8);
    p.blocks = (int64_t)8 * a.per_xcd;
    if (a.splits > 1) p.part_bytes = (size_t)round_up64((int64_t)a.splits * I * O * 4, 256);
    return kStatusOk;
}

inline int check_q4(int N, int I, int O, int dtype)
{
    if (N < 0 || I <= 0 || O <= 0) return kErrInvalidArg;
    if (!glue_elem_bytes(dtype)) return kErrBadDtype;
    if (N * pitch_of(I) >= kMaxElements || O * pitch_of(I) >= kMaxElements || (int64_t)N * O >= kMaxElements) return kErrTooLarge;
    return kStatusOk;
}

// The kernel for N > 32 samples: 0 the one for few, else the edge of the tiles.  Large tiles feed the matrix units with half the
// traffic, where there is one for most of the CUs and the sum is long (x and y bfloat16, us a call, tiles of 256 and of 128):
// 2048 x 8192 -> 8192 78 and 99, 1024 x 8192 -> 8192 58 and 53, 4096 x 4096 -> 4096 50 and 58, 2048 x 4096 -> 4096 39 and 33,
// 8192 x 1024 -> 8192 77 and 70.  Few samples: what the two would take in us, by fits to calls like these (for few, and tiles of
// 128): 64 x 8192 -> 8192 15 and 24, 256 x 8192 -> 8192 39 and 27, 256 x 9216 -> 4096 26 and 29, 512 x 9216 -> 4096 44 and 31,
// 256 x 4096 -> 4096 16.6 and 15.9, 512 x 4096 -> 1000 11 and 16, 1024 x 4096 -> 1000 19 and 17.
inline int q4_tile(int N, int O, int steps)
{
    if ((int64_t)ceil_div(N, 256) * ceil_div(O, 256) >= 192 && steps >= 16) return 256;
    const double units = (double)ceil_div(N, 64) * ceil_div(O, 32), tiles = (double)ceil_div(N, 128) * ceil_div(O, 128);
    const double few = 5.0 + 2.0 * ceil(units / 256) + units * 96 * 64 * steps / 12e6;
    const double many = 6.3 + 0.31 * steps * std::max(1.0, tiles / 240);
    return few < many ? 0 : 128;
}

// How a call runs, and where its scratch lies: x's codes, and the exponents of both operands by steps.
struct Q4Plan {
    bool fused;
    int tile;                                        // of the kernel for many samples, 0: the one for few
    int steps, nrows, orows;
    int wide;                                        // blocks of 16 samples to a work-group of the kernel for few
    size_t xs, ws, total;
};

inline Q4Plan plan_q4(int N, int I, int O)
{
    Q4Plan p = {};
    p.steps = (int)(pitch_of(I) / kRowFill);
    p.tile = N > 32 ? q4_tile(N, O, p.steps) : 0;
    // a launch for x less (4 samples 4096 -> 4096 5.5 us, and 8.8), as long as every work-group's putting x into blocks takes less
    // than that: 8 x 4096 -> 4096 7.2 and 8.9, 4 x 8192 -> 8192 11.7 and 12.4, 4 x 9216 -> 4096 8.3 and 8.0, 8 x 8192 -> 8192 21 and 13
    p.fused = N <= 16 && (int64_t)N * p.steps * 128 <= 32768;
    if (p.fused) return p;
    p.wide = N <= 16 ? 1 : N <= 32 ? 2 : 4;
    p.xs = (size_t)round_up64((int64_t)N * p.steps * 64, 256);
    p.nrows = round_up(N, p.tile ? p.tile : 16 * p.wide);
    p.orows = round_up(O, p.tile ? p.tile : 32);
    p.ws = p.xs + (size_t)p.steps * p.nrows * 4;
    p.total = p.ws + (size_t)p.steps * p.orows * 4;
    return p;
}
