// Group normalisation with an activation, forward and backward.
// Part of train_ops.hip: included there, inside its anonymous namespace, after vectors.h.
//
//   mean = sum x / M, var = sum (x - mean)^2 / M, xh = (x - mean) rstd, z = gamma xh + beta, y = act(z)
//   dz = dy act'(z); per channel A = sum dz, B = sum dz xh; m1 = sum_c gamma A / M, m2 = sum_c gamma B / M
//   dx = rstd (gamma dz - m1 - xh m2); dbeta = sum_n A, dgamma = sum_n B
//
// Bound by memory: forward has to read x and write y, backward to read x and dy and write dx; some 10 to 30 vector
// operations to a value fit beside that.  So a value is read once and stays in registers until its result is written
// (whole), wherever what belongs to a statistic fits the registers of one work-group: 16 waves of up to 8 vectors of 16
// bytes a lane, of each tensor (channels last 16 forward, 8 or, fp32, 10 backward).  What does not fit is read twice: a
// launch that leaves sums of tiles (kSums), one that joins them, and one that applies them (kApply).  A large copy moves
// 5.0 TB/s on this card.
//
// Planes: a group's C / groups planes are one run of memory.  A wave's unit is 64 vectors of it: of one plane where planes
// fill units well (long planes: sums per channel are then sums over lanes), or of the planes' vectors one after the other
// (flat; every lane leaves its own sums in LDS, 16 lanes add a plane's).
// Channels last: a work-group takes `cw` neighbouring channels (whole groups) of a sample; a lane keeps its columns and
// walks down the positions.
// A plane's last vector is moved back so that it ends where the plane ends.  The values of the vector before that it holds
// then are zeros for the sums: of x, then of the distances from the mean (forward), and of dy (backward), whose share in
// every sum is then 0.  Only the lanes with such a vector spend operations on it.  (Sums that take in copies of a value and
// take them off again turn an infinity into a NaN.)  A slab's last vector is moved back too; its first values are the ones
// of the vector before it, are left out of the sums and written twice, the same.

constexpr int kWhole = 0, kSums = 1, kApply = 2;
constexpr float kLog2e = 1.44269504088896340736f;

struct NormArgs {
    const void *x, *dy;
    void *out;                       // y or dx
    const float *gamma, *beta;       // nullptr: ones, zeros
    float *mean, *rstd;              // forward: results (nullptr: not wanted); backward and kApply: read
    float *part;                     // sums of tiles.  forward: {mean, sum of squares, count}; backward: A, then B, of a row of C
    float *joined;                   // forward kApply, unless it joins the tiles itself (join): means, then rstds
    float *group_sums;               // backward kApply: {m1, m2} of every sample and group
    float *sample_sums;              // backward: A, then B, of every sample and channel (`part` itself where a sample has one row)
    float *dgamma, *dbeta;
    int N, C, S, groups, cpg, act, join;
    double inv_m64;                  // 1 / M, also as inv_m
    float eps, inv_m;
    FastDiv div_groups, div_cpg;
    int part_rows, rows_per_sample;  // rows of C sums in `part`, and of those a sample's
    int join_lanes;                  // threads to channels where a group's sums are joined
    // planes
    int flat, vectors, chunks, units;         // vectors and units to a plane (long planes); units of a group
    int run;                                  // units to a wave
    int tiles, parts, span;                   // of a group; of a plane (0: a tile is whole planes); units or planes of a tile
    float inv_vectors, half_vectors;          // 1 / vectors, and half of that
    FastDiv div_chunks, div_tiles;
    // channels last
    int cw, slab_groups, slabs, lanes, rows;  // channels, groups of a slab; slabs; lanes to a row; rows at a time
    int tile_rows, pitch, group_lanes, channel_lanes, units_per_xcd, work;
    FastDiv div_lanes, div_slabs, div_width;  // width: sums of a group in a thread row (forward)
};

// z is taken the same way everywhere, d = x - mean first and then one multiply-add with gamma rstd and beta: exact at the
// mean however far from zero that is, and the same bits backward as forward, so that both agree on the side of a ReLU.

// The activation is decided once for a vector, so that its values' chains (two of the slow instructions each in a SiLU)
// run beside each other.
// v = act(v * scale + shift)
template <int V, typename F, typename G>
__device__ __forceinline__ void act_fwd(float (&v)[V], int act, F scale, G shift)
{
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = fmaf(v[k], scale(k), shift(k));
    if (act == kActRelu) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = v[k] < 0.f ? 0.f : v[k];           // (a NaN stays)
    } else if (act == kActSilu) {
        // exp2's argument and the reciprocal are rounded: a relative error of about (|z| + 2) 2^-23 below zero, where y is
        // smaller than 2^-24 |z| from z = -17 on
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v[k]));
    }
}

// dy = dy * act'(z) at z = d * scale + shift
template <int V, typename F, typename G>
__device__ __forceinline__ void act_bwd(float (&dy)[V], const float (&d)[V], int act, F scale, G shift)
{
    if (act == kActRelu) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float z = fmaf(d[k], scale(k), shift(k));
            dy[k] = z > 0.f ? dy[k] : 0.f;
        }
    } else if (act == kActSilu) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float z = fmaf(d[k], scale(k), shift(k));
            const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
            dy[k] *= s * fmaf(z, 1.f - s, 1.f);
        }
    }
}

// s / n, with n's reciprocal at hand: the remainder of the first quotient corrects it (a group of one value has that mean)
__device__ __forceinline__ float quotient(float s, float n, float inv)
{
    const float q = s * inv;
    return fmaf(fmaf(-q, n, s), inv, q);
}

// the waves' values joined in their order; `red` holds one per wave.  Every thread gets the sum.
template <typename F>
__device__ __forceinline__ F join_waves(F v, F *red, int nw)
{
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    F s = red[0];
    for (int i = 1; i < nw; ++i) s += red[i];
    return s;
}

// The tiles' means and squared distances of a group, joined to the group's over the lanes of a wave, four loads of each
// kind in flight at once.  In 64 bits, as distances from the first tile's mean r0: sum n (m_t - r0) and
// sum (d_t + n (m_t - r0)^2).  The variance is then a difference, but of terms that r0's own tile bounds by the number of tiles
// times the variance, below 2^20 of them; tiles of one mean have exactly that mean; and an infinite one stays infinite.
__device__ __forceinline__ void join_tiles(const NormArgs &a, int64_t group, int lane, float &mean, float &rstd)
{
    const float *p = a.part + group * a.tiles * 3;
    const double r0 = __builtin_isfinite(p[0]) ? p[0] : 0.;
    double s = 0., d = 0.;
    for (int t0 = lane; t0 < a.tiles; t0 += 256) {
        float tm[4], td[4], tn[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int t = min(t0 + 64 * u, a.tiles - 1);
            tm[u] = p[3 * t];
            td[u] = p[3 * t + 1];
            tn[u] = p[3 * t + 2];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (t0 + 64 * u < a.tiles) {
                const double gap = tm[u] - r0, w = tn[u] * gap;
                s += w;
                d += fma(w, gap, (double)td[u]);
            }
    }
    const double shift = wave_sum(s) * a.inv_m64;
    mean = (float)(r0 + shift);
    rstd = 1.f / sqrtf((float)(wave_sum(d) * a.inv_m64 - shift * shift) + a.eps);
}

// ---------------------------------------------------------------------------
// Planes
// ---------------------------------------------------------------------------
// Forward 128 x 96 planes of 3025 fp32 in 32 groups 58 us, 5.1 TB/s: at the copy's rate.  One sample of 256 planes of 169: 3.7
// us, the launch and one trip to memory.  Backward 128 x 256 planes of 729 fp32 53 us, 5.4 TB/s (part of it stays in the
// last cache), and 4.8 us for the gradients of gamma and beta, a launch.  Bfloat16 is bound by the vector units, which are
// busy for 91 % of the cycles of CUs that hold work in backward on 256 x 384 planes of 169 with a SiLU (26 us, 3.9 TB/s; two
// quarter-rate operations and some 25 others to a value), and for 85 % in forward with a ReLU there (18 to 20 us, 3.6 TB/s).
// (The bound on the registers costs the sums of bfloat16 tiles one spilt register.)
// The group, planes and units of a work-group (SOLO: of a wave; four groups to a work-group, then).
struct PlaneTile {
    int64_t group;
    int g, tile;
    int first, planes;               // of the group
    int u0, u1;                      // units: long planes: of the group; flat: of the tile
    bool live;
};

template <bool SOLO, int MODE>
__device__ __forceinline__ PlaneTile plane_tile(const NormArgs &a)
{
    PlaneTile t;
    t.tile = 0;
    t.first = 0;
    t.planes = a.cpg;
    t.u0 = 0;
    t.u1 = a.units;
    t.live = true;
    int group;
    if (SOLO) {
        const int total = a.N * a.groups;
        group = uniform((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
        t.live = group < total;
        group = min(group, total - 1);
    } else if (MODE == kWhole) {
        group = blockIdx.x;
    } else {
        group = fastdiv(blockIdx.x, a.div_tiles);
        t.tile = blockIdx.x - group * a.tiles;
        if (a.parts) {                           // a part of one plane
            t.first = t.tile / a.parts;
            t.planes = 1;
            t.u0 = t.first * a.chunks + (t.tile - t.first * a.parts) * a.span;
            t.u1 = min(t.u0 + a.span, (t.first + 1) * a.chunks);
        } else {                                 // a.span whole planes
            t.first = t.tile * a.span;
            t.planes = min(a.span, a.cpg - t.first);
            t.u0 = a.flat ? 0 : t.first * a.chunks;
            t.u1 = a.flat ? (t.planes * a.vectors + 63) >> 6 : t.u0 + t.planes * a.chunks;
        }
    }
    t.g = group - fastdiv(group, a.div_groups) * a.groups;
    t.group = group;
    return t;
}

// A lane's vector: channel in the group, first value in the group (before the plane if it is shorter than a vector), and
// whether there is one and it is moved back.
struct PlaneLane {
    int c, off;
    bool on, tail;
};

template <int V>
__device__ __forceinline__ PlaneLane plane_lane(const NormArgs &a, const PlaneTile &t, int u, int lane)
{
    PlaneLane p;
    int pos;
    if (a.flat) {
        // f / vectors: f is below 2^16 here, and (f + 1/2) / vectors in fp32 is far enough from a whole number.  Full-rate
        // operations; a division by multiplication of integers takes four times as long, and so do their products.
        const int f = u * 64 + lane, j = (int)fmaf((float)f, a.inv_vectors, a.half_vectors);
        p.c = t.first + j;
        pos = (f - __mul24(j, a.vectors)) * V;
        p.on = j < t.planes;
        p.off = t.first * a.S + __mul24(j, a.S) + min(pos, a.S - V);
    } else {
        p.c = fastdiv(u, a.div_chunks);
        pos = ((u - p.c * a.chunks) * 64 + lane) * V;
        p.on = pos < a.S;
        p.off = p.c * a.S + min(pos, a.S - V);
    }
    p.tail = pos > a.S - V;
    if (!p.on) {
        p.c = 0;
        p.off = 0;
    }
    return p;
}

template <typename T>
__device__ __forceinline__ typename Vec<T>::Raw plane_load(const NormArgs &a, const T *p, const PlaneLane &l, int moved)
{
    if (a.S >= Vec<T>::V) return Vec<T>::load(p + l.off);
    return Vec<T>::ends(p + l.off, l.on ? moved : Vec<T>::V);
}

template <typename T>
__device__ __forceinline__ void plane_store(T *p, const PlaneLane &l, int moved, const float (&v)[Vec<T>::V])
{
    if (l.on && !l.tail) Vec<T>::store(p + l.off, v);
    if (moved == 0) return;
#pragma unroll
    for (int k = 0; k < Vec<T>::V; ++k)
        if (k >= moved && l.on && l.tail) Vec<T>::put(p, l.off + k, v[k]);
}

template <typename T, int R, bool SOLO, int MODE>
__global__ __launch_bounds__(SOLO ? 256 : 1024, R <= 4 ? 8 : 6) void group_norm_planes_fwd(NormArgs a)
{
    constexpr int V = Vec<T>::V;
    __shared__ float red[3][16];
    const int lane = threadIdx.x & 63, wave = SOLO ? 0 : uniform((int)(threadIdx.x >> 6));
    const int nw = SOLO ? 1 : (int)(blockDim.x >> 6);
    const PlaneTile t = plane_tile<SOLO, MODE>(a);
    const int64_t base = t.group * a.cpg * a.S;
    const T *x = static_cast<const T *>(a.x) + base;
    typename Vec<T>::Raw raw[R];
    PlaneLane pl[R];
    const int u0 = t.u0 + wave * a.run, n = min(a.run, t.u1 - u0);
    const int moved = (V - a.S % V) % V;         // values of a moved-back vector that are the vector's before it
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < n) {
            pl[r] = plane_lane<V>(a, t, u0 + r, lane);
            raw[r] = plane_load(a, x, pl[r], moved);
        }
    float mean, rstd;
    if (MODE == kApply) {
        if (a.join) {
            join_tiles(a, t.group, lane, mean, rstd);
            if (t.tile == 0 && threadIdx.x == 0) {
                if (a.mean) a.mean[t.group] = mean;
                if (a.rstd) a.rstd[t.group] = rstd;
            }
        } else {
            mean = a.joined[t.group];
            rstd = a.joined[a.N * a.groups + t.group];
        }
    } else {
        float s = 0.f, cnt = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < n) {
                if (moved && pl[r].tail) {
                    as_branch();
                    Vec<T>::clear_first(raw[r], moved);
                }
                float v[V];
                Vec<T>::open(raw[r], v);
                if (pl[r].on) {
#pragma unroll
                    for (int k = 0; k < V; ++k) s += v[k];
                    if (MODE == kSums) cnt += pl[r].tail ? V - moved : V;
                }
            }
        s = wave_sum(s);
        if (!SOLO) s = join_waves(s, red[0], nw);
        mean = (float)(s * a.inv_m64);
        if (MODE == kSums) {
            cnt = join_waves(wave_sum(cnt), red[2], nw);       // at most 2^16 values to a tile: exact
            mean = s / cnt;
        }
        s = 0.f;
        if (MODE == kWhole) open_again(raw);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < n) {
                float v[V];
                Vec<T>::open(raw[r], v);
                if (pl[r].on) {
#pragma unroll
                    for (int k = 0; k < V; ++k) v[k] -= mean;
                    if (moved && pl[r].tail) {
                        as_branch();
#pragma unroll
                        for (int k = 0; k < V - 1; ++k)
                            if (k < moved) v[k] = 0.f;
                    }
#pragma unroll
                    for (int k = 0; k < V; ++k) s = fmaf(v[k], v[k], s);
                }
            }
        s = wave_sum(s);
        if (!SOLO) s = join_waves(s, red[1], nw);
        if (MODE == kSums) {
            if (threadIdx.x == 0) {
                float *p = a.part + (t.group * a.tiles + t.tile) * 3;
                p[0] = mean;
                p[1] = s;
                p[2] = cnt;
            }
            return;
        }
        rstd = 1.f / sqrtf(s * a.inv_m + a.eps);
        if (t.live && lane == 0 && wave == 0) {
            if (a.mean) a.mean[t.group] = mean;
            if (a.rstd) a.rstd[t.group] = rstd;
        }
    }
    if (MODE == kWhole) open_again(raw);
    T *y = static_cast<T *>(a.out) + base;
    const int c0 = t.g * a.cpg;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < n && t.live) {
            const float scale = rstd * (a.gamma ? a.gamma[c0 + pl[r].c] : 1.f);
            const float shift = a.beta ? a.beta[c0 + pl[r].c] : 0.f;
            float v[V];
            Vec<T>::open(raw[r], v);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] -= mean;
            act_fwd(v, a.act, [&](int) { return scale; }, [&](int) { return shift; });
            plane_store(y, pl[r], moved, v);
        }
}

// With d = x - mean: z = gamma rstd d + beta, B = rstd sum dz d, dx = gamma rstd dz - rstd m1 - d rstd^2 m2.
// Sums per channel go through slots in LDS: of long planes four to a unit (16 lanes are added by moves within a row of
// lanes; consecutive units of a wave that lie in one plane are added before that), flat one to a lane.
template <typename T, int R, bool SOLO, int MODE>
__global__ __launch_bounds__(SOLO ? 256 : 1024, R <= 2 ? 8 : R <= 4 ? 5 : 4) void group_norm_planes_bwd(NormArgs a)
{
    constexpr int V = Vec<T>::V;
    constexpr bool kKeep = MODE == kWhole && (sizeof(T) == 4 || R <= 4);       // dz stays in registers, else it is computed twice
    extern __shared__ float slots[];             // A of every unit's runs, then B
    const int lane = threadIdx.x & 63, wave = SOLO ? 0 : uniform((int)(threadIdx.x >> 6));
    const PlaneTile t = plane_tile<SOLO, MODE>(a);
    const int64_t base = t.group * a.cpg * a.S;
    const T *x = static_cast<const T *>(a.x) + base, *dy = static_cast<const T *>(a.dy) + base;
    typename Vec<T>::Raw rx[R], rd[R];
    // where a vector lies, gamma rstd and beta there: kept, or with many vectors found again for each use (`at` is the
    // lane, hidden from the compiler so that it does not keep them after all)
    constexpr bool kFew = R <= 4;
    PlaneLane pl[kFew ? R : 1];
    float scale[kFew ? R : 1], shift[kFew ? R : 1];
    int at = lane;
    float dz[kKeep ? R : 1][V];
    const int u0 = t.u0 + wave * a.run, n = min(a.run, t.u1 - u0);
    const int c0 = t.g * a.cpg;
    const int moved = (V - a.S % V) % V;         // values of a moved-back vector that are the vector's before it
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < n) {
            const PlaneLane l = plane_lane<V>(a, t, u0 + r, lane);
            rx[r] = plane_load(a, x, l, moved);
            rd[r] = plane_load(a, dy, l, moved);
            if constexpr (kFew) {
                pl[r] = l;
                scale[r] = a.gamma ? a.gamma[c0 + l.c] : 1.f;
                shift[r] = a.beta ? a.beta[c0 + l.c] : 0.f;
            }
        }
    const float mean = a.mean[t.group], rstd = a.rstd[t.group];
    auto find = [&](int r, PlaneLane &l, float &sc, float &sh) {
        if constexpr (kFew) {
            l = pl[r];
            sc = scale[r] * rstd;
            sh = shift[r];
        } else {
            l = plane_lane<V>(a, t, u0 + r, at);
            sc = (a.gamma ? a.gamma[c0 + l.c] : 1.f) * rstd;
            sh = a.beta ? a.beta[c0 + l.c] : 0.f;
        }
    };
    float m1, m2;
    if (MODE == kApply) {
        m1 = a.group_sums[2 * t.group];
        m2 = a.group_sums[2 * t.group + 1];
    } else {
        // slots of the tile; a plane's are neighbours.  Then the planes' sums, times gamma
        const int per = a.flat ? a.vectors : 4 * (a.parts ? t.u1 - t.u0 : a.chunks), count = per * t.planes;
        float *slot_a = slots + (SOLO ? (int)(threadIdx.x >> 6) * 2 * (count + t.planes) : 0), *slot_b = slot_a + count;
        float *plane_a = slot_b + count, *plane_b = plane_a + t.planes;
        float A = 0.f, B = 0.f;
        if (!kFew) asm volatile("" : "+v"(at));
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < n) {
                PlaneLane l;
                float sc, sh, xv[V], dv[V];
                find(r, l, sc, sh);
                if (moved && l.tail) {
                    as_branch();
                    Vec<T>::clear_first(rd[r], moved);
                }
                Vec<T>::open(rx[r], xv);
                Vec<T>::open(rd[r], dv);
#pragma unroll
                for (int k = 0; k < V; ++k) xv[k] -= mean;
                act_bwd(dv, xv, a.act, [&](int) { return sc; }, [&](int) { return sh; });
                if (l.on) {
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        A += dv[k];
                        B = fmaf(dv[k], xv[k], B);
                    }
                }
                if constexpr (kKeep) {
#pragma unroll
                    for (int k = 0; k < V; ++k) dz[r][k] = dv[k];
                }
                const int u = u0 + r;
                if (a.flat) {
                    const int slot = u * 64 + lane;
                    if (slot < count) {
                        slot_a[slot] = A;
                        slot_b[slot] = B * rstd;
                    }
                    A = B = 0.f;
                } else {
                    // a wave's last unit in a plane gets the sum of those before it there
                    float ta = 0.f, tb = 0.f;
                    if (r + 1 == n || (int)fastdiv(u + 1, a.div_chunks) != (int)fastdiv(u, a.div_chunks)) {
                        ta = run_sum(A, 16);
                        tb = run_sum(B, 16) * rstd;
                        A = B = 0.f;
                    }
                    if ((lane & 15) == 0) {
                        const int slot = (u - t.u0) * 4 + (lane >> 4);
                        slot_a[slot] = ta;
                        slot_b[slot] = tb;
                    }
                }
            }
        __syncthreads();
        const int64_t n_group = fastdiv((uint32_t)t.group, a.div_groups);
        const int64_t row = n_group * a.rows_per_sample + (a.parts ? t.tile - t.first * a.parts : 0);
        const int teams = SOLO ? 4 : (int)(blockDim.x >> 4), sub = lane & 15;
        for (int j0 = 0; j0 < t.planes; j0 += teams) {
            const int j = j0 + ((SOLO ? lane : (int)threadIdx.x) >> 4), c = c0 + t.first + j;
            float sa = 0.f, sb = 0.f;
            if (j < t.planes)
                for (int i = j * per + sub; i < (j + 1) * per; i += 16) {
                    sa += slot_a[i];
                    sb += slot_b[i];
                }
            sa = run_sum(sa, 16);
            sb = run_sum(sb, 16);
            if (j < t.planes && sub == 0) {
                const float gamma = a.gamma ? a.gamma[c] : 1.f;
                plane_a[j] = gamma * sa;
                plane_b[j] = gamma * sb;
                if (t.live) {
                    a.part[row * a.C + c] = sa;
                    a.part[((int64_t)a.part_rows + row) * a.C + c] = sb;
                }
            }
        }
        if (MODE == kWhole) {
            __syncthreads();
            float p = 0.f, q = 0.f;
            for (int j = lane; j < t.planes; j += 64) {
                p += plane_a[j];
                q += plane_b[j];
            }
            m1 = wave_sum(p) * a.inv_m;
            m2 = wave_sum(q) * a.inv_m;
        }
        if (MODE == kSums) return;
    }
    const float c1 = rstd * m1, c2 = rstd * rstd * m2;
    T *dx = static_cast<T *>(a.out) + base;
    if (!kFew) asm volatile("" : "+v"(at));
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < n && t.live) {
            PlaneLane l;
            float sc, sh, xv[V], dv[V];
            find(r, l, sc, sh);
            Vec<T>::open(rx[r], xv);
            Vec<T>::open(rd[r], dv);
#pragma unroll
            for (int k = 0; k < V; ++k) xv[k] -= mean;
            if constexpr (kKeep) {
#pragma unroll
                for (int k = 0; k < V; ++k) dv[k] = dz[r][k];
            } else {
                act_bwd(dv, xv, a.act, [&](int) { return sc; }, [&](int) { return sh; });
            }
#pragma unroll
            for (int k = 0; k < V; ++k) dv[k] = fmaf(-xv[k], c2, fmaf(sc, dv[k], -c1));
            plane_store(dx, l, moved, dv);
        }
}

// ---------------------------------------------------------------------------
// Channels last
// ---------------------------------------------------------------------------
// Forward 128 x 256 x 27 x 27 bf16 in 32 groups 23 us, 4.2 TB/s (vector units busy for 72 % of the cycles of CUs that hold
// work).  4 x 64 x 224 x 224 bf16 in 8 groups, in tiles: 9.0 us for the sums and 13.9 for the rest, 2.2 TB/s counting x once, 3.4
// as it is read.  Backward 64 x 96 x 55 x 55 fp32 70 us, 3.2 TB/s: columns of 48 bytes in the registers of 1008 threads, so
// that one work-group lives on a CU, two of them one after the other, and the reads, sums and writes of one do not overlap
// with another's; and parts of lines are written, 110 MB in place of 74.  In tiles, which do overlap but read x and dy twice,
// 84 us (and 5 for their join).
//
// Backward on bfloat16 has eight fp32 sums of each kind to a thread beside its vectors, and with 6 or 8 vectors of several
// groups 7 and 24 registers go to memory and back (8 vectors of one group: 3), 4 waves to a SIMD as it is.
struct SlabTile {
    int n, slab, tile, s0, count;    // sample, slab, tile of positions [s0, s0 + count)
    int j, p;                        // this thread's column vector and first row
    int q, k0, k1;                   // its first channel in the slab, valid values k0 <= k < k1
    bool on, live;
};

// Neighbouring slabs share lines of memory, so that a sample's slabs and tiles go to one XCD: work item = (work-groups of
// an XCD) * XCD + its number there, as work-groups go to the eight XCDs in turn.
template <int V>
__device__ __forceinline__ SlabTile slab_tile(const NormArgs &a)
{
    SlabTile t;
    const int item = (int)(blockIdx.x & 7) * a.units_per_xcd + (int)(blockIdx.x >> 3);
    t.live = (int)(blockIdx.x >> 3) < a.units_per_xcd && item < a.work;
    const int i = t.live ? item : 0;
    const int nt = fastdiv(i, a.div_slabs);
    t.slab = i - nt * a.slabs;
    t.n = fastdiv(nt, a.div_tiles);
    t.tile = nt - t.n * a.tiles;
    t.s0 = t.tile * a.tile_rows;
    t.count = min(a.tile_rows, a.S - t.s0);
    t.p = fastdiv(threadIdx.x, a.div_lanes);
    t.j = threadIdx.x - t.p * a.lanes;
    t.on = t.p < a.rows;
    const int c = t.j * V;
    if (a.cw >= V) {
        t.q = min(c, a.cw - V);
        t.k0 = c - t.q;
        t.k1 = V;
    } else {
        t.q = 0;
        t.k0 = 0;
        t.k1 = a.cw;
    }
    return t;
}

template <typename T>
__device__ __forceinline__ typename Vec<T>::Raw slab_load(const NormArgs &a, const T *p, const SlabTile &t)
{
    return a.cw >= Vec<T>::V ? Vec<T>::load(p) : Vec<T>::some(p, t.k1);
}

template <typename T>
__device__ __forceinline__ void slab_store(const NormArgs &a, T *p, const SlabTile &t, const float (&v)[Vec<T>::V])
{
    if (a.cw >= Vec<T>::V) {
        Vec<T>::store(p, v);
    } else {
        for (int k = 0; k < Vec<T>::V; ++k)
            if (k < t.k1) Vec<T>::put(p, k, v[k]);
    }
}

// V neighbouring channels' values of a vector over the channels (nullptr: `none`); a slab of fewer channels than a vector
// repeats its last
template <int V>
__device__ __forceinline__ void slab_params(const NormArgs &a, const SlabTile &t, const float *p, float none, float (&v)[V])
{
    const int ch = t.slab * a.cw + t.q;
    if (!p) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = none;
    } else if (a.cw >= V) {
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const f32x4 q = *reinterpret_cast<const f32x4_any *>(p + ch + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k + i] = q[i];
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = p[ch + min(k, a.cw - 1)];
    }
}

// the group (in the slab) of a vector's values one after the other, from one division
struct GroupWalk {
    int g, left;
    __device__ __forceinline__ GroupWalk(const NormArgs &a, const SlabTile &t)
    {
        g = fastdiv(t.q, a.div_cpg);
        left = a.cpg * (g + 1) - t.q;
    }
    __device__ __forceinline__ int next(const NormArgs &a)
    {
        const int now = g;
        if (--left == 0) {
            left = a.cpg;
            g = min(g + 1, a.slab_groups - 1);       // (past the slab: a vector's values that do not exist)
        }
        return now;
    }
};

// where the sums of channel c of the slab over the rows of thread row p lie: [value of the vector][thread], so that the
// lanes of a wave write neighbouring words
template <int V>
__device__ __forceinline__ int slab_slot(const NormArgs &a, int p, int c)
{
    const int j = c / V, q = a.cw >= V ? min(j * V, a.cw - V) : 0;
    return (c - q) * a.pitch + p * a.lanes + j;
}

// ONE: every vector lies in one group (C / groups a multiple of the vector): a thread then has one sum, not one per value.
// A thread of kSums and kApply takes R rows after R rows of its tile.
template <typename T, int R, int MODE, bool ONE>
__global__ __launch_bounds__(1024) void group_norm_last_fwd(NormArgs a)
{
    constexpr int V = Vec<T>::V, W = ONE ? 1 : V;      // W sums to a thread, of V / W values a row each
    extern __shared__ float lds[];
    float *sum = lds, *dev = lds + W * a.pitch, *gmean = dev + W * a.pitch, *grstd = gmean + a.slab_groups;
    const SlabTile t = slab_tile<V>(a);
    if (!t.live) return;
    const int64_t base = ((int64_t)t.n * a.S + t.s0) * a.C + t.slab * a.cw + t.q;
    const T *x = static_cast<const T *>(a.x) + base;
    typename Vec<T>::Raw raw[R];
    auto load = [&](int p) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (t.on && p + r * a.rows < t.count) raw[r] = slab_load(a, x + (p + r * a.rows) * a.C, t);
    };
    if (MODE == kWhole) load(t.p);
    const int64_t group0 = (int64_t)t.n * a.groups + t.slab * a.slab_groups;
    if (MODE != kApply) {
        // every thread's sums, and squared distances from its own means
        const int whole = t.count / a.rows, extra = t.count - whole * a.rows;       // rows of a thread: whole (+ 1)
        const int mine = whole + (t.p < extra);
        if (t.on) {
            float s[W], d[W];
#pragma unroll
            for (int k = 0; k < W; ++k) s[k] = d[k] = 0.f;
            int done = 0;
            do {
                const int p = t.p + done * a.rows;
                if (MODE != kWhole) load(p);
                const int cnt = min(R, mine - done);
                const float n2 = cnt * (V / W), inv = cnt > 0 ? 1.f / n2 : 0.f;
                float bs[W], bd[W], bm[W];
#pragma unroll
                for (int k = 0; k < W; ++k) bs[k] = bd[k] = 0.f;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (r < cnt) {
                        float v[V];
                        Vec<T>::open(raw[r], v);
#pragma unroll
                        for (int k = 0; k < V; ++k) bs[k % W] += v[k];
                    }
#pragma unroll
                for (int k = 0; k < W; ++k) bm[k] = quotient(bs[k], n2, inv);
                open_again(raw);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (r < cnt) {
                        float v[V];
                        Vec<T>::open(raw[r], v);
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            const float e = v[k] - bm[k % W];
                            bd[k % W] = fmaf(e, e, bd[k % W]);
                        }
                    }
                // joined with the rows before: n1 n2 / (n1 + n2) times the square of the means' distance comes on top
                const float n1 = done * (V / W), inv1 = done ? 1.f / n1 : 0.f, both = n1 * n2 / (n1 + n2);
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    if (MODE != kWhole && done) {
                        const float gap = bm[k] - quotient(s[k], n1, inv1);
                        d[k] += gap * gap * both;
                    }
                    s[k] += bs[k];
                    d[k] += bd[k];
                }
                done += R;
            } while (MODE != kWhole && done < mine);
#pragma unroll
            for (int k = 0; k < W; ++k) {
                sum[k * a.pitch + threadIdx.x] = s[k];
                dev[k * a.pitch + threadIdx.x] = d[k];
            }
        }
        __syncthreads();
        // a group's sum, then its squared distances: those of the parts, and the parts' means' own
        const int width = ONE ? a.cpg / V : a.cpg;                                  // sums of a group in a thread row
        const int lane = threadIdx.x & (a.group_lanes - 1), entries = a.rows * width;
        const int at = threadIdx.x / a.group_lanes, step = blockDim.x / a.group_lanes;
        const float total = (float)t.count * a.cpg;                                 // below 2^24: exact
        const float n_whole = whole * (V / W), n_more = (whole + 1) * (V / W);
        const float inv_whole = whole ? 1.f / n_whole : 0.f, inv_more = 1.f / n_more;
        auto slot = [&](int p, int g, int i) {
            return ONE ? p * a.lanes + g * width + i : slab_slot<V>(a, p, g * width + i);
        };
        for (int g0 = 0; g0 < a.slab_groups; g0 += step) {
            const int g = g0 + at;
            const bool some = g < a.slab_groups;
            float s = 0.f, d = 0.f;
            if (some)
                for (int e = lane; e < entries; e += a.group_lanes) {
                    const int p = fastdiv(e, a.div_width);
                    s += sum[slot(p, g, e - p * width)];
                }
            const float mean = run_sum(s, a.group_lanes) / total;
            if (some)
                for (int e = lane; e < entries; e += a.group_lanes) {
                    const int p = fastdiv(e, a.div_width), i = slot(p, g, e - p * width);
                    const bool more = p < extra;
                    const float diff = quotient(sum[i], more ? n_more : n_whole, more ? inv_more : inv_whole) - mean;
                    if (more || whole) d += dev[i] + (more ? n_more : n_whole) * diff * diff;
                }
            d = run_sum(d, a.group_lanes);
            if (some && lane == 0) {
                if (MODE == kSums) {
                    float *p = a.part + ((group0 + g) * a.tiles + t.tile) * 3;
                    p[0] = mean;
                    p[1] = d;
                    p[2] = total;
                } else {
                    const float rstd = 1.f / sqrtf(d * a.inv_m + a.eps);
                    gmean[g] = mean;
                    grstd[g] = rstd;
                    if (a.mean) a.mean[group0 + g] = mean;
                    if (a.rstd) a.rstd[group0 + g] = rstd;
                }
            }
        }
        if (MODE == kSums) return;
    } else {
        load(t.p);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        if (a.join) {
            for (int g = wave; g < a.slab_groups; g += waves) {
                float mean, rstd;
                join_tiles(a, group0 + g, lane, mean, rstd);
                if (lane == 0) {
                    gmean[g] = mean;
                    grstd[g] = rstd;
                    if (t.tile == 0 && a.mean) a.mean[group0 + g] = mean;
                    if (t.tile == 0 && a.rstd) a.rstd[group0 + g] = rstd;
                }
            }
        } else {
            for (int g = threadIdx.x; g < a.slab_groups; g += blockDim.x) {
                gmean[g] = a.joined[group0 + g];
                grstd[g] = a.joined[a.N * a.groups + group0 + g];
            }
        }
    }
    __syncthreads();
    if (!t.on) return;
    float scale[V], shift[V];
    slab_params<V>(a, t, a.gamma, 1.f, scale);
    slab_params<V>(a, t, a.beta, 0.f, shift);
    float mean[W], rstd = 0.f;
    GroupWalk walk(a, t);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if (k < W) {
            const int g = walk.next(a);
            mean[k] = gmean[g];
            rstd = grstd[g];
        }
        scale[k] *= rstd;
    }
    T *y = static_cast<T *>(a.out) + base;
    if (MODE == kWhole) open_again(raw);
    int p = t.p;
    do {
        if (MODE == kApply && p != t.p) load(p);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int s = p + r * a.rows;
            if (s < t.count) {
                float v[V];
                Vec<T>::open(raw[r], v);
#pragma unroll
                for (int k = 0; k < V; ++k) v[k] -= mean[k % W];
                act_fwd(v, a.act, [&](int k) { return scale[k]; }, [&](int k) { return shift[k]; });
                slab_store(a, y + s * a.C, t, v);
            }
        }
        p += R * a.rows;
    } while (MODE != kWhole && p < t.count);
}

template <typename T, int R, int MODE, bool ONE>
__global__ __launch_bounds__(1024) void group_norm_last_bwd(NormArgs a)
{
    constexpr int V = Vec<T>::V, W = ONE ? 1 : V;      // W groups to a vector at most
    // d and dz stay in registers, in fp32 in the places of x and dy; with many bfloat16 vectors they are computed twice
    constexpr bool kInPlace = MODE == kWhole && sizeof(T) == 4, kKeep = MODE == kWhole && sizeof(T) == 2 && R <= 4 && ONE;
    extern __shared__ float lds[];
    float *sa = lds, *sb = lds + V * a.pitch, *ca = sb + V * a.pitch, *cb = ca + a.cw, *g1 = cb + a.cw, *g2 = g1 + a.slab_groups;
    const SlabTile t = slab_tile<V>(a);
    if (!t.live) return;
    const int64_t base = ((int64_t)t.n * a.S + t.s0) * a.C + t.slab * a.cw + t.q;
    const T *x = static_cast<const T *>(a.x) + base, *dy = static_cast<const T *>(a.dy) + base;
    typename Vec<T>::Raw rx[R], rd[R];
    float dz[kKeep ? R : 1][V];
    auto load = [&](int p) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (t.on && p + r * a.rows < t.count) {
                rx[r] = slab_load(a, x + (p + r * a.rows) * a.C, t);
                rd[r] = slab_load(a, dy + (p + r * a.rows) * a.C, t);
            }
    };
    if (MODE == kWhole) load(t.p);
    const int64_t group0 = (int64_t)t.n * a.groups + t.slab * a.slab_groups;
    float mean[W], scale[V], shift[V];
    slab_params<V>(a, t, a.gamma, 1.f, scale);
    slab_params<V>(a, t, a.beta, 0.f, shift);
    {
        float rstd = 0.f;
        GroupWalk walk(a, t);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (k < W) {
                const int64_t g = group0 + walk.next(a);
                mean[k] = a.mean[g];
                rstd = a.rstd[g];
            }
            scale[k] *= rstd;
        }
    }
    // d = x - mean and dz of a vector
    auto slopes = [&](int r, float (&xv)[V], float (&dv)[V]) {
        Vec<T>::open(rx[r], xv);
        Vec<T>::open(rd[r], dv);
#pragma unroll
        for (int k = 0; k < V; ++k) xv[k] -= mean[k % W];
        act_bwd(dv, xv, a.act, [&](int k) { return scale[k]; }, [&](int k) { return shift[k]; });
    };
    if (MODE != kApply) {
        if (t.on) {
            float A[V], B[V];
#pragma unroll
            for (int k = 0; k < V; ++k) A[k] = B[k] = 0.f;
            int p = t.p;
            do {
                if (MODE == kSums) load(p);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (p + r * a.rows < t.count) {
                        float xv[V], dv[V];
                        slopes(r, xv, dv);
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            A[k] += dv[k];
                            B[k] = fmaf(dv[k], xv[k], B[k]);
                            if constexpr (kKeep) dz[r][k] = dv[k];
                            if constexpr (kInPlace) {
                                rx[r][k] = xv[k];
                                rd[r][k] = dv[k];
                            }
                        }
                    }
                p += R * a.rows;
            } while (MODE != kWhole && p < t.count);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                sa[k * a.pitch + threadIdx.x] = A[k];
                sb[k * a.pitch + threadIdx.x] = B[k];
            }
        }
        __syncthreads();
        // channels: the sums over the thread rows
        const int64_t row = (int64_t)t.n * a.rows_per_sample + t.tile;
        {
            const int lane = threadIdx.x & (a.channel_lanes - 1);
            const int at = threadIdx.x / a.channel_lanes, step = blockDim.x / a.channel_lanes;
            for (int c0 = 0; c0 < a.cw; c0 += step) {
                const int c = c0 + at;
                float A = 0.f, B = 0.f;
                if (c < a.cw)
                    for (int p = lane; p < a.rows; p += a.channel_lanes) {
                        const int s = slab_slot<V>(a, p, c);
                        A += sa[s];
                        B += sb[s];
                    }
                A = run_sum(A, a.channel_lanes);
                B = run_sum(B, a.channel_lanes);
                if (c < a.cw && lane == 0) {
                    const int ch = t.slab * a.cw + c;
                    const float gamma = a.gamma ? a.gamma[ch] : 1.f;
                    B *= a.rstd[group0 + fastdiv(c, a.div_cpg)];
                    ca[c] = gamma * A;
                    cb[c] = gamma * B;
                    a.part[row * a.C + ch] = A;
                    a.part[((int64_t)a.part_rows + row) * a.C + ch] = B;
                }
            }
        }
        if (MODE == kSums) return;
        __syncthreads();
        const int lane = threadIdx.x & (a.group_lanes - 1);
        const int at = threadIdx.x / a.group_lanes, step = blockDim.x / a.group_lanes;
        for (int g0 = 0; g0 < a.slab_groups; g0 += step) {
            const int g = g0 + at;
            float p = 0.f, q = 0.f;
            if (g < a.slab_groups)
                for (int e = lane; e < a.cpg; e += a.group_lanes) {
                    p += ca[g * a.cpg + e];
                    q += cb[g * a.cpg + e];
                }
            p = run_sum(p, a.group_lanes);
            q = run_sum(q, a.group_lanes);
            if (g < a.slab_groups && lane == 0) {
                g1[g] = p * a.inv_m;
                g2[g] = q * a.inv_m;
            }
        }
        __syncthreads();
    }
    if (!t.on) return;
    float c1[W], c2[W];
    GroupWalk walk(a, t);
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const int g = walk.next(a);
        const float rstd = a.rstd[group0 + g];
        c1[k] = rstd * (MODE == kApply ? a.group_sums[2 * (group0 + g)] : g1[g]);
        c2[k] = rstd * rstd * (MODE == kApply ? a.group_sums[2 * (group0 + g) + 1] : g2[g]);
    }
    T *dx = static_cast<T *>(a.out) + base;
    if (MODE == kWhole) {
        open_again(rx);
        open_again(rd);
    }
    int p = t.p;
    do {
        if (MODE == kApply) load(p);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int s = p + r * a.rows;
            if (s < t.count) {
                float xv[V], dv[V];
                if constexpr (kKeep) {
                    Vec<T>::open(rx[r], xv);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        xv[k] -= mean[k % W];
                        dv[k] = dz[r][k];
                    }
                } else if constexpr (kInPlace) {
                    Vec<T>::open(rx[r], xv);
                    Vec<T>::open(rd[r], dv);
                } else {
                    slopes(r, xv, dv);
                }
#pragma unroll
                for (int k = 0; k < V; ++k) dv[k] = fmaf(-xv[k], c2[k % W], fmaf(scale[k], dv[k], -c1[k % W]));
                slab_store(a, dx + s * a.C, t, dv);
            }
        }
        p += R * a.rows;
    } while (MODE != kWhole && p < t.count);
}

// ---------------------------------------------------------------------------
// Joining the tiles
// ---------------------------------------------------------------------------
// A thread's sums here and in the wide kernels below run over as many tiles, samples or channels as a call has, so they are
// kept in 64 bits (a chain of 4096 like terms in fp32 is off by 600 of its roundings, and all threads' the same way).

// A wave per sample and group, where the tiles are too many for every work-group to join them again.
__global__ __launch_bounds__(256) void group_norm_join_stats(NormArgs a)
{
    const int lane = threadIdx.x & 63, total = a.N * a.groups, i = blockIdx.x * 4 + (threadIdx.x >> 6);
    float mean, rstd;
    join_tiles(a, min(i, total - 1), lane, mean, rstd);
    if (lane == 0 && i < total) {
        a.joined[i] = mean;
        a.joined[total + i] = rstd;
        if (a.mean) a.mean[i] = mean;
        if (a.rstd) a.rstd[i] = rstd;
    }
}

// A work-group per sample and group: its channels' sums over the sample's rows, and {m1, m2} from them.  join_lanes threads
// to neighbouring channels (so that a wave reads runs of memory), the others to the rows, four loads of each kind in flight
// at once.
__global__ __launch_bounds__(1024) void group_norm_join_groups(NormArgs a)
{
    __shared__ float red[2][1024];
    __shared__ double shares[2][16];
    const int n = fastdiv(blockIdx.x, a.div_groups), c0 = (blockIdx.x - n * a.groups) * a.cpg, rows = a.rows_per_sample;
    const float *pa = a.part + (int64_t)n * rows * a.C + c0, *pb = pa + (int64_t)a.part_rows * a.C;
    const int i = threadIdx.x, x = i & (a.join_lanes - 1), sub = i / a.join_lanes, subs = blockDim.x / a.join_lanes;
    double m1 = 0., m2 = 0.;
    for (int c1 = 0; c1 < a.cpg; c1 += a.join_lanes) {
        const int own = min(c1 + x, a.cpg - 1), c = c0 + own;
        double A64 = 0., B64 = 0.;
        for (int t0 = sub; t0 < rows; t0 += 4 * subs) {
            float va[4], vb[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t at = (int64_t)min(t0 + u * subs, rows - 1) * a.C + own;
                va[u] = pa[at];
                vb[u] = pb[at];
            }
#pragma unroll
            for (int u = 1; u < 4; ++u)
                if (t0 + u * subs >= rows) va[u] = vb[u] = 0.f;
            A64 += (va[0] + va[1]) + (va[2] + va[3]);
            B64 += (vb[0] + vb[1]) + (vb[2] + vb[3]);
        }
        float A = (float)A64, B = (float)B64;
        if (subs > 1) {
            __syncthreads();                             // the channels before are read
            red[0][i] = A;
            red[1][i] = B;
            for (int s = subs >> 1; s > 0; s >>= 1) {
                __syncthreads();
                if (sub < s) {
                    red[0][i] = A += red[0][i + s * a.join_lanes];
                    red[1][i] = B += red[1][i + s * a.join_lanes];
                }
            }
        }
        if (sub == 0 && c1 + x < a.cpg) {
            const double gamma = a.gamma ? a.gamma[c] : 1.f;
            m1 += gamma * A;
            m2 += gamma * B;
            a.sample_sums[(int64_t)n * a.C + c] = A;
            a.sample_sums[(int64_t)(a.N + n) * a.C + c] = B;
        }
    }
    m1 = join_waves(wave_sum(m1), shares[0], (int)(blockDim.x >> 6));
    m2 = join_waves(wave_sum(m2), shares[1], (int)(blockDim.x >> 6));
    if (i == 0) {
        a.group_sums[2 * (int64_t)blockIdx.x] = (float)(m1 * a.inv_m64);
        a.group_sums[2 * (int64_t)blockIdx.x + 1] = (float)(m2 * a.inv_m64);
    }
}

// Gradients of gamma and beta: a work-group adds the samples' sums of 16 channels; 16 threads to a channel, eight loads of
// each kind in flight at once.
__global__ __launch_bounds__(256) void group_norm_join_channels(NormArgs a)
{
    __shared__ float red[2][16][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = min((int)(blockIdx.x * 16) + x, a.C - 1);
    const float *pa = a.sample_sums + c, *pb = pa + (int64_t)a.N * a.C;
    double A64 = 0., B64 = 0.;
    for (int n0 = y; n0 < a.N; n0 += 128) {
        float va[8], vb[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t n = min(n0 + 16 * u, a.N - 1);
            va[u] = pa[n * a.C];
            vb[u] = pb[n * a.C];
        }
#pragma unroll
        for (int u = 1; u < 8; ++u)
            if (n0 + 16 * u >= a.N) va[u] = vb[u] = 0.f;
        A64 += ((va[0] + va[1]) + (va[2] + va[3])) + ((va[4] + va[5]) + (va[6] + va[7]));
        B64 += ((vb[0] + vb[1]) + (vb[2] + vb[3])) + ((vb[4] + vb[5]) + (vb[6] + vb[7]));
    }
    red[0][x][y] = (float)A64;
    red[1][x][y] = (float)B64;
    __syncthreads();
    // 16 lanes to a channel
    const int ch = blockIdx.x * 16 + y;
    const float A = run_sum(red[0][y][x], 16), B = run_sum(red[1][y][x], 16);
    if (x == 0 && ch < a.C) {
        if (a.dbeta) a.dbeta[ch] = A;
        if (a.dgamma) a.dgamma[ch] = B;
    }
}

// ---------------------------------------------------------------------------
// Groups of very many channels, channels last (a row of a group is more than a work-group's vectors): one work-group per
// sample and group, a pass over memory for every step, a thread to a channel
// ---------------------------------------------------------------------------
__device__ __forceinline__ double block_sum(double v, double *red)
{
    __syncthreads();
    return join_waves(wave_sum(v), red, (int)(blockDim.x >> 6));
}

template <typename T>
__global__ __launch_bounds__(1024) void group_norm_wide_fwd(NormArgs a)
{
    __shared__ double red[16];
    const int n = fastdiv(blockIdx.x, a.div_groups), c0 = (blockIdx.x - n * a.groups) * a.cpg;
    const T *x = static_cast<const T *>(a.x) + (int64_t)n * a.S * a.C;
    T *y = static_cast<T *>(a.out) + (int64_t)n * a.S * a.C;
    double s = 0.;
    for (int r = 0; r < a.S; ++r)
        for (int c = c0 + threadIdx.x; c < c0 + a.cpg; c += blockDim.x) s += ld_elem(x, r * a.C + c);
    const float mean = (float)(block_sum(s, red) * a.inv_m64);
    s = 0.;
    for (int r = 0; r < a.S; ++r)
        for (int c = c0 + threadIdx.x; c < c0 + a.cpg; c += blockDim.x) {
            const double d = ld_elem(x, r * a.C + c) - mean;
            s = fma(d, d, s);
        }
    const float rstd = 1.f / sqrtf((float)(block_sum(s, red) * a.inv_m64) + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
    for (int c = c0 + threadIdx.x; c < c0 + a.cpg; c += blockDim.x) {
        const float scale = rstd * (a.gamma ? a.gamma[c] : 1.f), shift = a.beta ? a.beta[c] : 0.f;
        for (int r = 0; r < a.S; ++r) {
            float v[1] = {ld_elem(x, r * a.C + c) - mean};
            act_fwd(v, a.act, [&](int) { return scale; }, [&](int) { return shift; });
            st_elem(y, r * a.C + c, v[0]);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void group_norm_wide_bwd(NormArgs a)
{
    __shared__ double red[16];
    const int n = fastdiv(blockIdx.x, a.div_groups), c0 = (blockIdx.x - n * a.groups) * a.cpg;
    const T *x = static_cast<const T *>(a.x) + (int64_t)n * a.S * a.C, *dy = static_cast<const T *>(a.dy) + (int64_t)n * a.S * a.C;
    T *dx = static_cast<T *>(a.out) + (int64_t)n * a.S * a.C;
    const float mean = a.mean[blockIdx.x], rstd = a.rstd[blockIdx.x];
    double m1 = 0., m2 = 0.;
    for (int c = c0 + threadIdx.x; c < c0 + a.cpg; c += blockDim.x) {
        const float gamma = a.gamma ? a.gamma[c] : 1.f, beta = a.beta ? a.beta[c] : 0.f, scale = rstd * gamma;
        double A = 0., B = 0.;
        for (int r = 0; r < a.S; ++r) {
            const float d[1] = {ld_elem(x, r * a.C + c) - mean};
            float dz[1] = {ld_elem(dy, r * a.C + c)};
            act_bwd(dz, d, a.act, [&](int) { return scale; }, [&](int) { return beta; });
            A += dz[0];
            B = fma((double)dz[0], (double)d[0], B);
        }
        B *= rstd;
        a.part[(int64_t)n * a.C + c] = (float)A;
        a.part[((int64_t)a.part_rows + n) * a.C + c] = (float)B;
        m1 += gamma * A;
        m2 += gamma * B;
    }
    const float mean1 = (float)(block_sum(m1, red) * a.inv_m64), mean2 = (float)(block_sum(m2, red) * a.inv_m64);
    for (int c = c0 + threadIdx.x; c < c0 + a.cpg; c += blockDim.x) {
        const float gamma = a.gamma ? a.gamma[c] : 1.f, beta = a.beta ? a.beta[c] : 0.f, scale = rstd * gamma;
        for (int r = 0; r < a.S; ++r) {
            const float d[1] = {ld_elem(x, r * a.C + c) - mean};
            float dz[1] = {ld_elem(dy, r * a.C + c)};
            act_bwd(dz, d, a.act, [&](int) { return scale; }, [&](int) { return beta; });
            st_elem(dx, r * a.C + c, rstd * (gamma * dz[0] - mean1 - d[0] * rstd * mean2));
        }
    }
}
