// Group norms with an activation over the graphs of a batch, forward and backward; rows are nodes, a graph
// is a run of rows, a group a run of D = F / groups features.
//
// With m and v the mean and variance over the M = nodes * D elements of graph b and group g, r = 1 / sqrt(v + eps):
//   u = (X - m) r,  p = weight u + bias,  Y = act(p)
// and for a gradient dY of Y:
//   d = dY act'(p),  dbias = sum d,  dweight = sum d u                  (over all rows of graphs)
//   dX = r (t - mean(t) - u mean(t u)),  t = weight d                   (means over the graph and group)
// so that the sums of t and t u of a group are those of d and d u, column by column, times the weight.
//
// Sums are float64: of x - s and its square for the statistics, s the first element of the graph's group (the
// variance then loses nothing where the mean is large beside it, and is 0 for equal elements).  The differences
// x - m are formed with m as two float32 numbers, so that they are as exact as float32 can be.
//
// A team of one wavefront (where graphs are many and short) or of a workgroup's four takes
//   graphs of up to `limit` rows whole: its second reading of the rows comes from the caches;
// and a workgroup
//   tiles of at most `limit` rows, of which it sums the pieces of longer graphs.  Such a graph has more rows than a tile, so that
//     only those of a tile's first and last row can be in it.  A second launch joins the tiles' sums and a third applies them;
//     neither is made where all rows together are no more than the limit.
// Columns go over the grid's second dimension: whole groups of up to 256 columns, or one wider group in chunks of 256.
// The graphs' offsets are read on the device: the host knows neither their lengths nor whether one of them is long.
//
// Measured: one graph of 2^21 x 256, float32 to bfloat16 with SiLU: 358 us for the sums (6.0 TB/s), 8, and 668 for the rest (4.8 TB/s);
// 4,096 graphs of 0 to 250 nodes, 123,457 x 128: 33.9, 4.8 and 12.4 us, of which memory takes 23: the chain offsets - rows - sums - rows of a
// wavefront's graph, and long graphs' two more launches.  Backward, 2^20 x 128 in seven graphs: 202, 9 and 311 us (5.2 TB/s);
// 30,011 x 99 in 300 graphs with SiLU: 20.7, 5.3 and 12.6 us, chains too.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSlice = 256;                          // columns of a workgroup at a time, at most
constexpr int kAhead = 8, kAheadBack = 4;            // rows a thread has in flight, forward and backward
constexpr int kFew = 32;                             // elements, at most, of a group whose gradient is formed in float64

struct GroupArgs {
    const void *X, *dY;
    const int32_t *ptr;
    const float *weight, *bias;
    void *out;                                       // Y, or dX
    double2 *stats;                                  // [B][G]: mean, r
    int4 *pieces;                                    // [tiles][2] the long graphs of a tile's first and last row: number, first row, rows
    double2 *slots;                                  // [tiles][2][G] their partial sums there; where one graph has both rows, the first
    double2 *joined;                                 // backward: [tiles][G] the sums of the long graph that starts in a tile
    double *columns;                                 // backward: [workgroups][2][F] sums of d u and d
    float *dweight, *dbias;
    double eps;
    int32_t n, B, F, G, D;
    int32_t tile_rows, tiles, limit;
    int32_t width;                                   // columns of a workgroup: whole groups, or kSlice where D is more
    int32_t graph_groups, workgroups;                // workgroups over graphs, and over graphs and tiles
    int32_t lanes;                                   // of a group of whole quads in a power of two of lanes, else 0
    int32_t act;                                     // 0, DUALGCN_RELU or DUALGCN_SILU
    bool fill;                                       // rows of no graph receive zeros
    bool streaming;                                  // the output is more than the caches keep
    bool split;                                      // a workgroup has one group, in chunks of kSlice columns
};

// Where graph b starts, and graph b - 1 ends: within [0, n] whatever the offsets hold.
__device__ __forceinline__ int32_t offset_of(const GroupArgs &a, int b) { return a.ptr ? min(max(a.ptr[b], 0), a.n) : b ? a.n : 0; }

struct Graph {
    int number, first, rows;                         // number < 0: none
    __device__ __forceinline__ double count(const GroupArgs &a) const { return static_cast<double>(rows) * a.D; }
};
// The graphs that two rows are in: with c of the B + 1 offsets at or below a row it is in graph c - 1, before the first
// (0) or behind the last (B + 1).  64 places a step, for both rows in one go.
__device__ __forceinline__ void graphs_at(const GroupArgs &a, const int (&row)[2], Graph (&g)[2]) {
    const int lane = threadIdx.x & 63, end = a.B + 1;
    int lo[2] = {0, 0}, len[2] = {end, end};
    if (a.ptr)
        while (len[0] > 0 || len[1] > 0) {
            int step[2], at[2], below[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                step[i] = (len[i] + 63) / 64;
                at[i] = lo[i] + (lane + 1) * step[i] - 1;
                below[i] = a.ptr[min(max(at[i], 0), end - 1)];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (len[i] <= 0) continue;
                const int k = __popcll(__ballot(at[i] < lo[i] + len[i] && below[i] <= row[i])), was = lo[i] + len[i];
                lo[i] = min(lo[i] + k * step[i], was);
                len[i] = min(step[i] - 1, was - lo[i]);
            }
        }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = a.ptr ? __builtin_amdgcn_readfirstlane(lo[i]) : 1;
        g[i] = Graph{-1, row[i], 0};
        if (c == 0 || c > a.B) continue;
        const int first = min(offset_of(a, c - 1), row[i]);
        g[i] = Graph{c - 1, first, max(offset_of(a, c), row[i] + 1) - first};
    }
}
__device__ __forceinline__ int tile_end(const GroupArgs &a, int t0) { return t0 + min(a.tile_rows, a.n - t0); }

// f(graph, its place of two, its first row in the tile, its rows there) for the long graphs of tile [t0, t1), which the first launch
// finds and writes down for the others.
template <class Fn>
__device__ __forceinline__ void long_pieces(const GroupArgs &a, int tile, int t0, int t1, bool find, Fn f) {
    Graph g[2];
    if (find) {
        graphs_at(a, {t0, t1 - 1}, g);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (g[i].rows <= a.limit) g[i].number = -1;
            if (threadIdx.x == 0 && blockIdx.y == 0) a.pieces[2 * tile + i] = make_int4(g[i].number, g[i].first, g[i].rows, 0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int4 p = a.pieces[2 * tile + i];
            g[i] = Graph{p.x, p.y, p.z};
        }
    }
#pragma unroll 1
    for (int end = 0; end < 2; ++end) {
        const Graph one = end ? g[1] : g[0];
        if (one.number < 0 || (end && one.number == g[0].number)) continue;
        const int from = max(one.first, t0);
        f(one, end, from, min(one.first + one.rows, t1) - from);
    }
}

// A thread's four columns of chunk `chunk` of the workgroup's: their groups, and the place of its first row.  L lanes have a
// row, W wavefronts are a team.
template <int L, int W>
struct Columns {
    static constexpr int kRows = 64 * W / L;         // rows side by side
    int c0, end, first, slot;                        // the chunk's first column and its end, the thread's first, its row
    QuadPlace at;                                    // of the slot's row in a window
    int group[4];
    bool odd;
    __device__ __forceinline__ Columns(const GroupArgs &a, int chunk) {
        c0 = a.split ? static_cast<int>(blockIdx.y) * a.D + chunk * kSlice : static_cast<int>(blockIdx.y) * a.width;
        end = a.split ? min((static_cast<int>(blockIdx.y) + 1) * a.D, c0 + kSlice) : min(a.F, c0 + a.width);
        first = c0 + 4 * (threadIdx.x % L);
        slot = threadIdx.x % (64 * W) / L;
        odd = (end - c0) & 3;
        at.set(static_cast<uint32_t>(slot) * a.F, first, end);
#pragma unroll
        for (int i = 0; i < 4; ++i) group[i] = min(first + i, end - 1) / a.D;
    }
    __device__ __forceinline__ row_f32x4 vector(const float *v, float otherwise) const {
        if (v) return load_quad<false>(v, first, end - first);
        return row_f32x4{otherwise, otherwise, otherwise, otherwise};
    }
    // The place `rows` rows behind the slot's, if that is one of `all`.
    __device__ __forceinline__ QuadPlace row(const GroupArgs &a, int rows, int all) const {
        QuadPlace q = at;
        if (rows + slot >= all) {
            q.at = kNoQuad;
            q.count = q.part = 0;
        } else if (at.at != kNoQuad) {
            q.at = at.at + static_cast<uint32_t>(rows) * a.F;
        }
        return q;
    }
};
__device__ __forceinline__ int chunks_of(const GroupArgs &a) { return a.split ? (a.D + kSlice - 1) / kSlice : 1; }

template <bool BF>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const GroupArgs &a, const void *base, int first, int rows) {
    return row_window<BF>(base, static_cast<int64_t>(first) * a.F, static_cast<int64_t>(rows) * a.F);
}

// What a team has in LDS: the columns' two sums of its wavefronts, two buffers in turn, and the groups' results.
template <int L, int W>
struct TeamMemory {
    double2 buffer[W > 1 ? 2 : 1][W * 4 * L];
    double2 result[4 * L];
};
template <int W>
__device__ __forceinline__ void team_barrier() {
    if constexpr (W > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        __builtin_amdgcn_wave_barrier();
    }
}
__device__ __forceinline__ double from_lane_xor8(double v) { return dpp<0x128>(v); }    // row_ror 8
__device__ __forceinline__ double plus_xor16(double v) {
    const auto h = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    const auto l = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    return __hiloint2double(h[0], l[0]) + __hiloint2double(h[1], l[1]);
}
__device__ __forceinline__ double plus_xor32(double v) {
    const auto h = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
    const auto l = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
    return __hiloint2double(h[0], l[0]) + __hiloint2double(h[1], l[1]);
}
// The sum over the lanes of a wavefront that have the same column (of L) ...
template <int L>
__device__ __forceinline__ double over_rows(double v) {
    if constexpr (L <= 1) {
        v += dpp<0xB1>(v);
        v += dpp<0x4E>(v);
        v += dpp<0x141>(v);
    }
    if constexpr (L <= 8) v += from_lane_xor8(v);
    if constexpr (L <= 16) v = plus_xor16(v);
    if constexpr (L <= 32) v = plus_xor32(v);
    return v;
}
// ... and over `lanes` consecutive ones (a power of two; the same for all): after each step the lanes of a part agree,
// so that mirrors serve as exchanges.
__device__ __forceinline__ double over_lanes(double v, int lanes) {
    if (lanes > 1) v += dpp<0xB1>(v);
    if (lanes > 2) v += dpp<0x4E>(v);
    if (lanes > 4) v += dpp<0x141>(v);
    if (lanes > 8) v += dpp<0x140>(v);
    if (lanes > 16) v = plus_xor16(v);
    if (lanes > 32) v = plus_xor32(v);
    return v;
}

// Two sums of each thread's four columns, over the team's rows and the columns' groups; made(group, sums) turns a group's into
// what the team is to know of it: v[i] for a thread's column i.  Called once or more for each group; `mine` is true for one of the calls.
template <int L, int W, class Made>
__device__ __forceinline__ void group_sums(const GroupArgs &a, const Columns<L, W> &c, double (&s)[4], double (&q)[4], TeamMemory<L, W> &sh, int &turn,
                                           double2 (&v)[4], Made made) {
    double2 *b = sh.buffer[W > 1 ? turn++ & 1 : 0];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6 & (W - 1);
    if (a.lanes) {                                   // a thread has columns of one group, which is so many lanes of a row
        double x = over_lanes(over_rows<L>((s[0] + s[1]) + (s[2] + s[3])), a.lanes);
        double y = over_lanes(over_rows<L>((q[0] + q[1]) + (q[2] + q[3])), a.lanes);
        if constexpr (W > 1) {
            if (lane < L) b[wave * L + lane] = make_double2(x, y);
            team_barrier<W>();
            x = y = 0.0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const double2 one = b[w * L + lane % L];
                x += one.x;
                y += one.y;
            }
        }
        const double2 r = made(c.group[0], make_double2(x, y), threadIdx.x % (64 * W) < L && lane % a.lanes == 0 && c.first < c.end);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = over_rows<L>(s[i]);
        q[i] = over_rows<L>(q[i]);
        if (lane < L) b[wave * 4 * L + 4 * lane + i] = make_double2(s[i], q[i]);
    }
    team_barrier<W>();
    const int groups = (c.end - c.c0) / a.D;
    int lanes = 64;                                  // of a group
    while (lanes * groups > 64 * W && lanes > 1) lanes >>= 1;
    const int k = threadIdx.x % lanes;
    for (int j = threadIdx.x % (64 * W) / lanes; j < (groups + 64 * W / lanes - 1) / (64 * W / lanes) * (64 * W / lanes); j += 64 * W / lanes) {
        double x = 0.0, y = 0.0;
        if (j < groups)
            for (int i = k; i < a.D; i += lanes)
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const double2 one = b[w * 4 * L + j * a.D + i];
                    x += one.x;
                    y += one.y;
                }
        x = over_lanes(x, lanes);
        y = over_lanes(y, lanes);
        if (j < groups) {
            const double2 r = made(c.c0 / a.D + j, make_double2(x, y), k == 0);
            if (k == 0) sh.result[j] = r;
        }
    }
    team_barrier<W>();
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = sh.result[c.group[i] - c.c0 / a.D];
    // (the results stay until every thread has left the next call's first barrier)
}

// 1 / x and 1 / sqrt(x) of normal numbers: the hardware's approximations and Newton's steps for them, to the last place or two.
__device__ __forceinline__ double reciprocal(double x) {
    double y = __builtin_amdgcn_rcp(x);
    y = fma(y, fma(-x, y, 1.0), y);
    return fma(y, fma(-x, y, 1.0), y);
}
__device__ __forceinline__ double reciprocal_root(double x) {
    double y = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-x * y, y, 1.0), y);
    return y;
}

// The mean and r from sums of x - shift and its square.  The quotient's rest is divided too: a mean that float64 holds is met exactly, so that
// elements that are their group's mean (as whole numbers often are) are on no side of it.
__device__ __forceinline__ double2 statistics(double2 sums, double shift, double count, double eps) {
    const double one = reciprocal(count), about = sums.x * one, d = fma(fma(-about, count, sums.x), one, about), v = fma(sums.y, one, -d * d);
    return make_double2(shift + d, reciprocal_root((v > 0.0 ? v : v != v ? v : 0.0) + eps));
}

// The first element of a graph's group.
template <bool BF>
__device__ __forceinline__ double shift_of(const GroupArgs &a, int first, int group) {
    const int64_t at = static_cast<int64_t>(first) * a.F + static_cast<int64_t>(group) * a.D;
    return BF ? bf16_to_float(static_cast<const unsigned short *>(a.X)[at]) : static_cast<const float *>(a.X)[at];
}

// m as two float32 numbers, r, and with them u; for a thread's four columns of one graph.  x - m may be twice float32's largest
// number, and r, more than 2^-128, is then none of its normal ones: half of x and of m, and 2 r, are in its range (2 r but for a
// last place).  A product with 1/2 and a difference round once together; halves lose nothing but where x - m is below 2^-125, whose last places
// they take: there x - m is off by 2^-148 at most.
struct Unit {
    row_f32x4 hi, lo, r;                             // of m / 2, and 2 r
    __device__ __forceinline__ void set(int i, double2 st) {
        const double m = 0.5 * st.x;
        hi[i] = static_cast<float>(m);
        lo[i] = static_cast<float>(m - hi[i]);
        if (!(fabsf(hi[i]) < INFINITY)) lo[i] = 0.f;
        r[i] = static_cast<float>(2.0 * st.y);
    }
    __device__ __forceinline__ row_f32x4 operator()(row_f32x4 x) const {
        row_f32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = (fmaf(0.5f, x[i], -hi[i]) - lo[i]) * r[i];
        return u;
    }
};

// 1 / (1 + exp(-v)) to about 3 units in the last place: exp by base 2, with what the product's rounding leaves off put back.
// (expf and a division take several times the instructions, and the kernels' code is longer than what short graphs do in it.)
__device__ __forceinline__ float sigmoid(float v) {
    constexpr float kLog2e = 0x1.715476p0f, kRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;        // log2(e) = kLog2e + kRest
    const float x = -fminf(fmaxf(v, -120.f), 120.f), a = x * kLog2e;
    const float rest = fmaf(x, kRest, fmaf(x, kLog2e, -a));
    const float e = __builtin_amdgcn_exp2f(a) * fmaf(rest, kLn2, 1.f);
    return __builtin_amdgcn_rcpf(1.f + e);
}

// act(p) (NaN stays NaN)
__device__ __forceinline__ row_f32x4 activated(row_f32x4 p, int act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (act == DUALGCN_RELU) p[i] = p[i] <= 0.f ? 0.f : p[i];
        else if (act) p[i] *= sigmoid(p[i]);
    }
    return p;
}

// Zeros to the rows of tile [t0, t1) that are in no graph.
template <int L, bool BF>
__device__ __forceinline__ void zero_rest(const GroupArgs &a, int t0, int t1) {
    if (!a.ptr) return;
    const int before = min(offset_of(a, 0), t1), behind = max(offset_of(a, a.B), t0);
    for (int part = 0; part < 2; ++part) {
        const int from = part ? behind : t0, rows = (part ? t1 : before) - from;
        if (rows <= 0) continue;
        const __amdgpu_buffer_rsrc_t w = rows_of<BF>(a, a.out, from, rows);
        for (int chunk = 0; chunk < chunks_of(a); ++chunk) {
            const Columns<L, kWaves> c(a, chunk);
            for (int row = 0; row < rows; row += c.kRows)
                store_row_quad<BF, L == 1>(w, c.row(a, row, rows), row_f32x4{0.f, 0.f, 0.f, 0.f}, c.odd, false);
        }
    }
}

// ------------------------------------------------------------------ forward

template <int L, int W, bool X_BF, bool Y_BF>
struct Forward {
    static constexpr bool TINY = L == 1;
    using Cols = Columns<L, W>;

    // The sums of rows [first, first + rows) of a graph that starts at `start`.
    // shift: the thread's columns' groups' first elements.
    static __device__ __forceinline__ void sum(const GroupArgs &a, int start, int first, int rows, double (&s)[4], double (&q)[4], double (&shift)[4]) {
        const __amdgpu_buffer_rsrc_t w = rows_of<X_BF>(a, a.X, first, rows);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = q[i] = 0.0;
        for (int chunk = 0; chunk < chunks_of(a); ++chunk) {
            const Cols c(a, chunk);
#pragma unroll
            for (int i = 0; i < 4; ++i) shift[i] = shift_of<X_BF>(a, start, c.group[i]);
            for (int row = 0; row < rows; row += c.kRows * kAhead) {
                RawRowQuad<X_BF, TINY> in[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const QuadPlace at = c.row(a, row + k * c.kRows, rows);
                    in[k].load(w, at.at, at.count);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (row + k * c.kRows >= rows) break;                // uniform
                    const row_f32x4 x = in[k].get(c.at, c.odd);
                    const bool there = row + k * c.kRows + c.slot < rows;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // (columns behind the chunk's have no part in the sums of a thread's four)
                        const double d = there && c.first + i < c.end ? static_cast<double>(x[i]) - shift[i] : 0.0;
                        s[i] += d;
                        q[i] = fma(d, d, q[i]);
                    }
                }
            }
        }
    }
    // Y of rows [first, first + rows); stats(i): the statistics of the thread's column i of the chunk `c`.
    // `vectors`: the weights and biases of chunk 0.
    struct Vectors {
        row_f32x4 weight, bias;
        __device__ __forceinline__ Vectors(const GroupArgs &a, const Cols &c) : weight(c.vector(a.weight, 1.f)), bias(c.vector(a.bias, 0.f)) {}
    };
    template <class Stats>
    static __device__ __forceinline__ void apply(const GroupArgs &a, int first, int rows, const Vectors &vectors, Stats stats) {
        const __amdgpu_buffer_rsrc_t wx = rows_of<X_BF>(a, a.X, first, rows), wy = rows_of<Y_BF>(a, a.out, first, rows);
        for (int chunk = 0; chunk < chunks_of(a); ++chunk) {
            const Cols c(a, chunk);
            Vectors v = vectors;
            if (chunk) v = Vectors(a, c);
            Unit unit;
#pragma unroll
            for (int i = 0; i < 4; ++i) unit.set(i, stats(c, i));
            for (int row = 0; row < rows; row += c.kRows * kAhead) {
                RawRowQuad<X_BF, TINY> in[kAhead];
                QuadPlace at[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    at[k] = c.row(a, row + k * c.kRows, rows);
                    in[k].load(wx, at[k].at, at[k].count);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (row + k * c.kRows >= rows) break;                // uniform
                    store_row_quad<Y_BF, TINY>(wy, at[k], activated(unit(in[k].get(c.at, c.odd)) * v.weight + v.bias, a.act), c.odd, a.streaming);
                }
            }
        }
    }
};

template <int L, int W, bool X_BF, bool Y_BF>
__global__ __launch_bounds__(kThreads, 4) void group_kernel(GroupArgs a) {
    using K = Forward<L, W, X_BF, Y_BF>;
    constexpr int kTeams = kWaves / W;
    __shared__ union Memory {
        TeamMemory<L, W> graph[kTeams];
        TeamMemory<L, kWaves> tile;
        __device__ Memory() {}
    } sh;
    int turn = 0;
    if (static_cast<int>(blockIdx.x) < a.graph_groups) {
        const int team = threadIdx.x / (64 * W);
        const Columns<L, W> c(a, 0);
        const typename K::Vectors vectors(a, c);
        for (int b = blockIdx.x * kTeams + team; b < a.B; b += a.graph_groups * kTeams) {
            const int first = offset_of(a, b), rows = offset_of(a, b + 1) - first;
            if (rows > a.limit) continue;
            double2 *stats = a.stats + static_cast<int64_t>(b) * a.G;
            if (rows <= 0) {
                for (int g = c.c0 / a.D + threadIdx.x % (64 * W); g <= (c.end - 1) / a.D; g += 64 * W) stats[g] = make_double2(0.0, reciprocal_root(a.eps));
                continue;
            }
            double s[4], q[4], shift[4];
            K::sum(a, first, first, rows, s, q, shift);
            double2 v[4];
            group_sums(a, c, s, q, sh.graph[team], turn, v, [&](int g, double2 sums, bool mine) {
                const double from = a.lanes ? shift[0] : shift_of<X_BF>(a, first, g);
                const double2 st = statistics(sums, from, static_cast<double>(rows) * a.D, a.eps);
                if (mine) stats[g] = st;
                return st;
            });
            K::apply(a, first, rows, vectors, [&](const Columns<L, W> &, int i) { return v[i]; });
        }
        return;
    }
    const int t = static_cast<int>(blockIdx.x) - a.graph_groups, t0 = t * a.tile_rows, t1 = tile_end(a, t0);
    if (a.fill) zero_rest<L, Y_BF>(a, t0, t1);
    if (a.n <= a.limit) return;
    const Columns<L, kWaves> c(a, 0);
    long_pieces(a, t, t0, t1, true, [&](const Graph &g, int end, int from, int rows) {
        double s[4], q[4], shift[4];
        Forward<L, kWaves, X_BF, Y_BF>::sum(a, g.first, from, rows, s, q, shift);
        double2 v[4];
        group_sums(a, c, s, q, sh.tile, turn, v, [&](int j, double2 sums, bool mine) {
            if (mine) a.slots[(2 * static_cast<int64_t>(t) + end) * a.G + j] = sums;
            return sums;
        });
    });
}

constexpr int kJoinGroups = 8;                       // groups a workgroup joins, 32 threads each

// The long graph that starts in a tile, if there is one: f(graph, group, its sums over the tiles).
template <class Fn>
__device__ __forceinline__ void join_tile(const GroupArgs &a, int tile, int g0, Fn f) {
    constexpr int kLanes = kThreads / kJoinGroups;
    __shared__ double2 sh[kThreads];
    const int4 p = a.pieces[2 * tile + 1];
    const Graph graph{p.x, p.y, p.z};
    if (graph.number < 0 || graph.first < tile * a.tile_rows) return;
    const int j = threadIdx.x % kJoinGroups, k = threadIdx.x / kJoinGroups, g = g0 + j;
    const int to = (graph.first + graph.rows - 1) / a.tile_rows;
    const int last = a.pieces[2 * tile].x != graph.number;               // its place in this tile; in the others it has the first row
    double x = 0.0, y = 0.0;
    if (g < a.G)
#pragma unroll 4
        for (int t = tile + k; t <= to; t += kLanes) {
            const double2 v = a.slots[(2 * static_cast<int64_t>(t) + (t == tile ? last : 0)) * a.G + g];
            x += v.x;
            y += v.y;
        }
    sh[threadIdx.x] = make_double2(x, y);
    __syncthreads();
    for (int m = kLanes / 2; m > 0; m >>= 1) {
        if (k < m) {
            sh[threadIdx.x].x += sh[threadIdx.x + m * kJoinGroups].x;
            sh[threadIdx.x].y += sh[threadIdx.x + m * kJoinGroups].y;
        }
        __syncthreads();
    }
    if (k == 0 && g < a.G) f(graph, g, sh[threadIdx.x]);
}

template <bool X_BF>
__global__ __launch_bounds__(kThreads) void group_join_kernel(GroupArgs a) {
    join_tile(a, blockIdx.x, blockIdx.y * kJoinGroups, [&](const Graph &p, int g, double2 v) {
        a.stats[static_cast<int64_t>(p.number) * a.G + g] = statistics(v, shift_of<X_BF>(a, p.first, g), p.count(a), a.eps);
    });
}

template <int L, bool X_BF, bool Y_BF>
__global__ __launch_bounds__(kThreads) void group_apply_kernel(GroupArgs a) {
    // the tiles that were read last come first: they may still be in the memory-side cache
    using K = Forward<L, kWaves, X_BF, Y_BF>;
    const int tile = a.tiles - 1 - static_cast<int>(blockIdx.x), t0 = tile * a.tile_rows, t1 = tile_end(a, t0);
    const typename K::Vectors vectors(a, typename K::Cols(a, 0));
    long_pieces(a, tile, t0, t1, false, [&](const Graph &g, int, int from, int rows) {
        const double2 *stats = a.stats + static_cast<int64_t>(g.number) * a.G;
        K::apply(a, from, rows, vectors, [&](const Columns<L, kWaves> &c, int i) { return stats[c.group[i]]; });
    });
}

// ------------------------------------------------------------------ backward

template <int L, int W, bool X_BF, bool G_BF>
struct Backward {
    static constexpr bool TINY = L == 1;
    using Cols = Columns<L, W>;

    // f(place, d, u, x) for rows [first, first + rows) of graph `number` in chunk `chunk`, where d = dY act'(p).  Next to 0 it is the
    // sign of p in float64 that decides what a ReLU passes.
    // after() follows each AHEAD of a thread's rows.
    template <int AHEAD, class Fn, class After>
    static __device__ __forceinline__ void rows_do(const GroupArgs &a, const Cols &c, const Unit &unit, row_f32x4 weight, row_f32x4 bias, int number,
                                                   int first, int rows, Fn f, After after) {
        const __amdgpu_buffer_rsrc_t wx = rows_of<X_BF>(a, a.X, first, rows), wg = rows_of<G_BF>(a, a.dY, first, rows);
        for (int row = 0; row < rows; row += c.kRows * AHEAD) {
            RawRowQuad<X_BF, TINY> xs[AHEAD];
            RawRowQuad<G_BF, TINY> gs[AHEAD];
            QuadPlace at[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                at[k] = c.row(a, row + k * c.kRows, rows);
                xs[k].load(wx, at[k].at, at[k].count);
                gs[k].load(wg, at[k].at, at[k].count);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (row + k * c.kRows + c.slot >= rows) continue;
                const row_f32x4 x = xs[k].get(c.at, c.odd), u = unit(x);
                row_f32x4 g = gs[k].get(c.at, c.odd);
                if (a.act) {
                    const row_f32x4 uw = u * weight, p = uw + bias;
                    if (a.act == DUALGCN_RELU) {
                        bool near = false;
#pragma unroll
                        for (int i = 0; i < 4; ++i) near |= fabsf(p[i]) <= 0x1p-20f * (fabsf(uw[i]) + fabsf(bias[i]));
                        if (near) {
                            const double2 *st = a.stats + static_cast<int64_t>(number) * a.G;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                g[i] = (static_cast<double>(x[i]) - st[c.group[i]].x) * st[c.group[i]].y * weight[i] + bias[i] > 0.0 ? g[i] : 0.f;
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) g[i] = p[i] > 0.f ? g[i] : 0.f;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float s = sigmoid(p[i]);
                            g[i] *= s + p[i] * s * (1.f - s);
                        }
                    }
                }
                f(at[k], g, u, x);
                __builtin_amdgcn_sched_barrier(0);       // a row after the other: four at once take twice the registers
            }
            after();
        }
    }
    static __device__ __forceinline__ Unit unit_of(const GroupArgs &a, const Cols &c, int number) {
        Unit u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u.set(i, a.stats[static_cast<int64_t>(number) * a.G + c.group[i]]);
        return u;
    }
    // dX of rows [first, first + rows) of a graph; sums(c, i): those of t and t u of the group of the thread's column i.
    template <class Sums>
    static __device__ __forceinline__ void apply(const GroupArgs &a, const Graph &g, int first, int rows, Sums sums) {
        const __amdgpu_buffer_rsrc_t to = rows_of<G_BF>(a, a.out, first, rows);
        const double one = reciprocal(g.count(a));
        for (int chunk = 0; chunk < chunks_of(a); ++chunk) {
            const Cols c(a, chunk);
            const row_f32x4 weight = c.vector(a.weight, 1.f), bias = c.vector(a.bias, 0.f);
            const Unit unit = unit_of(a, c, g.number);
            row_f32x4 m1, m2;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double2 v = sums(c, i);
                m1[i] = static_cast<float>(v.x * one);
                m2[i] = static_cast<float>(v.y * one);
            }
            rows_do<kAheadBack>(a, c, unit, weight, bias, g.number, first, rows, [&](const QuadPlace &at, row_f32x4 d, row_f32x4 u, row_f32x4) {
                store_row_quad<G_BF, TINY>(to, at, unit.r * (0.5f * (d * weight - m1 - u * m2)), c.odd, a.streaming);
            }, [] {});
        }
    }
    // dX of a graph whose groups have kFew elements at most, and the columns' sums.  What is left of t - mean(t) - u mean(t u) there may be
    // next to nothing beside its terms (0 of one element, eps r^2 of two), and r up to 1 / sqrt(eps): u, the sums and the difference are
    // float64.  Both passes go by the same code, so that they have the same d and its roundings cancel as d does.
    static __device__ __forceinline__ void few(const GroupArgs &a, const Cols &c, const Graph &g, TeamMemory<L, W> &sh, int &turn,
                                               double (&d1)[4], double (&d2)[4]) {
        const __amdgpu_buffer_rsrc_t to = rows_of<G_BF>(a, a.out, g.first, g.rows);
        const row_f32x4 weight = c.vector(a.weight, 1.f), bias = c.vector(a.bias, 0.f);
        const double2 *stats = a.stats + static_cast<int64_t>(g.number) * a.G;
        double2 st[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            st[i] = stats[c.group[i]];
            v[i] = make_double2(0.0, 0.0);
            d1[i] = d2[i] = 0.0;
        }
        const Unit unit = unit_of(a, c, g.number);
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            rows_do<1>(a, c, unit, weight, bias, g.number, g.first, g.rows, [&](const QuadPlace &at, row_f32x4 d, row_f32x4, row_f32x4 x) {
                double u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = (static_cast<double>(x[i]) - st[i].x) * st[i].y;
                if (pass) {
                    row_f32x4 y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = static_cast<float>(st[i].y * (static_cast<double>(d[i]) * weight[i] - v[i].x - u[i] * v[i].y));
                    store_row_quad<G_BF, TINY>(to, at, y, c.odd, a.streaming);
                    return;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    d1[i] += d[i];
                    d2[i] = fma(d[i], u[i], d2[i]);
                }
            }, [] {});
            if (pass || !a.out) break;
            double t1[4], t2[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (c.first + i >= c.end) d1[i] = d2[i] = 0.0;           // columns behind the last
                t1[i] = d1[i] * weight[i];
                t2[i] = d2[i] * weight[i];
            }
            const double count = g.count(a);
            group_sums(a, c, t1, t2, sh, turn, v, [&](int, double2 sums, bool) { return make_double2(sums.x / count, sums.y / count); });
        }
    }
};

// The columns' sums of d u and d over a workgroup's rows.  They stay in registers over its graphs or its tile; where it has
// several chunks of columns they are added to its part of `columns` after each.
template <int L>
struct ColumnSums {
    double du[4], d[4];
    __device__ __forceinline__ ColumnSums(const GroupArgs &a) {
#pragma unroll
        for (int i = 0; i < 4; ++i) du[i] = d[i] = 0.0;
        if (!a.columns || !a.split) return;
        double *to = a.columns + static_cast<int64_t>(blockIdx.x) * 2 * a.F + static_cast<int64_t>(blockIdx.y) * a.D;
        for (int i = threadIdx.x; i < a.D; i += kThreads) to[i] = to[a.F + i] = 0.0;
        __syncthreads();
    }
    // By all threads of the workgroup, whose columns start at c0; `sh` holds kWaves * 4 L pairs.
    __device__ __forceinline__ void leave(const GroupArgs &a, int c0, int end, double2 *sh, bool more) {
        __syncthreads();
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            du[i] = over_rows<L>(du[i]);
            d[i] = over_rows<L>(d[i]);
            if (lane < L) sh[wave * 4 * L + 4 * lane + i] = make_double2(du[i], d[i]);
            du[i] = d[i] = 0.0;
        }
        __syncthreads();
        double *to = a.columns + static_cast<int64_t>(blockIdx.x) * 2 * a.F;
        for (int i = threadIdx.x; i < end - c0; i += kThreads) {
            double x = more ? to[c0 + i] : 0.0, y = more ? to[a.F + c0 + i] : 0.0;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) {
                x += sh[v * 4 * L + i].x;
                y += sh[v * 4 * L + i].y;
            }
            to[c0 + i] = x;
            to[a.F + c0 + i] = y;
        }
        __syncthreads();
    }
};

template <int L, int W, bool X_BF, bool G_BF>
__global__ __launch_bounds__(kThreads, 3) void group_back_kernel(GroupArgs a) {
    constexpr int kTeams = kWaves / W;
    __shared__ union Memory {
        TeamMemory<L, W> graph[kTeams];
        TeamMemory<L, kWaves> tile;
        __device__ Memory() {}
    } sh;
    double2 *const columns = sh.tile.buffer[0];      // the columns' sums take the same place, between barriers
    int turn = 0;
    ColumnSums<L> total(a);
    // The sums of t and t u of rows [first, first + rows) of a graph, and the columns' sums on the way.
    auto sum = [&](auto kind, int number, int first, int rows, double (&t1)[4], double (&t2)[4]) {
        using K = decltype(kind);
#pragma unroll
        for (int i = 0; i < 4; ++i) t1[i] = t2[i] = 0.0;
        for (int chunk = 0; chunk < chunks_of(a); ++chunk) {
            const typename K::Cols c(a, chunk);
            const row_f32x4 weight = c.vector(a.weight, 1.f), bias = c.vector(a.bias, 0.f);
            double d1[4] = {0.0, 0.0, 0.0, 0.0}, d2[4] = {0.0, 0.0, 0.0, 0.0};
            // float32 over kAheadBack rows, then float64
            const row_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            row_f32x4 s1 = zero, s2 = zero;
            K::template rows_do<kAheadBack>(a, c, K::unit_of(a, c, number), weight, bias, number, first, rows, [&](const QuadPlace &, row_f32x4 d, row_f32x4 u, row_f32x4) {
                s1 += d;
                s2 += d * u;
            }, [&] {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    d1[i] += s1[i];
                    d2[i] += s2[i];
                }
                s1 = s2 = zero;
            });
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (c.first + i >= c.end) d1[i] = d2[i] = 0.0;           // columns behind the chunk's
                total.d[i] += d1[i];
                total.du[i] += d2[i];
                t1[i] += d1[i] * weight[i];
                t2[i] += d2[i] * weight[i];
            }
            if (a.split && a.columns) total.leave(a, c.c0, c.end, columns, true);
        }
    };
    if (static_cast<int>(blockIdx.x) < a.graph_groups) {
        using K = Backward<L, W, X_BF, G_BF>;
        const int team = threadIdx.x / (64 * W);
        const Columns<L, W> c(a, 0);
        for (int b = blockIdx.x * kTeams + team; b < a.B; b += a.graph_groups * kTeams) {
            const int first = offset_of(a, b), rows = offset_of(a, b + 1) - first;
            if (rows > a.limit || rows <= 0) continue;
            if (rows <= kFew / a.D) {
                double d1[4], d2[4];
                K::few(a, c, Graph{b, first, rows}, sh.graph[team], turn, d1, d2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    total.d[i] += d1[i];
                    total.du[i] += d2[i];
                }
                continue;
            }
            double t1[4], t2[4];
            sum(K(), b, first, rows, t1, t2);
            if (!a.out) continue;
            double2 v[4];
            group_sums(a, c, t1, t2, sh.graph[team], turn, v, [&](int, double2 sums, bool) { return sums; });
            K::apply(a, Graph{b, first, rows}, first, rows, [&](const Columns<L, W> &, int i) { return v[i]; });
        }
    } else {
        using K = Backward<L, kWaves, X_BF, G_BF>;
        const Columns<L, kWaves> c(a, 0);
        const int t = static_cast<int>(blockIdx.x) - a.graph_groups, t0 = t * a.tile_rows, t1 = tile_end(a, t0);
        if (a.fill && a.out) zero_rest<L, G_BF>(a, t0, t1);
        if (a.n > a.limit)
            long_pieces(a, t, t0, t1, true, [&](const Graph &g, int end, int from, int rows) {
                double s1[4], s2[4];
                sum(K(), g.number, from, rows, s1, s2);
                if (!a.out) return;
                double2 v[4];
                group_sums(a, c, s1, s2, sh.tile, turn, v, [&](int j, double2 sums, bool mine) {
                    if (mine) a.slots[(2 * static_cast<int64_t>(t) + end) * a.G + j] = sums;
                    return sums;
                });
            });
    }
    if (a.columns && !a.split) {
        const Columns<L, kWaves> c(a, 0);
        total.leave(a, c.c0, c.end, columns, false);
    }
}

// Workgroups up to `joins` in x join long graphs' sums, the others columns' sums, 16 of the 2 F each.
constexpr int kJoinColumns = 16;
__global__ __launch_bounds__(kThreads) void group_back_join_kernel(GroupArgs a, int32_t joins) {
    if (static_cast<int>(blockIdx.x) < joins) {
        const int parts = (a.G + kJoinGroups - 1) / kJoinGroups, tile = blockIdx.x / parts;
        join_tile(a, tile, static_cast<int>(blockIdx.x) % parts * kJoinGroups,
                  [&](const Graph &, int g, double2 v) { a.joined[static_cast<int64_t>(tile) * a.G + g] = v; });
        return;
    }
    constexpr int kLanes = kThreads / kJoinColumns;
    __shared__ double sh[kThreads];
    const int64_t i = static_cast<int64_t>(blockIdx.x - joins) * kJoinColumns + threadIdx.x % kJoinColumns;
    const int k = threadIdx.x / kJoinColumns;
    double s = 0.0;
    if (i < 2 * static_cast<int64_t>(a.F))
#pragma unroll 8
        for (int t = k; t < a.workgroups; t += kLanes) s += a.columns[static_cast<int64_t>(t) * 2 * a.F + i];
    sh[threadIdx.x] = s;
    __syncthreads();
    for (int m = kLanes / 2; m > 0; m >>= 1) {
        if (k < m) sh[threadIdx.x] += sh[threadIdx.x + m * kJoinColumns];
        __syncthreads();
    }
    if (k == 0 && i < 2 * static_cast<int64_t>(a.F)) {
        float *to = i < a.F ? a.dweight : a.dbias;
        if (to) to[i < a.F ? i : i - a.F] = static_cast<float>(sh[threadIdx.x]);
    }
}

template <int L, bool X_BF, bool G_BF>
__global__ __launch_bounds__(kThreads) void group_back_apply_kernel(GroupArgs a) {
    const int tile = a.tiles - 1 - static_cast<int>(blockIdx.x), t0 = tile * a.tile_rows, t1 = tile_end(a, t0);
    long_pieces(a, tile, t0, t1, false, [&](const Graph &g, int, int from, int rows) {
        const double2 *sums = a.joined + static_cast<int64_t>(g.first / a.tile_rows) * a.G;
        Backward<L, kWaves, X_BF, G_BF>::apply(a, g, from, rows, [&](const Columns<L, kWaves> &c, int i) { return sums[c.group[i]]; });
    });
}

// ------------------------------------------------------------------ launches

// A wavefront is a team where there are many graphs, of rows that it takes in so many turns on the average.  Calls in us, forward and
// backward, by wavefronts and by workgroups: graphs of about 30 rows of 64 features, 1,024 of them 16.2, 34.7 and 15.5, 31.8; 2,048
// 18.8, 54.5 and 24.2, 48.4; 4,096 24.8, 94.5 and 37.0, 69.7; 8,192 39.6, 79.9 and 62.9, 114; of 128 features, 1,024 24.5, 53.4 and 18.7, 40.8;
// 2,048 29.1, 90.9 and 26.5, 60.4; 4,096 40.4, 79.0 and 41.5, 93.1; 8,192 72.3, 140 and 73.9, 186; 65,536 471, 835 and 599, 1,153.  (23 rows of 64
// by one wavefront 7.9, by a workgroup 6.1.)
constexpr int kWaveTurns = 16;
constexpr int kWaveGraphs = 2048;
// A team's turns, at least, for a graph that is not long, forward and backward: about what the two more launches for long ones take (calls
// with half as many, these and twice as many, graphs cut at random: 4,096 of 30 rows of 128 features forward 60.2, 48.1, 64.9 us; of 100 rows on
// the average, 300 of 128 25.1, 34.0, 46.2 and backward 39.1, 33.8, 39.5; 1,000 of 128 40.1, 46.5, 64.5 and 89.5, 73.4, 71.2; 4,000 of 64
// 66.8, 87.4, 74.6 and 164, 153, 141).  No graph of fewer rows than a tile is long, however: where there would be more than
// 4 * 1,024 tiles of so many turns, a tile has a 1,024th of the rows, and a team's graph may have as many.  One that is much longer than
// the others then ends the launch by itself: among 65,536 graphs of 32 rows of 128 on the average, where tiles have 2,048 rows, one of 1,937 makes 985 us of 471
// forward and 1,575 of 835 backward (by workgroups 742 of 599 and 1,329 of 1,153); among 300,000 of 56 rows of 64 one of 16,057 rows 4,050 us of
// 1,794 and 6,035 of 3,148.
constexpr int kLimitTurns = 32, kLimitTurnsBack = 8;

int lanes_of(int32_t width) { return width < 4 ? 1 : width <= 32 ? 8 : width <= 64 ? 16 : width <= 128 ? 32 : 64; }

// Tiles, and workgroups over graphs: many enough to fill the chip, few enough that their column sums stay small beside the rows.
constexpr int kMostTiles = 1024;
struct Shape {
    int32_t tile_rows, tiles, limit, width, sets, graph_groups, workgroups, team;
    bool split;
    Shape(int32_t n, int32_t B, int32_t F, int32_t groups, bool back) {
        const int32_t D = F / groups;
        split = D > kSlice;
        width = split ? kSlice : std::min(F, kSlice / D * D);
        sets = split ? groups : (F + width - 1) / width;
        const int64_t lanes = lanes_of(width), side = kThreads / lanes, turn = side * kAheadBack, chunks = split ? (D + kSlice - 1) / kSlice : 1;
        const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kMostTiles / sets, (int64_t{1} << 22) / F));
        team = !split && B >= kWaveGraphs && n / B * lanes <= 64 * kWaveTurns ? 1 : kWaves;
        const int64_t at_once = std::max<int64_t>(1, (back ? kLimitTurnsBack : kLimitTurns) * 64 * team / lanes / chunks);
        const int64_t least = back ? 2 * turn : turn;
        int64_t rows = ((n + most - 1) / most + least - 1) / least * least;
        if (rows > at_once && n / at_once <= 4 * most) rows = at_once;       // rather more tiles than long turns
        rows = std::min(rows, std::max<int64_t>(1, (int64_t{1} << 26) / F / turn) * turn);       // 32-bit offsets
        tile_rows = static_cast<int32_t>(rows);
        tiles = static_cast<int32_t>((n + rows - 1) / rows);
        // (a graph of kFew elements is not long)
        limit = static_cast<int32_t>(std::max<int64_t>({rows, at_once, back ? kFew / D : 0}));
        const int32_t teams = kWaves / team;
        graph_groups = static_cast<int32_t>(std::min<int64_t>(2 * most, (B - 1) / teams + 1));
        workgroups = graph_groups + tiles;
    }
};

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t slot_bytes(const Shape &s, int32_t n, int32_t G) {
    return n <= s.limit ? 0 : up(sizeof(double2) * 2 * static_cast<size_t>(s.tiles) * G) + up(sizeof(int4) * 2 * static_cast<size_t>(s.tiles));
}
size_t joined_bytes(const Shape &s, int32_t n, int32_t G) { return n <= s.limit ? 0 : up(sizeof(double2) * static_cast<size_t>(s.tiles) * G); }
size_t column_bytes(const Shape &s, int32_t F) { return up(sizeof(double) * 2 * static_cast<size_t>(s.workgroups) * F); }

template <template <int, bool, bool> class Launch>
int by_type(const GroupArgs &a, const Shape &shape, bool x_bf, bool y_bf, hipStream_t s) {
#define DGC_GROUP_TYPES(L)                                                                                      \
    return x_bf ? (y_bf ? Launch<L, true, true>::go(a, shape, s) : Launch<L, true, false>::go(a, shape, s))     \
                : (y_bf ? Launch<L, false, true>::go(a, shape, s) : Launch<L, false, false>::go(a, shape, s))
    switch (lanes_of(a.width)) {
        case 1: DGC_GROUP_TYPES(1);
        case 8: DGC_GROUP_TYPES(8);
        case 16: DGC_GROUP_TYPES(16);
        case 32: DGC_GROUP_TYPES(32);
        default: DGC_GROUP_TYPES(64);
    }
#undef DGC_GROUP_TYPES
}

// (tiles have nothing to do where no graph can be long and no row's to be filled)
int32_t first_groups(const GroupArgs &a) { return a.n > a.limit || (a.fill && a.ptr) ? a.workgroups : a.graph_groups; }

template <int L, bool X_BF, bool Y_BF>
struct ForwardLaunch {
    static int go(const GroupArgs &a, const Shape &shape, hipStream_t s) {
        const dim3 block(kThreads), grid(first_groups(a), shape.sets);
        if (shape.team == 1) hipLaunchKernelGGL((group_kernel<L, 1, X_BF, Y_BF>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((group_kernel<L, kWaves, X_BF, Y_BF>), grid, block, 0, s, a);
        if (a.n > a.limit) {
            hipLaunchKernelGGL((group_join_kernel<X_BF>), dim3(a.tiles, (a.G + kJoinGroups - 1) / kJoinGroups), block, 0, s, a);
            hipLaunchKernelGGL((group_apply_kernel<L, X_BF, Y_BF>), dim3(a.tiles, shape.sets), block, 0, s, a);
        }
        return hip_status(hipGetLastError());
    }
};

template <int L, bool X_BF, bool G_BF>
struct BackwardLaunch {
    static int go(GroupArgs a, const Shape &shape, hipStream_t s) {
        a.workgroups = first_groups(a);
        const dim3 block(kThreads), grid(a.workgroups, shape.sets);
        if (shape.team == 1) hipLaunchKernelGGL((group_back_kernel<L, 1, X_BF, G_BF>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((group_back_kernel<L, kWaves, X_BF, G_BF>), grid, block, 0, s, a);
        const bool more = a.out && a.n > a.limit;
        const int32_t joins = more ? a.tiles * ((a.G + kJoinGroups - 1) / kJoinGroups) : 0;
        const int32_t sums = a.columns ? (2 * a.F + kJoinColumns - 1) / kJoinColumns : 0;
        if (joins + sums) hipLaunchKernelGGL(group_back_join_kernel, dim3(joins + sums), block, 0, s, a, joins);
        if (more) hipLaunchKernelGGL((group_back_apply_kernel<L, X_BF, G_BF>), dim3(a.tiles, shape.sets), block, 0, s, a);
        return hip_status(hipGetLastError());
    }
};

int32_t graphs_of(const dualgcn_group_norm &p) { return p.ptr ? p.graphs : 1; }
Shape shape_of(const dualgcn_group_norm &p, int32_t n, bool back) { return Shape(n, graphs_of(p), p.F, p.groups, back); }

GroupArgs common(const dualgcn_group_norm &p, const void *X, int32_t n, const Shape &s, void *workspace) {
    GroupArgs a{};
    a.X = X;
    a.ptr = p.ptr;
    a.weight = p.weight;
    a.bias = p.bias;
    a.eps = p.eps;
    a.n = n;
    a.B = graphs_of(p);
    a.F = p.F;
    a.G = p.groups;
    a.D = p.F / p.groups;
    a.tile_rows = s.tile_rows;
    a.tiles = s.tiles;
    a.limit = s.limit;
    a.width = s.width;
    a.graph_groups = s.graph_groups;
    a.workgroups = s.workgroups;
    const int32_t quads = a.D % 4 ? 0 : a.D / 4;
    a.lanes = s.split ? 64 : quads & (quads - 1) ? 0 : quads;
    a.split = s.split;
    a.act = static_cast<int32_t>(p.flags & (DUALGCN_RELU | DUALGCN_SILU));
    a.fill = p.flags & DUALGCN_ZERO_REST;
    a.streaming = static_cast<int64_t>(n) * p.F >= int64_t{1} << 26;
    a.slots = static_cast<double2 *>(workspace);
    a.pieces = reinterpret_cast<int4 *>(static_cast<char *>(workspace) + up(sizeof(double2) * 2 * static_cast<size_t>(s.tiles) * a.G));
    return a;
}

}  // namespace

size_t group_norm_workspace_bytes(const dualgcn_group_norm &p, int32_t n) { return slot_bytes(shape_of(p, n, false), n, p.groups); }

size_t group_norm_backward_workspace_bytes(const dualgcn_group_norm &p, int32_t n) {
    const Shape s = shape_of(p, n, true);
    return slot_bytes(s, n, p.groups) + joined_bytes(s, n, p.groups) + column_bytes(s, p.F);
}

int launch_group_norm(const dualgcn_group_norm &p, const void *X, void *Y, double *stats, int32_t n, void *workspace,
                      hipStream_t s) {
    const Shape shape = shape_of(p, n, false);
    GroupArgs a = common(p, X, n, shape, workspace);
    a.out = Y;
    a.stats = reinterpret_cast<double2 *>(stats);
    return by_type<ForwardLaunch>(a, shape, p.flags & DUALGCN_IN_BF16, p.flags & DUALGCN_OUT_BF16, s);
}

int launch_group_norm_backward(const dualgcn_group_norm &p, const void *X, const void *dY, const double *stats, void *dX,
                               float *dweight, float *dbias, int32_t n, void *workspace, hipStream_t s) {
    const Shape shape = shape_of(p, n, true);
    GroupArgs a = common(p, X, n, shape, workspace);
    a.dY = dY;
    a.out = dX;
    a.stats = reinterpret_cast<double2 *>(const_cast<double *>(stats));
    char *more = static_cast<char *>(workspace) + slot_bytes(shape, n, a.G);
    a.joined = reinterpret_cast<double2 *>(more);
    more += joined_bytes(shape, n, a.G);
    a.columns = dweight || dbias ? reinterpret_cast<double *>(more) : nullptr;
    a.dweight = dweight;
    a.dbias = dbias;
    return by_type<BackwardLaunch>(a, shape, p.flags & DUALGCN_IN_BF16, p.flags & DUALGCN_GRAD_BF16, s);
}

}  // namespace dgc
