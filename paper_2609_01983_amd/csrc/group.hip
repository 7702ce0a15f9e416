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
// A workgroup has a tile of consecutive rows and up to 256 columns (a slice: whole groups, where they are no
// wider), and takes the pieces of graphs that lie in it one after the other.  A graph inside one tile is finished
// there: its rows are read a second time by the compute unit that has just read them.  One that crosses tiles
// leaves partial sums for each tile and slice, which a second launch joins and a third applies; only a tile's
// first and last graphs can be such, so neither launch looks at the others.  (Where a group goes over slices, no
// graph is finished at once.)  The graphs' offsets are read on the device: the host knows neither their lengths
// nor whether any graph crosses a tile.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSlice = 256;                          // columns of a workgroup, at most
constexpr int kAhead = 4;                            // rows a thread has in flight

struct GroupArgs {
    const void *X, *dY;
    const int32_t *ptr;
    const float *weight, *bias;
    void *out;                                       // Y, or dX
    double2 *stats;                                  // [B][G]: mean, r
    double2 *slots;                                  // [tiles + B][slices + G] partial sums of crossing graphs
    double2 *joined;                                 // backward: [tiles][G] the sums of the graph that starts in a tile
    double *columns;                                 // backward: [tiles][2][F] sums of d u and d
    float *dweight, *dbias;
    double eps;
    int32_t n, B, F, G, D;
    int32_t tile_rows, tiles, slices, width;         // width: columns of a slice, whole groups if D <= kSlice
    int32_t act;                                     // 0, DUALGCN_RELU or DUALGCN_SILU
    bool fill;                                       // rows of no graph receive zeros
    bool split;                                      // groups go over slices
};

// The rows of graph b, within [0, n] whatever the offsets hold.
__device__ __forceinline__ int32_t graph_end(const GroupArgs &a, int b) { return a.ptr ? min(max(a.ptr[b], 0), a.n) : b ? a.n : 0; }

// How many of the B + 1 offsets are at or below `row` (the same in every lane): the row is in graph
// count - 1, before the first (0) or behind the last (B + 1).  64 places a step.
__device__ __forceinline__ int offsets_up_to(const GroupArgs &a, int row) {
    if (!a.ptr) return row < a.n ? 1 : 2;
    const int lane = threadIdx.x & 63, end = a.B + 1;
    int lo = 0, len = end;
    while (len > 0) {
        const int step = (len + 63) / 64, at = lo + (lane + 1) * step - 1;
        const int k = __popcll(__ballot(at < lo + len && a.ptr[min(at, end - 1)] <= row));
        const int was = lo + len;
        lo = min(lo + k * step, was);
        len = min(step - 1, was - lo);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// A run of rows [lo, hi) of one graph (or of none: graph < 0) inside a tile [t0, t1), and whether the graph
// goes past the tile.
struct Piece {
    int lo, hi, graph, first, last;                  // first, last: the whole graph's rows
    bool crosses;
};
__device__ __forceinline__ Piece piece_at(const GroupArgs &a, int row, int t0, int t1) {
    const int c = offsets_up_to(a, row);
    Piece p;
    p.lo = row;
    if (c == 0 || c > a.B) {
        p.graph = -1;
        p.first = row;
        p.last = c ? a.n : max(graph_end(a, 0), row + 1);
    } else {
        p.graph = c - 1;
        p.first = min(graph_end(a, c - 1), row);
        p.last = max(graph_end(a, c), row + 1);
    }
    p.hi = min(p.last, t1);
    p.crosses = p.first < t0 || p.last > t1;
    return p;
}

__device__ __forceinline__ double count_of(const GroupArgs &a, const Piece &p) {
    return static_cast<double>(p.last - p.first) * a.D;
}

// A thread's four columns: their groups, weights, and the row it starts with.
template <int L, bool TINY>
struct Columns {
    static constexpr int kRows = kThreads / L;       // rows side by side
    int c0, end, first, slot;                        // the slice's first column and its end, the thread's first, its row
    QuadPlace at;                                    // of the slot's row in the tile's window
    int group[4];
    bool odd;
    __device__ __forceinline__ Columns(const GroupArgs &a) {
        c0 = blockIdx.y * a.width;
        end = min(a.F, c0 + a.width);
        first = c0 + 4 * (threadIdx.x % L);
        slot = threadIdx.x / L;
        odd = (end - c0) & 3;
        at.set(static_cast<uint32_t>(slot) * a.F, first, end);
#pragma unroll
        for (int i = 0; i < 4; ++i) group[i] = min(first + i, a.F - 1) / a.D;
    }
    __device__ __forceinline__ row_f32x4 vector(const GroupArgs &a, const float *v, float otherwise) const {
        if (v) return load_quad<false>(v, first, a.F - first);
        return row_f32x4{otherwise, otherwise, otherwise, otherwise};
    }
};

// The place of a row of the tile, `row` rows behind the slot's own.
__device__ __forceinline__ QuadPlace moved(const QuadPlace &p, uint32_t rows, int F, bool valid) {
    QuadPlace q = p;
    if (!valid) {
        q.at = kNoQuad;
        q.count = q.part = 0;
    } else if (p.at != kNoQuad) {
        q.at = p.at + rows * F;
    }
    return q;
}

// Two sums of each thread's four columns over the rows side by side, and over the groups: f(j, sums) is
// called by one thread for each group that has columns in the slice, j its place among the slices' segments
// (slice + group) and the group's number.  `sh`: two buffers of kWaves * 4 L pairs, taken in turn.
template <int L>
constexpr int buffer_pairs() { return kWaves * 4 * L; }

template <int L, class Fn>
__device__ __forceinline__ void group_sums(const GroupArgs &a, int c0, int end, double (&s)[4], double (&q)[4], double2 *sh, int &turn, Fn f) {
#pragma unroll
    for (int m = L; m < 64; m <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] += __shfl_xor(s[i], m);
            q[i] += __shfl_xor(q[i], m);
        }
    double2 *b = sh + (turn & 1) * buffer_pairs<L>();
    ++turn;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane < L)
#pragma unroll
        for (int i = 0; i < 4; ++i) b[wave * 4 * L + 4 * lane + i] = make_double2(s[i], q[i]);
    __syncthreads();
    const int g0 = c0 / a.D, groups = (end - 1) / a.D - g0 + 1;
    int lanes = 64;                                  // of a group
    while (lanes * groups > kThreads) lanes >>= 1;
    const int j = threadIdx.x / lanes, k = threadIdx.x % lanes;
    double x = 0.0, y = 0.0;
    if (j < groups) {
        const int lo = max((g0 + j) * a.D, c0), hi = min((g0 + j + 1) * a.D, end);
        for (int c = lo + k; c < hi; c += lanes)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const double2 v = b[w * 4 * L + c - c0];
                x += v.x;
                y += v.y;
            }
    }
    for (int m = 1; m < lanes; m <<= 1) {
        x += __shfl_xor(x, m);
        y += __shfl_xor(y, m);
    }
    if (j < groups && k == 0) f(g0 + j, make_double2(x, y));
}

// The mean and r from sums of x - shift and its square.
__device__ __forceinline__ double2 statistics(double2 sums, double shift, double count, double eps) {
    const double d = sums.x / count, v = sums.y / count - d * d;
    return make_double2(shift + d, 1.0 / sqrt((v > 0.0 ? v : v != v ? v : 0.0) + eps));
}

template <bool BF>
__device__ __forceinline__ double shift_of(const GroupArgs &a, int first, int group) {
    const int64_t at = static_cast<int64_t>(first) * a.F + static_cast<int64_t>(group) * a.D;
    return BF ? bf16_to_float(static_cast<const unsigned short *>(a.X)[at]) : static_cast<const float *>(a.X)[at];
}

// m of two float32 numbers, r, and with them u; for a thread's four columns of one graph.
struct Unit {
    row_f32x4 hi, lo, r;
    __device__ __forceinline__ void set(int i, double2 st) {
        hi[i] = static_cast<float>(st.x);
        lo[i] = static_cast<float>(st.x - hi[i]);
        if (!(fabsf(hi[i]) < INFINITY)) lo[i] = 0.f;
        r[i] = static_cast<float>(st.y);
    }
    __device__ __forceinline__ row_f32x4 operator()(row_f32x4 x) const { return ((x - hi) - lo) * r; }
};

__device__ __forceinline__ float sigmoid(float v) { return 1.f / (1.f + expf(-v)); }

// act(p) (NaN stays NaN), and its derivative
__device__ __forceinline__ row_f32x4 activated(row_f32x4 p, int act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (act == DUALGCN_RELU) p[i] = p[i] <= 0.f ? 0.f : p[i];
        else if (act) p[i] = p[i] / (1.f + expf(-p[i]));
    }
    return p;
}

// ------------------------------------------------------------------ forward

template <int L, bool X_BF, bool Y_BF>
struct Forward {
    static constexpr bool TINY = L == 1;
    using Cols = Columns<L, TINY>;

    // Y of a piece's rows
    static __device__ __forceinline__ void apply(const GroupArgs &a, const Cols &c, const Piece &p, int t0, int t1,
                                                 const Unit &unit, row_f32x4 w, row_f32x4 b) {
        const __amdgpu_buffer_rsrc_t wx = row_window<X_BF>(a.X, static_cast<int64_t>(t0) * a.F, static_cast<int64_t>(t1 - t0) * a.F);
        const __amdgpu_buffer_rsrc_t wy = row_window<Y_BF>(a.out, static_cast<int64_t>(t0) * a.F, static_cast<int64_t>(t1 - t0) * a.F);
        for (int row = p.lo; row < p.hi; row += Cols::kRows * kAhead) {
            RawRowQuad<X_BF, TINY> in[kAhead];
            QuadPlace at[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int r = row + k * Cols::kRows;
                at[k] = moved(c.at, r - t0, a.F, r + c.slot < p.hi);
                in[k].load(wx, at[k].at, at[k].count);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const row_f32x4 x = in[k].get(at[k], c.odd);
                store_row_quad<Y_BF, TINY>(wy, at[k], activated(unit(x) * w + b, a.act), c.odd, false);
            }
        }
    }
    static __device__ __forceinline__ void zero(const GroupArgs &a, const Cols &c, const Piece &p, int t0, int t1) {
        const __amdgpu_buffer_rsrc_t wy = row_window<Y_BF>(a.out, static_cast<int64_t>(t0) * a.F, static_cast<int64_t>(t1 - t0) * a.F);
        for (int row = p.lo; row < p.hi; row += Cols::kRows)
            store_row_quad<Y_BF, TINY>(wy, moved(c.at, row - t0, a.F, row + c.slot < p.hi), row_f32x4{0.f, 0.f, 0.f, 0.f}, c.odd, false);
    }
};

template <int L, bool X_BF, bool Y_BF>
__global__ __launch_bounds__(kThreads) void group_kernel(GroupArgs a) {
    using F = Forward<L, X_BF, Y_BF>;
    __shared__ double2 sh[2 * buffer_pairs<L>()];
    __shared__ double2 held[kSlice];                 // the statistics of a finished graph's groups
    int turn = 0;
    const typename F::Cols c(a);
    const int t0 = blockIdx.x * a.tile_rows, t1 = min(a.n, t0 + a.tile_rows);
    const row_f32x4 w = c.vector(a, a.weight, 1.f), b = c.vector(a, a.bias, 0.f);
    const int g0 = c.c0 / a.D;
    // graphs without rows
    if (a.ptr && blockIdx.y == 0)
        for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.B; i += gridDim.x * kThreads)
            if (graph_end(a, i) >= graph_end(a, i + 1))
                for (int g = 0; g < a.G; ++g) a.stats[static_cast<int64_t>(i) * a.G + g] = make_double2(0.0, 1.0 / sqrt(a.eps));
    const __amdgpu_buffer_rsrc_t wx = row_window<X_BF>(a.X, static_cast<int64_t>(t0) * a.F, static_cast<int64_t>(t1 - t0) * a.F);
    for (int row = t0; row < t1;) {
        const Piece p = piece_at(a, row, t0, t1);
        row = p.hi;
        if (p.graph < 0) {
            if (a.fill) F::zero(a, c, p, t0, t1);
            continue;
        }
        double shift[4], s[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            shift[i] = shift_of<X_BF>(a, p.first, c.group[i]);
            s[i] = q[i] = 0.0;
        }
        for (int r0 = p.lo; r0 < p.hi; r0 += F::Cols::kRows * kAhead) {
            RawRowQuad<X_BF, F::TINY> in[kAhead];
            QuadPlace at[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int r = r0 + k * F::Cols::kRows;
                at[k] = moved(c.at, r - t0, a.F, r + c.slot < p.hi);
                in[k].load(wx, at[k].at, at[k].count);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (r0 + k * F::Cols::kRows + c.slot >= p.hi) continue;
                const row_f32x4 x = in[k].get(at[k], c.odd);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double d = static_cast<double>(x[i]) - shift[i];
                    s[i] += d;
                    q[i] = fma(d, d, q[i]);
                }
            }
        }
        const bool whole = !p.crosses && !a.split;
        group_sums<L>(a, c.c0, c.end, s, q, sh, turn, [&](int g, double2 v) {
            if (whole) {
                const double2 st = statistics(v, shift_of<X_BF>(a, p.first, g), count_of(a, p), a.eps);
                a.stats[static_cast<int64_t>(p.graph) * a.G + g] = st;
                held[g - g0] = st;
            } else {
                a.slots[(static_cast<int64_t>(blockIdx.x) + p.graph) * (a.slices + a.G) + blockIdx.y + g] = v;
            }
        });
        if (whole) {
            __syncthreads();
            Unit unit;
#pragma unroll
            for (int i = 0; i < 4; ++i) unit.set(i, held[c.group[i] - g0]);
            F::apply(a, c, p, t0, t1, unit, w, b);
        }
    }
}

// The graph that starts in a tile and goes past it, if there is one.
__device__ __forceinline__ bool crossing_from(const GroupArgs &a, int tile, Piece &p) {
    const int t0 = tile * a.tile_rows, t1 = min(a.n, t0 + a.tile_rows);
    p = piece_at(a, t1 - 1, t0, t1);
    return p.graph >= 0 && p.first >= t0 && p.last > t1;
}

constexpr int kJoinGroups = 8;                       // groups a workgroup joins, 32 threads each

// f(group, sums of the graph)
template <class Fn>
__device__ __forceinline__ void join(const GroupArgs &a, const Piece &p, int g0, Fn f) {
    constexpr int kLanes = kThreads / kJoinGroups;
    __shared__ double2 sh[kThreads];
    const int j = threadIdx.x % kJoinGroups, k = threadIdx.x / kJoinGroups, g = g0 + j;
    const int from = p.first / a.tile_rows, to = (p.last - 1) / a.tile_rows;
    double x = 0.0, y = 0.0;
    if (g < a.G) {
        const int s0 = g * a.D / a.width, s1 = ((g + 1) * a.D - 1) / a.width;
        for (int s = s0; s <= s1; ++s)
#pragma unroll 4
            for (int t = from + k; t <= to; t += kLanes) {
                const double2 v = a.slots[(static_cast<int64_t>(t) + p.graph) * (a.slices + a.G) + s + g];
                x += v.x;
                y += v.y;
            }
    }
    __syncthreads();
    sh[threadIdx.x] = make_double2(x, y);
    __syncthreads();
    for (int m = kLanes / 2; m > 0; m >>= 1) {
        if (k < m) {
            sh[threadIdx.x].x += sh[threadIdx.x + m * kJoinGroups].x;
            sh[threadIdx.x].y += sh[threadIdx.x + m * kJoinGroups].y;
        }
        __syncthreads();
    }
    if (k == 0 && g < a.G) f(g, sh[threadIdx.x]);
}

// The one crossing graph that starts in a tile; with groups that go over slices, every graph that starts in it.
template <class Fn>
__device__ __forceinline__ void join_tile(const GroupArgs &a, int tile, int g0, Fn f) {
    const int t0 = tile * a.tile_rows, t1 = min(a.n, t0 + a.tile_rows);
    if (!a.split) {
        Piece p;
        if (crossing_from(a, tile, p)) join(a, p, g0, [&](int g, double2 v) { f(p, g, v); });
        return;
    }
    for (int row = t0; row < t1;) {
        const Piece p = piece_at(a, row, t0, t1);
        row = p.hi;
        if (p.graph >= 0 && p.first >= t0) join(a, p, g0, [&](int g, double2 v) { f(p, g, v); });
    }
}

template <bool X_BF>
__global__ __launch_bounds__(kThreads) void group_join_kernel(GroupArgs a) {
    join_tile(a, blockIdx.x, blockIdx.y * kJoinGroups, [&](const Piece &p, int g, double2 v) {
        a.stats[static_cast<int64_t>(p.graph) * a.G + g] = statistics(v, shift_of<X_BF>(a, p.first, g), count_of(a, p), a.eps);
    });
}

// Calls f for the pieces of a tile that are not finished: the first and the last if they cross, or all.
template <class Fn>
__device__ __forceinline__ void unfinished(const GroupArgs &a, int t0, int t1, Fn f) {
    for (int row = t0; row < t1;) {
        const Piece p = piece_at(a, row, t0, t1);
        if (p.graph >= 0 && (p.crosses || a.split)) f(p);
        // the next piece; behind a finished one, the last of the tile
        row = a.split || p.hi == t1 ? p.hi : max(p.hi, piece_at(a, t1 - 1, t0, t1).first);
    }
}

template <int L, bool X_BF, bool Y_BF>
__global__ __launch_bounds__(kThreads) void group_apply_kernel(GroupArgs a) {
    using F = Forward<L, X_BF, Y_BF>;
    const typename F::Cols c(a);
    // the tiles that were read last come first: they may still be in the memory-side cache
    const int tile = a.tiles - 1 - static_cast<int>(blockIdx.x);
    const int t0 = tile * a.tile_rows, t1 = min(a.n, t0 + a.tile_rows);
    const row_f32x4 w = c.vector(a, a.weight, 1.f), b = c.vector(a, a.bias, 0.f);
    unfinished(a, t0, t1, [&](const Piece &p) {
        Unit unit;
#pragma unroll
        for (int i = 0; i < 4; ++i) unit.set(i, a.stats[static_cast<int64_t>(p.graph) * a.G + c.group[i]]);
        F::apply(a, c, p, t0, t1, unit, w, b);
    });
}

// ------------------------------------------------------------------ backward

template <int L, bool X_BF, bool G_BF>
struct Backward {
    static constexpr bool TINY = L == 1;
    using Cols = Columns<L, TINY>;

    // d of four elements: dY act'(p).  Next to 0 it is the sign of p in float64 that decides what a ReLU passes.
    static __device__ __forceinline__ row_f32x4 inner(const GroupArgs &a, row_f32x4 g, row_f32x4 x, row_f32x4 u, row_f32x4 w,
                                                      row_f32x4 b, const double2 *stats, const int (&group)[4]) {
        if (!a.act) return g;
        const row_f32x4 uw = u * w, p = uw + b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (a.act == DUALGCN_RELU) {
                bool pass = p[i] > 0.f;
                if (fabsf(p[i]) <= 0x1p-20f * (fabsf(uw[i]) + fabsf(b[i]))) {
                    const double2 st = stats[group[i]];
                    pass = (static_cast<double>(x[i]) - st.x) * st.y * w[i] + b[i] > 0.0;
                }
                g[i] = pass ? g[i] : 0.f;
            } else {
                const float q = sigmoid(p[i]);
                g[i] *= q + p[i] * q * (1.f - q);
            }
        }
        return g;
    }

    // f(row quad place, d, u) for a piece's rows
    template <class Fn>
    static __device__ __forceinline__ void rows(const GroupArgs &a, const Cols &c, const Piece &p, int t0, int t1, const Unit &unit,
                                                row_f32x4 w, row_f32x4 b, Fn f) {
        const int64_t first = static_cast<int64_t>(t0) * a.F, elems = static_cast<int64_t>(t1 - t0) * a.F;
        const __amdgpu_buffer_rsrc_t wx = row_window<X_BF>(a.X, first, elems);
        const __amdgpu_buffer_rsrc_t wg = row_window<G_BF>(a.dY, first, elems);
        const double2 *stats = a.stats + static_cast<int64_t>(p.graph) * a.G;
        for (int row = p.lo; row < p.hi; row += Cols::kRows * kAhead) {
            RawRowQuad<X_BF, TINY> x[kAhead];
            RawRowQuad<G_BF, TINY> g[kAhead];
            QuadPlace at[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int r = row + k * Cols::kRows;
                at[k] = moved(c.at, r - t0, a.F, r + c.slot < p.hi);
                x[k].load(wx, at[k].at, at[k].count);
                g[k].load(wg, at[k].at, at[k].count);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (row + k * Cols::kRows + c.slot >= p.hi) continue;
                const row_f32x4 xs = x[k].get(at[k], c.odd), u = unit(xs);
                f(at[k], inner(a, g[k].get(at[k], c.odd), xs, u, w, b, stats, c.group), u);
            }
        }
    }
    // dX of a piece's rows, from the sums of t and t u of its groups (`sums`: of the first group on)
    static __device__ __forceinline__ void apply(const GroupArgs &a, const Cols &c, const Piece &p, int t0, int t1, const Unit &unit,
                                                 row_f32x4 w, row_f32x4 b, const double2 *sums, int g0) {
        const __amdgpu_buffer_rsrc_t wd = row_window<G_BF>(a.out, static_cast<int64_t>(t0) * a.F, static_cast<int64_t>(t1 - t0) * a.F);
        row_f32x4 m1, m2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double2 v = sums[c.group[i] - g0];
            m1[i] = static_cast<float>(v.x / count_of(a, p));
            m2[i] = static_cast<float>(v.y / count_of(a, p));
        }
        rows(a, c, p, t0, t1, unit, w, b, [&](const QuadPlace &at, row_f32x4 d, row_f32x4 u) {
            store_row_quad<G_BF, TINY>(wd, at, unit.r * (d * w - m1 - u * m2), c.odd, false);
        });
    }
};

template <int L, bool X_BF, bool G_BF>
__global__ __launch_bounds__(kThreads) void group_back_kernel(GroupArgs a) {
    using K = Backward<L, X_BF, G_BF>;
    __shared__ double2 sh[2 * buffer_pairs<L>()];
    __shared__ double2 held[kSlice];
    int turn = 0;
    const typename K::Cols c(a);
    const int t0 = blockIdx.x * a.tile_rows, t1 = min(a.n, t0 + a.tile_rows);
    const row_f32x4 w = c.vector(a, a.weight, 1.f), b = c.vector(a, a.bias, 0.f);
    const int g0 = c.c0 / a.D;
    double sum_du[4] = {0.0, 0.0, 0.0, 0.0}, sum_d[4] = {0.0, 0.0, 0.0, 0.0};      // over all the tile's rows
    for (int row = t0; row < t1;) {
        const Piece p = piece_at(a, row, t0, t1);
        row = p.hi;
        if (p.graph < 0) {
            if (a.fill) Forward<L, X_BF, G_BF>::zero(a, c, p, t0, t1);
            continue;
        }
        Unit unit;
#pragma unroll
        for (int i = 0; i < 4; ++i) unit.set(i, a.stats[static_cast<int64_t>(p.graph) * a.G + c.group[i]]);
        double d1[4] = {0.0, 0.0, 0.0, 0.0}, d2[4] = {0.0, 0.0, 0.0, 0.0};
        K::rows(a, c, p, t0, t1, unit, w, b, [&](const QuadPlace &, row_f32x4 d, row_f32x4 u) {
            const row_f32x4 du = d * u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                d1[i] += d[i];
                d2[i] += du[i];
            }
        });
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum_d[i] += d1[i];
            sum_du[i] += d2[i];
            d1[i] *= w[i];
            d2[i] *= w[i];
        }
        const bool whole = !p.crosses && !a.split;
        group_sums<L>(a, c.c0, c.end, d1, d2, sh, turn, [&](int g, double2 v) {
            if (whole) held[g - g0] = v;
            else a.slots[(static_cast<int64_t>(blockIdx.x) + p.graph) * (a.slices + a.G) + blockIdx.y + g] = v;
        });
        if (whole) {
            __syncthreads();
            K::apply(a, c, p, t0, t1, unit, w, b, held, g0);
        }
    }
    // the columns' sums over the rows side by side
    if (!a.columns) return;
#pragma unroll
    for (int m = L; m < 64; m <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum_du[i] += __shfl_xor(sum_du[i], m);
            sum_d[i] += __shfl_xor(sum_d[i], m);
        }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane < L)
#pragma unroll
        for (int i = 0; i < 4; ++i) sh[wave * 4 * L + 4 * lane + i] = make_double2(sum_du[i], sum_d[i]);
    __syncthreads();
    double *to = a.columns + static_cast<int64_t>(blockIdx.x) * 2 * a.F;
    for (int i = threadIdx.x; i < 4 * L; i += kThreads) {
        if (c.c0 + i >= c.end) continue;
        double x = 0.0, y = 0.0;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            x += sh[v * 4 * L + i].x;
            y += sh[v * 4 * L + i].y;
        }
        to[c.c0 + i] = x;
        to[a.F + c.c0 + i] = y;
    }
}

// Workgroups up to `joins` in x join crossing graphs' sums, the others columns' sums, 16 of the 2 F each.
constexpr int kJoinColumns = 16;
__global__ __launch_bounds__(kThreads) void group_back_join_kernel(GroupArgs a, int32_t joins) {
    if (static_cast<int>(blockIdx.x) < joins) {
        const int parts = (a.G + kJoinGroups - 1) / kJoinGroups, tile = blockIdx.x / parts;
        join_tile(a, tile, static_cast<int>(blockIdx.x) % parts * kJoinGroups,
                  [&](const Piece &p, int g, double2 v) { a.joined[static_cast<int64_t>(p.graph) * a.G + g] = v; });
        return;
    }
    constexpr int kLanes = kThreads / kJoinColumns;
    __shared__ double sh[kThreads];
    const int64_t i = static_cast<int64_t>(blockIdx.x - joins) * kJoinColumns + threadIdx.x % kJoinColumns;
    const int k = threadIdx.x / kJoinColumns;
    double s = 0.0;
    if (i < 2 * static_cast<int64_t>(a.F))
#pragma unroll 8
        for (int t = k; t < a.tiles; t += kLanes) s += a.columns[static_cast<int64_t>(t) * 2 * a.F + i];
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
    using K = Backward<L, X_BF, G_BF>;
    const typename K::Cols c(a);
    const int tile = a.tiles - 1 - static_cast<int>(blockIdx.x);
    const int t0 = tile * a.tile_rows, t1 = min(a.n, t0 + a.tile_rows);
    const row_f32x4 w = c.vector(a, a.weight, 1.f), b = c.vector(a, a.bias, 0.f);
    unfinished(a, t0, t1, [&](const Piece &p) {
        Unit unit;
#pragma unroll
        for (int i = 0; i < 4; ++i) unit.set(i, a.stats[static_cast<int64_t>(p.graph) * a.G + c.group[i]]);
        K::apply(a, c, p, t0, t1, unit, w, b, a.joined + static_cast<int64_t>(p.graph) * a.G, 0);
    });
}

// ------------------------------------------------------------------ launches

int lanes_of(int32_t width) { return width < 4 ? 1 : width <= 32 ? 8 : width <= 64 ? 16 : width <= 128 ? 32 : 64; }

// Tiles: many enough to fill the chip, few enough that their partial sums stay small beside the rows, and of
// 32-bit offsets.
constexpr int kTiles = 2048;
struct Shape {
    int32_t tile_rows, tiles, slices, width;
    Shape(int32_t n, int32_t F, int32_t groups) {
        const int32_t D = F / groups;
        width = std::min(F, D > kSlice ? kSlice : kSlice / D * D);
        slices = (F + width - 1) / width;
        const int64_t side = kThreads / lanes_of(width), turn = side * kAhead;
        const int64_t want = std::max<int64_t>(1, kTiles / slices);
        int64_t rows = (n + want - 1) / want;
        rows = (rows + turn - 1) / turn * turn;
        const int64_t most = std::max<int64_t>(1, (int64_t{1} << 26) / F / turn) * turn;
        rows = std::min(rows, most);
        tile_rows = static_cast<int32_t>(rows);
        tiles = static_cast<int32_t>((n + rows - 1) / rows);
    }
};

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t slot_bytes(const Shape &s, int32_t B, int32_t G) {
    return up(sizeof(double2) * (static_cast<size_t>(s.tiles) + B) * (static_cast<size_t>(s.slices) + G));
}
size_t column_bytes(const Shape &s, int32_t F) { return up(sizeof(double) * 2 * static_cast<size_t>(s.tiles) * F); }

template <template <int, bool, bool> class Launch>
int by_type(const GroupArgs &a, bool x_bf, bool y_bf, hipStream_t s) {
#define DGC_GROUP_TYPES(L)                                                 \
    return x_bf ? (y_bf ? Launch<L, true, true>::go(a, s) : Launch<L, true, false>::go(a, s)) \
                : (y_bf ? Launch<L, false, true>::go(a, s) : Launch<L, false, false>::go(a, s))
    switch (lanes_of(a.width)) {
        case 1: DGC_GROUP_TYPES(1);
        case 8: DGC_GROUP_TYPES(8);
        case 16: DGC_GROUP_TYPES(16);
        case 32: DGC_GROUP_TYPES(32);
        default: DGC_GROUP_TYPES(64);
    }
#undef DGC_GROUP_TYPES
}

template <int L, bool X_BF, bool Y_BF>
struct ForwardLaunch {
    static int go(const GroupArgs &a, hipStream_t s) {
        const dim3 grid(a.tiles, a.slices), block(kThreads);
        hipLaunchKernelGGL((group_kernel<L, X_BF, Y_BF>), grid, block, 0, s, a);
        if (a.tiles > 1 || a.split) {
            hipLaunchKernelGGL((group_join_kernel<X_BF>), dim3(a.tiles, (a.G + kJoinGroups - 1) / kJoinGroups), block, 0, s, a);
            hipLaunchKernelGGL((group_apply_kernel<L, X_BF, Y_BF>), grid, block, 0, s, a);
        }
        return hip_status(hipGetLastError());
    }
};

template <int L, bool X_BF, bool G_BF>
struct BackwardLaunch {
    static int go(const GroupArgs &a, hipStream_t s) {
        const dim3 grid(a.tiles, a.slices), block(kThreads);
        hipLaunchKernelGGL((group_back_kernel<L, X_BF, G_BF>), grid, block, 0, s, a);
        const bool more = a.tiles > 1 || a.split;
        const int32_t joins = more ? a.tiles * ((a.G + kJoinGroups - 1) / kJoinGroups) : 0;
        const int32_t sums = a.columns ? (2 * a.F + kJoinColumns - 1) / kJoinColumns : 0;
        if (joins + sums) hipLaunchKernelGGL(group_back_join_kernel, dim3(joins + sums), block, 0, s, a, joins);
        if (more) hipLaunchKernelGGL((group_back_apply_kernel<L, X_BF, G_BF>), grid, block, 0, s, a);
        return hip_status(hipGetLastError());
    }
};

GroupArgs common(const dualgcn_group_norm &p, const void *X, int32_t n, const Shape &s, void *workspace) {
    GroupArgs a{};
    a.X = X;
    a.ptr = p.ptr;
    a.weight = p.weight;
    a.bias = p.bias;
    a.eps = p.eps;
    a.n = n;
    a.B = p.ptr ? p.graphs : 1;
    a.F = p.F;
    a.G = p.groups;
    a.D = p.F / p.groups;
    a.tile_rows = s.tile_rows;
    a.tiles = s.tiles;
    a.slices = s.slices;
    a.width = s.width;
    a.split = a.D > kSlice;
    a.act = static_cast<int32_t>(p.flags & (DUALGCN_RELU | DUALGCN_SILU));
    a.fill = p.flags & DUALGCN_ZERO_REST;
    a.slots = static_cast<double2 *>(workspace);
    return a;
}

}  // namespace

size_t group_norm_workspace_bytes(const dualgcn_group_norm &p, int32_t n) {
    return slot_bytes(Shape(n, p.F, p.groups), p.ptr ? p.graphs : 1, p.groups);
}

size_t group_norm_backward_workspace_bytes(const dualgcn_group_norm &p, int32_t n) {
    const Shape s(n, p.F, p.groups);
    const int32_t B = p.ptr ? p.graphs : 1;
    return slot_bytes(s, B, p.groups) + up(sizeof(double2) * static_cast<size_t>(B) * p.groups) + column_bytes(s, p.F);
}

int launch_group_norm(const dualgcn_group_norm &p, const void *X, void *Y, double *stats, int32_t n, void *workspace,
                      hipStream_t s) {
    GroupArgs a = common(p, X, n, Shape(n, p.F, p.groups), workspace);
    a.out = Y;
    a.stats = reinterpret_cast<double2 *>(stats);
    return by_type<ForwardLaunch>(a, p.flags & DUALGCN_IN_BF16, p.flags & DUALGCN_OUT_BF16, s);
}

int launch_group_norm_backward(const dualgcn_group_norm &p, const void *X, const void *dY, const double *stats, void *dX,
                               float *dweight, float *dbias, int32_t n, void *workspace, hipStream_t s) {
    const Shape shape(n, p.F, p.groups);
    GroupArgs a = common(p, X, n, shape, workspace);
    a.dY = dY;
    a.out = dX;
    a.stats = reinterpret_cast<double2 *>(const_cast<double *>(stats));
    char *more = static_cast<char *>(workspace) + slot_bytes(shape, a.B, a.G);
    a.joined = reinterpret_cast<double2 *>(more);
    more += up(sizeof(double2) * static_cast<size_t>(a.B) * a.G);
    a.columns = dweight || dbias ? reinterpret_cast<double *>(more) : nullptr;
    a.dweight = dweight;
    a.dbias = dbias;
    return by_type<BackwardLaunch>(a, p.flags & DUALGCN_IN_BF16, p.flags & DUALGCN_GRAD_BF16, s);
}

}  // namespace dgc
