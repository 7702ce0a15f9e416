// The norm of many gradients together, and what is done with it: the gradients scaled to a norm of max_norm
// at most, or an SGD step with them.
//
//   norm = sqrt(sum over tensors and elements of g^2),  f = min(1, max_norm / (norm + eps))
//   out = f g,  or  out = W - lr f g
//
// Squares and sums are float64: squares of float32 numbers are exact there and neither overflow nor vanish,
// and the vector unit's float64 rate is many times what memory asks for.  The results are formed in float64
// too and rounded once (to bfloat16 by way of float32).
//
// A launch takes up to a few hundred tensors, whose addresses and sizes are its arguments: nothing is copied to
// the device, so that calls can be captured.  Tensors are cut into chunks, the chunks are numbered over all tensors of a
// launch, and workgroups take them in turn.  Each workgroup leaves one partial sum; where those are no more than one launch's,
// every workgroup of the second pass joins all of them in the same order, which costs it about a load's time and saves a launch; where there
// are more, one workgroup joins them first, in that order too.
//
// Bound by memory: 322 tensors of 2.7e8 elements, half of them bfloat16, squares 158 us (0.8 GB, 5.1 TB/s) and step 568 us
// (2.95 GB, 5.2 TB/s), besides 37 us of launches for the vectors and the join; 40,960 elements of two tensors in one launch 7.3 us.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kQuads = 8;                            // a thread's loads of four elements in flight
constexpr int kChunk = kThreads * kQuads * 4;        // elements
constexpr int kGrid = kClipPartials;                 // workgroups of a launch, at most

// The tensors of a launch; first[t] is the number of tensor t's first chunk.
template <int N>
struct SumTable {
    const void *grad[N];
    int64_t count[N];                                // negative: bfloat16
    uint32_t first[N + 1];
    int32_t tensors;
};
template <int N>
struct ApplyTable {
    const void *grad[N];
    const float *weight[N];
    void *out[N];
    int64_t count[N];
    uint32_t first[N + 1];
    int32_t tensors;
};
constexpr int kSumTensors = 160, kApplyTensors = 88;  // about 3.3 KB of arguments

// The tensor that a chunk is of.
template <class Table>
__device__ __forceinline__ int tensor_of(const Table &t, uint32_t chunk) {
    int lo = 0, hi = t.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The sum over a workgroup, the same in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ row_f32x4 sh[row_reduce_quads<THREADS>()];
    int turn = 0;
    return row_sum<THREADS>(v, sh, turn);
}

template <bool BF>
__device__ __forceinline__ double squares(const void *g, int64_t at, int64_t count, int thread) {
    row_f32x4 v[kQuads];
    const int64_t left = count - at;
    if (left >= kChunk) {
#pragma unroll
        for (int k = 0; k < kQuads; ++k) v[k] = load_quad<BF>(g, at + 4 * (k * kThreads + thread), 4);
    } else {
#pragma unroll
        for (int k = 0; k < kQuads; ++k) {
            const int i = 4 * (k * kThreads + thread);
            v[k] = load_quad<BF>(g, at + i, static_cast<int>(left) - i);
        }
    }
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double d = v[k][i];
            s[i] = fma(d, d, s[i]);
        }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Chunk c of a table: its elements' squares' sum, or the result.
template <class Table>
__device__ __forceinline__ double squares_of(const Table &t, uint32_t c, int thread) {
    const int k = tensor_of(t, c);
    const int64_t at = static_cast<int64_t>(c - t.first[k]) * kChunk, n = t.count[k];
    return n < 0 ? squares<true>(t.grad[k], at, -n, thread) : squares<false>(t.grad[k], at, n, thread);
}

template <int N>
__global__ __launch_bounds__(kThreads) void square_kernel(SumTable<N> t, double *__restrict__ partial) {
    double s = 0.0;
    const uint32_t chunks = t.first[t.tensors];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) s += squares_of(t, c, threadIdx.x);
    s = block_sum<kThreads>(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The partial sums' sum, in a fixed order; the norm is its root.
__device__ __forceinline__ double sum_of(const double *partial, int32_t partials) {
    double s = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
    return block_sum<kThreads>(s);
}
__device__ __forceinline__ double norm_of(const double *__restrict__ partial, int32_t partials) { return sqrt(sum_of(partial, partials)); }

// Partial sums that every workgroup of the second pass joins for itself, at most; that takes time by their number times the tensors', a launch
// before it 3 to 4 us (steps in us, each for itself and by a launch: 9 tensors of 8,192 elements 36.8, 40.1; 160 of 131,072, 2,048
// partial sums, 68.0, 69.2; 320, 4,096 sums, 155, 149; 640 336, 311; 2,000 1,181, 885; 10^5 of 100 elements 22,600, 10,100).
constexpr int32_t kJoined = kGrid;

// Leaves the partial sums' sum in the place of the first.
__global__ __launch_bounds__(kThreads) void join_kernel(double *partial, int32_t partials) {
    const double s = sum_of(partial, partials);
    if (threadIdx.x == 0) *partial = s;              // (all have been read: the sum needs every thread's)
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double *__restrict__ partial, int32_t partials, float *norm) {
    const double v = norm_of(partial, partials);
    if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

template <bool BF>
__device__ __forceinline__ void scale_chunk(const void *g, const float *w, void *out, int64_t at, int64_t count, double f, int thread) {
    row_f32x4 v[kQuads], x[kQuads];
    const int64_t left = count - at;
    const int most = left < kChunk ? static_cast<int>(left) : kChunk;
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
        const int i = 4 * (k * kThreads + thread);
        v[k] = load_quad<BF>(g, at + i, most - i);
        if (w) x[k] = load_quad<false>(w, at + i, most - i);
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
        const int i = 4 * (k * kThreads + thread);
        row_f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = static_cast<float>(w ? fma(f, static_cast<double>(v[k][e]), static_cast<double>(x[k][e])) : f * static_cast<double>(v[k][e]));
        if (BF && !w) store_quad<true>(out, at + i, most - i, y);
        else store_quad<false>(out, at + i, most - i, y);
    }
}

__device__ __forceinline__ double factor_of(double norm, double max_norm, double eps) {
    return norm + eps <= max_norm ? 1.0 : max_norm / (norm + eps);       // (a NaN stays one)
}
template <class Table>
__device__ __forceinline__ void scale_of(const Table &t, uint32_t c, double f, double lr, int thread) {
    const int k = tensor_of(t, c);
    const int64_t at = static_cast<int64_t>(c - t.first[k]) * kChunk, n = t.count[k];
    const double by = t.weight[k] ? -lr * f : f;
    if (n < 0) scale_chunk<true>(t.grad[k], t.weight[k], t.out[k], at, -n, by, thread);
    else scale_chunk<false>(t.grad[k], t.weight[k], t.out[k], at, n, by, thread);
}

template <int N>
__global__ __launch_bounds__(kThreads) void apply_kernel(ApplyTable<N> t, const double *__restrict__ partial, int32_t partials, double max_norm,
                                                         double eps, double lr, float *norm) {
    const double v = norm_of(partial, partials);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(v);
    const double f = factor_of(v, max_norm, eps);
    const uint32_t chunks = t.first[t.tensors];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) scale_of(t, c, f, lr, threadIdx.x);
}

// Few small tensors: both passes by one workgroup, four chunks at a time (two tensors of 40,960 elements: 11 us a call against 13.5 by
// two launches, most of it on the host).
constexpr int kSmallThreads = 4 * kThreads, kSmallTensors = 8, kSmallChunks = 8;
__global__ __launch_bounds__(kSmallThreads) void small_kernel(ApplyTable<kSmallTensors> t, bool apply, double max_norm, double eps, double lr, float *norm) {
    const uint32_t chunks = t.first[t.tensors], first = threadIdx.x / kThreads;
    const int thread = threadIdx.x % kThreads;
    double s = 0.0;
    for (uint32_t c = first; c < chunks; c += kSmallThreads / kThreads) s += squares_of(t, c, thread);
    const double v = sqrt(block_sum<kSmallThreads>(s)), f = factor_of(v, max_norm, eps);
    if (threadIdx.x == 0) *norm = static_cast<float>(v);
    if (apply)
        for (uint32_t c = first; c < chunks; c += kSmallThreads / kThreads) scale_of(t, c, f, lr, thread);
}

// Launches over the tensors, as many at a time as a table holds: fill(table, place, tensor) and
// go(table, chunks).
template <class Table, int N, class Fill, class Go>
void in_tables(const dualgcn_grad *g, int32_t tensors, Fill fill, Go go) {
    Table t;
    t.tensors = 0;
    t.first[0] = 0;
    for (int32_t i = 0; i < tensors; ++i) {
        const int64_t chunks = (g[i].count + kChunk - 1) / kChunk;
        if (!chunks) continue;
        if (t.tensors == N) {
            go(t);
            t.tensors = 0;
        }
        t.grad[t.tensors] = g[i].grad;
        t.count[t.tensors] = g[i].flags & DUALGCN_GRAD_BF16 ? -g[i].count : g[i].count;
        fill(t, t.tensors, g[i]);
        t.first[t.tensors + 1] = t.first[t.tensors] + static_cast<uint32_t>(chunks);
        ++t.tensors;
    }
    if (t.tensors) go(t);
}

}  // namespace

size_t clip_workspace_bytes(int32_t tensors) {
    // a table's workgroups leave kGrid partial sums at most
    const size_t tables = (static_cast<size_t>(tensors) + kSumTensors - 1) / kSumTensors;
    return tables * kGrid * sizeof(double);
}

namespace {

template <int S, int A>
int launch_tables(const dualgcn_grad *g, int32_t tensors, bool apply, double max_norm, double eps, double lr, float *norm, double *partial,
                  hipStream_t s) {
    int32_t partials = 0;
    in_tables<SumTable<S>, S>(
        g, tensors, [](SumTable<S> &, int, const dualgcn_grad &) {},
        [&](const SumTable<S> &t) {
            const int32_t grid = static_cast<int32_t>(std::min<uint32_t>(t.first[t.tensors], kGrid));
            hipLaunchKernelGGL(square_kernel<S>, dim3(grid), dim3(kThreads), 0, s, t, partial + partials);
            partials += grid;
        });
    if (apply && partials > kJoined) {
        hipLaunchKernelGGL(join_kernel, dim3(1), dim3(kThreads), 0, s, partial, partials);
        partials = 1;
    }
    if (apply)
        in_tables<ApplyTable<A>, A>(
            g, tensors,
            [](ApplyTable<A> &t, int at, const dualgcn_grad &one) {
                t.weight[at] = one.weight;
                t.out[at] = one.out;
            },
            [&](const ApplyTable<A> &t) {
                const uint32_t grid = std::min<uint32_t>(t.first[t.tensors], kGrid);
                hipLaunchKernelGGL(apply_kernel<A>, dim3(grid), dim3(kThreads), 0, s, t, partial, partials, max_norm, eps, lr, norm);
                norm = nullptr;
            });
    if (norm) hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, s, partial, partials, norm);
    return hip_status(hipGetLastError());
}

}  // namespace

int launch_clip(const dualgcn_grad *g, int32_t tensors, bool apply, double max_norm, double eps, double lr, float *norm,
                void *workspace, hipStream_t s) {
    double *partial = static_cast<double *>(workspace);
    if (tensors > kSmallTensors)
        return launch_tables<kSumTensors, kApplyTensors>(g, tensors, apply, max_norm, eps, lr, norm, partial, s);
    int64_t chunks = 0;
    for (int32_t i = 0; i < tensors; ++i) chunks += (g[i].count + kChunk - 1) / kChunk;
    if (chunks == 0 || chunks > kSmallChunks)
        return launch_tables<kSmallTensors, kSmallTensors>(g, tensors, apply, max_norm, eps, lr, norm, partial, s);
    in_tables<ApplyTable<kSmallTensors>, kSmallTensors>(
        g, tensors,
        [](ApplyTable<kSmallTensors> &t, int at, const dualgcn_grad &one) {
            t.weight[at] = one.weight;
            t.out[at] = one.out;
        },
        [&](const ApplyTable<kSmallTensors> &t) { hipLaunchKernelGGL(small_kernel, dim3(1), dim3(kSmallThreads), 0, s, t, apply, max_norm, eps, lr, norm); });
    return hip_status(hipGetLastError());
}

}  // namespace dgc
