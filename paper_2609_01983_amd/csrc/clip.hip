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
// launch, and workgroups take them in turn.  Each workgroup leaves one partial sum; every workgroup of the second pass
// joins all of them in the same order, which costs it about a load's time and saves a launch.
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
__device__ __forceinline__ double block_sum(double v) {
    __shared__ row_f32x4 sh[row_reduce_quads<kThreads>()];
    int turn = 0;
    return row_sum<kThreads>(v, sh, turn);
}

template <bool BF>
__device__ __forceinline__ double squares(const void *g, int64_t at, int64_t count) {
    row_f32x4 v[kQuads];
    const int64_t left = count - at;
    if (left >= kChunk) {
#pragma unroll
        for (int k = 0; k < kQuads; ++k) v[k] = load_quad<BF>(g, at + 4 * (k * kThreads + static_cast<int>(threadIdx.x)), 4);
    } else {
#pragma unroll
        for (int k = 0; k < kQuads; ++k) {
            const int i = 4 * (k * kThreads + static_cast<int>(threadIdx.x));
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

__global__ __launch_bounds__(kThreads) void square_kernel(SumTable<kSumTensors> t, double *__restrict__ partial) {
    double s = 0.0;
    const uint32_t chunks = t.first[t.tensors];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int k = tensor_of(t, c);
        const int64_t at = static_cast<int64_t>(c - t.first[k]) * kChunk, n = t.count[k];
        s += n < 0 ? squares<true>(t.grad[k], at, -n) : squares<false>(t.grad[k], at, n);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// sqrt of the partial sums' sum, in a fixed order.
__device__ __forceinline__ double norm_of(const double *__restrict__ partial, int32_t partials) {
    double s = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
    return sqrt(block_sum(s));
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double *__restrict__ partial, int32_t partials, float *norm) {
    const double v = norm_of(partial, partials);
    if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

template <bool BF>
__device__ __forceinline__ void scale_chunk(const void *g, const float *w, void *out, int64_t at, int64_t count, double f) {
    row_f32x4 v[kQuads], x[kQuads];
    const int64_t left = count - at;
    const int most = left < kChunk ? static_cast<int>(left) : kChunk;
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
        const int i = 4 * (k * kThreads + static_cast<int>(threadIdx.x));
        v[k] = load_quad<BF>(g, at + i, most - i);
        if (w) x[k] = load_quad<false>(w, at + i, most - i);
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
        const int i = 4 * (k * kThreads + static_cast<int>(threadIdx.x));
        row_f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = static_cast<float>(w ? fma(f, static_cast<double>(v[k][e]), static_cast<double>(x[k][e])) : f * static_cast<double>(v[k][e]));
        if (BF && !w) store_quad<true>(out, at + i, most - i, y);
        else store_quad<false>(out, at + i, most - i, y);
    }
}

__global__ __launch_bounds__(kThreads) void apply_kernel(ApplyTable<kApplyTensors> t, const double *__restrict__ partial,
                                                         int32_t partials, double max_norm, double eps, double lr, float *norm) {
    const double v = norm_of(partial, partials), with = v + eps;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(v);
    double f = with <= max_norm ? 1.0 : max_norm / with;         // (a NaN stays one)
    const uint32_t chunks = t.first[t.tensors];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int k = tensor_of(t, c);
        const int64_t at = static_cast<int64_t>(c - t.first[k]) * kChunk, n = t.count[k];
        const double by = t.weight[k] ? -lr * f : f;
        if (n < 0) scale_chunk<true>(t.grad[k], t.weight[k], t.out[k], at, -n, by);
        else scale_chunk<false>(t.grad[k], t.weight[k], t.out[k], at, n, by);
    }
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
        if (t.tensors == N || t.first[t.tensors] + chunks > 0x40000000) {
            if (t.first[t.tensors]) go(t);
            t.tensors = 0;
        }
        if (!chunks) continue;
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

int launch_clip(const dualgcn_grad *g, int32_t tensors, bool apply, double max_norm, double eps, double lr, float *norm,
                void *workspace, hipStream_t s) {
    double *partial = static_cast<double *>(workspace);
    int32_t partials = 0;
    in_tables<SumTable<kSumTensors>, kSumTensors>(
        g, tensors, [](SumTable<kSumTensors> &, int, const dualgcn_grad &) {},
        [&](const SumTable<kSumTensors> &t) {
            const int32_t grid = static_cast<int32_t>(std::min<uint32_t>(t.first[t.tensors], kGrid));
            hipLaunchKernelGGL(square_kernel, dim3(grid), dim3(kThreads), 0, s, t, partial + partials);
            partials += grid;
        });
    if (apply)
        in_tables<ApplyTable<kApplyTensors>, kApplyTensors>(
            g, tensors,
            [](ApplyTable<kApplyTensors> &t, int at, const dualgcn_grad &one) {
                t.weight[at] = one.weight;
                t.out[at] = one.out;
            },
            [&](const ApplyTable<kApplyTensors> &t) {
                const uint32_t grid = std::min<uint32_t>(t.first[t.tensors], kGrid);
                hipLaunchKernelGGL(apply_kernel, dim3(grid), dim3(kThreads), 0, s, t, partial, partials, max_norm, eps, lr, norm);
                norm = nullptr;
            });
    if (norm) hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, s, partial, partials, norm);
    return hip_status(hipGetLastError());
}

}  // namespace dgc
