// Norms before and after a block, with the block's gate and residual scale, forward and backward.
//
// Forward, row by row (R the residual stream, B the block's output):
//   post(B) = w1 * u1 + b1,  u1 = (B - m1) r1,  r1 = 1 / sqrt(mean((B - m1)^2) + eps)
//   R' = R + scale * gate * post(B)
//   Z  = w2 * u2 + b2,       u2 = (R' - m2) r2  (the norm before the next block)
// with m = the row's mean (layer norm) or 0 (RMS norm).
//
// Backward, for gradients dZ of Z and dR' of R' from elsewhere:
//   t = dZ w2,  d = dR' + r2 (t - [mean(t)] - u2 mean(t u2)),  dR = d
//   dgate = scale d post(B),  v = scale d gate,  s = v w1
//   dB = r1 (s - [mean(s)] - u1 mean(s u1))
//   dw2 = sum dZ u2,  db2 = sum dZ,  dw1 = sum v u1,  db1 = sum v
// ([.] for the layer norm only).  The statistics are computed again from B and R', which the
// backward pass reads in any case: that costs two reductions in registers and no bytes.
//
// Z norms the stream as it is stored.  Where the stream is bfloat16 and Z float32, the last bits of a sum that lies
// beside the middle of two bfloat16 numbers decide over half a percent of an element of Z (of float32 sums, one
// element in 20,000 was not the formula's): there the sum is formed in float64, with eps and scale as the caller has
// them, rounded to float32 and stored as any float32 sum.  (So a sum that is the middle but for the last bits of a
// float64, as 0.7 B often makes it, goes to the even number.)
//
// Both passes are bound by memory (about one flop a byte): a row stays in the registers of
// its threads from the load to the store, so every operand is read and every output written
// once.  The threads of a row are as many as hold it in few quads: 8 to 64 lanes of a
// wavefront up to 768 features, a workgroup of 128 to 1,024 threads up to 8,192.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 1024;                     // workgroups, hence partial column sums, of a backward pass
template <int TPR>
constexpr int kMostBlocks = TPR > 256 ? kMaxBlocks / 2 : kMaxBlocks;     // (at most one a CU where they are so large)
// Rows that a group of threads adds to a column sum in float32, one after another.  The error of such a chain grows
// with its length (67M rows of 4 in chains of 4,096 terms of 0.1: 4e-5 of the sum), so longer passes are done in parts,
// whose sums are added in float64 (us whole, in parts of 256, 128, 64 steps: 2^20 x 128 605, 605, 591, 602; 2^21 x 128 1,295, 1,200,
// 1,169, 1,186; 2^17 x 1,024 595, 596, 607, 633; 2^17 x 4,096 bfloat16 1,654, 1,670, 1,709, 1,784).
constexpr int kChain = 128;
constexpr int64_t kMaxForwardBlocks = int64_t{1} << 21;

// ------------------------------------------------------------------ shared by both directions

template <int TPR, int Q>
struct Shape {
    static constexpr int kBlock = TPR > 64 ? TPR : kThreads;         // threads of a workgroup
    static constexpr int kGroups = kBlock / TPR;                     // rows it works on at a time
};

// Where a vector of F features may be: a window of it, or what stands for a missing one.
struct Vector {
    __amdgpu_buffer_rsrc_t w;
    bool there;
    float missing;
    __device__ __forceinline__ Vector(const void *p, int F, float missing_)
        : w(row_window<false>(p, 0, p ? F : 0)), there(p != nullptr), missing(missing_) {}
    template <int Q, bool TINY>
    __device__ __forceinline__ void load(const QuadPlace (&at)[Q], bool odd, row_f32x4 (&out)[Q]) const {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (there) {
                RawRowQuad<false, TINY> raw;
                raw.load(w, at[q].col, at[q].count);
                out[q] = raw.get(at[q], odd);
            } else {
                out[q] = row_f32x4{missing, missing, missing, missing};
            }
        }
    }
};

// zeros behind the row's end; ragged: the row has fewer columns than its threads have places
template <int Q>
__device__ __forceinline__ void cut(row_f32x4 (&x)[Q], const QuadPlace (&at)[Q], bool ragged) {
    if (ragged)
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i >= at[q].count) x[q][i] = 0.f;
}

template <int Q>
__device__ __forceinline__ void centre(row_f32x4 (&x)[Q], float mean, const QuadPlace (&at)[Q], bool ragged) {
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] -= mean;
    cut(x, at, ragged);
}

template <int Q>
__device__ __forceinline__ float sum_of(const row_f32x4 (&x)[Q]) {
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) s += (x[q][0] + x[q][1]) + (x[q][2] + x[q][3]);
    return s;
}

template <int Q>
__device__ __forceinline__ float dot_of(const row_f32x4 (&x)[Q], const row_f32x4 (&y)[Q]) {
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) s = fmaf(x[q][i], y[q][i], s);
    return s;
}

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// x on entry, (x - mean) r on return; the row's threads share the statistics
template <int TPR, int Q, bool LAYER>
__device__ __forceinline__ void normalise(row_f32x4 (&x)[Q], const QuadPlace (&at)[Q], bool ragged, float inv_f,
                                          float eps, row_f32x4 *sh, int &turn) {
    if constexpr (LAYER) {
        float m[1] = {sum_of(x)};
        row_reduce<TPR>(m, AddOp(), sh, turn);
        centre(x, m[0] * inv_f, at, ragged);
    }
    float s[1] = {dot_of(x, x)};
    row_reduce<TPR>(s, AddOp(), sh, turn);
    const float r = __builtin_amdgcn_rsqf(fmaf(s[0], inv_f, eps));
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] *= r;
}

__device__ __forceinline__ double sigmoid(double x) { return 1.0 / (1.0 + exp(-x)); }

// 1 / sqrt(x) of a float64: the hardware's estimate (2^-23) and two of Newton's steps; 0 of infinity
__device__ __forceinline__ double inverse_root(double x) {
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int k = 0; k < 2; ++k) r = fma(0.5 * r, fma(-x * r, r, 1.0), r);
    return x == INFINITY ? 0.0 : r;
}

// normalise() in float64
template <int TPR, int Q, bool LAYER>
__device__ __forceinline__ void normalise(row_f64x4 (&x)[Q], const QuadPlace (&at)[Q], bool ragged, double inv_f,
                                          double eps, row_f32x4 *sh, int &turn) {
    if constexpr (LAYER) {
        double m = 0.0;
#pragma unroll
        for (int q = 0; q < Q; ++q) m += (x[q][0] + x[q][1]) + (x[q][2] + x[q][3]);
        m = row_sum<TPR>(m, sh, turn) * inv_f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            x[q] -= m;
            if (ragged)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= at[q].count) x[q][i] = 0.0;
        }
    }
    double s = 0.0;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) s = fma(x[q][i], x[q][i], s);
    s = row_sum<TPR>(s, sh, turn);
    const double r = inverse_root(fma(s, inv_f, eps));
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] *= r;
}

// ------------------------------------------------------------------ forward

struct ForwardArgs {
    const void *R, *B, *gate;
    void *Rn, *Z;
    const float *w1, *b1, *w2, *b2;
    int32_t n, F;
    float eps, scale;
    uint32_t flags;
    bool streaming;                  // outputs past the L2s: stored with a non-temporal hint
    double inv_f, eps64, scale64;    // for float64 sums: 1 / F, and eps and scale as the caller has them
};

// LAYER: layer norms; A: B and a full gate are bfloat16; S: the stream is; EXACT (S, B there, a float32 Z): the stream's
// sum is formed in float64.  Behind a row's end every operand and weight is zero, so RMS norms need no masks; a
// mean taken off is cut there.
// Measured: 2^21 x 256, both RMS norms and a gate a feature, float32 in, bfloat16 Z: 7.5 GB in 1.29 ms, 5.8 TB/s
// (a copy of that size: 5.2 to 5.5); one row of 256: 2.0 us, the launch itself.  The weights' vectors are
// read again by each workgroup, from the caches.
template <int TPR, int Q, bool LAYER, bool A, bool S, bool EXACT>
__global__ __launch_bounds__((Shape<TPR, Q>::kBlock)) void norm_residual_kernel(ForwardArgs a) {
    constexpr bool TINY = TPR == 1;
    constexpr int kGroups = Shape<TPR, Q>::kGroups;
    __shared__ row_f32x4 sh[row_reduce_quads<TPR>()];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int F = a.F;
    const bool odd = F & 3, ragged = F != 4 * TPR * Q;
    const float inv_f = 1.f / static_cast<float>(F);
    const bool post = a.flags & DUALGCN_NORM_POST, sig = a.flags & DUALGCN_GATE_SIGMOID;
    QuadPlace at[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) at[q].set(static_cast<uint32_t>(g) * F, 4 * (l + q * TPR), F);

    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kGroups; row0 < a.n;
         row0 += static_cast<int64_t>(gridDim.x) * kGroups) {
        const int64_t first = row0 * F;
        const int rows = static_cast<int>(min(static_cast<int64_t>(kGroups), a.n - row0));
        const int64_t elems = static_cast<int64_t>(rows) * F;
        RawRowQuad<S, TINY> rr[Q];
        RawRowQuad<A, TINY> rb[Q], rg[Q];
        float gn = 1.f;
        const __amdgpu_buffer_rsrc_t wr = row_window<S>(a.R, first, elems);
#pragma unroll
        for (int q = 0; q < Q; ++q) rr[q].load(wr, at[q].at, at[q].count);
        if (a.B) {
            const __amdgpu_buffer_rsrc_t wb = row_window<A>(a.B, first, elems);
#pragma unroll
            for (int q = 0; q < Q; ++q) rb[q].load(wb, at[q].at, at[q].count);
            if (a.flags & DUALGCN_GATE_FULL) {
                const __amdgpu_buffer_rsrc_t wg = row_window<A>(a.gate, first, elems);
#pragma unroll
                for (int q = 0; q < Q; ++q) rg[q].load(wg, at[q].at, at[q].count);
            }
            if (a.flags & DUALGCN_GATE_NODE) gn = static_cast<const float *>(a.gate)[row0 + (g < rows ? g : 0)];
        }
        row_f32x4 x[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) x[q] = rr[q].get(at[q], odd);
        if (a.B) {
            typedef typename std::conditional<EXACT, row_f64x4, row_f32x4>::type Sum4;
            typedef typename std::conditional<EXACT, double, float>::type Sum;
            Sum4 v[Q];
            row_f32x4 w[Q], c[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) v[q] = __builtin_convertvector(rb[q].get(at[q], odd), Sum4);
            if (post) {
                Vector(a.w1, F, 1.f).load<Q, TINY>(at, odd, w);
                if constexpr (LAYER) Vector(a.b1, F, 0.f).load<Q, TINY>(at, odd, c);
                if constexpr (EXACT) normalise<TPR, Q, LAYER>(v, at, ragged, a.inv_f, a.eps64, sh, turn);
                else normalise<TPR, Q, LAYER>(v, at, ragged, inv_f, a.eps, sh, turn);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    v[q] *= __builtin_convertvector(w[q], Sum4);
                    if constexpr (LAYER) v[q] += __builtin_convertvector(c[q], Sum4);
                }
            }
            if (a.flags & (DUALGCN_GATE_FEATURE | DUALGCN_GATE_FULL)) {
                if (a.flags & DUALGCN_GATE_FEATURE) {
                    Vector(a.gate, F, 1.f).load<Q, TINY>(at, odd, w);
                } else {
#pragma unroll
                    for (int q = 0; q < Q; ++q) w[q] = rg[q].get(at[q], odd);
                }
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    Sum4 gate = __builtin_convertvector(w[q], Sum4);
                    if (sig)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            gate[i] = sigmoid(gate[i]);
                            if constexpr (EXACT) __builtin_amdgcn_sched_barrier(0);    // registers for one exponential at a time
                        }
                    v[q] *= gate;
                }
            }
            Sum node = gn;
            if (sig && (a.flags & DUALGCN_GATE_NODE)) node = sigmoid(node);
            const Sum scale = EXACT ? node : a.scale * node;
            const __amdgpu_buffer_rsrc_t wn = row_window<S>(a.Rn, first, elems);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // the next norm (and the backward pass) take the stream as it is stored
                    // (anew: the compiler would join the two roundings to one)
                    if constexpr (EXACT) x[q][i] = anew(static_cast<float>(fma(a.scale64, scale * v[q][i], static_cast<double>(x[q][i]))));
                    else x[q][i] = fmaf(scale, v[q][i], x[q][i]);
                    if constexpr (S) x[q][i] = through_bf16(x[q][i]);
                }
                store_row_quad<S, TINY>(wn, at[q], x[q], odd, a.streaming);
            }
        }
        if (a.Z) {
            row_f32x4 w[Q], c[Q];
            Vector(a.w2, F, 1.f).load<Q, TINY>(at, odd, w);
            if constexpr (LAYER) Vector(a.b2, F, 0.f).load<Q, TINY>(at, odd, c);
            normalise<TPR, Q, LAYER>(x, at, ragged, inv_f, a.eps, sh, turn);
#pragma unroll
            for (int q = 0; q < Q; ++q) x[q] = LAYER ? x[q] * w[q] + c[q] : x[q] * w[q];
            if (!EXACT && (a.flags & DUALGCN_OUT_BF16)) {
                const __amdgpu_buffer_rsrc_t wz = row_window<true>(a.Z, first, elems);
#pragma unroll
                for (int q = 0; q < Q; ++q) store_row_quad<true, TINY>(wz, at[q], x[q], odd, a.streaming);
            } else {
                const __amdgpu_buffer_rsrc_t wz = row_window<false>(a.Z, first, elems);
#pragma unroll
                for (int q = 0; q < Q; ++q) store_row_quad<false, TINY>(wz, at[q], x[q], odd, a.streaming);
            }
        }
    }
}

// ------------------------------------------------------------------ backward

// Column sums of a backward pass, in this order in a workgroup's partial sums; each is there
// only if it is wanted.
enum Slot { kW1 = 0, kB1 = 1, kW2 = 2, kB2 = 3, kGate = 4, kSlots = 5 };

struct BackwardArgs {
    const void *Rn, *B, *gate, *dZ, *dRn;
    void *dR, *dB, *dgate;
    const float *w1, *b1, *w2;
    float *partial;                  // [workgroups][slots wanted][F]
    int32_t n, F;
    float eps, scale;
    uint32_t flags;
    uint32_t want;                   // bit s: slot s is wanted
    bool streaming;
};

// What a backward pass reads of its rows, from `row0` on.
template <int Q, bool TINY, bool A, bool S, bool G>
struct RowIn {
    RawRowQuad<S, TINY> r[Q], d[Q];
    RawRowQuad<G, TINY> z[Q];
    RawRowQuad<A, TINY> b[Q], g[Q];
    float gn;

    template <class T>
    __device__ __forceinline__ static void take(T (&to)[Q], __amdgpu_buffer_rsrc_t w, const QuadPlace (&at)[Q]) {
#pragma unroll
        for (int q = 0; q < Q; ++q) to[q].load(w, at[q].at, at[q].count);
    }
    // no rows (row0 >= n): zeros
    __device__ __forceinline__ void load(const BackwardArgs &a, int64_t row0, int groups, int group, const QuadPlace (&at)[Q]) {
        const int64_t rows = max(int64_t{0}, min(static_cast<int64_t>(groups), a.n - row0));
        const int64_t first = row0 * a.F, elems = rows * a.F;
        if (a.dZ) {
            take(r, row_window<S>(a.Rn, first, elems), at);
            take(z, row_window<G>(a.dZ, first, elems), at);
        }
        if (a.dRn) take(d, row_window<S>(a.dRn, first, elems), at);
        if (a.B) {
            take(b, row_window<A>(a.B, first, elems), at);
            if (a.flags & DUALGCN_GATE_FULL) take(g, row_window<A>(a.gate, first, elems), at);
            gn = 1.f;
            if (a.flags & DUALGCN_GATE_NODE)
                gn = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row_window<false>(a.gate, row0, rows), group * 4u, 0, 0));
        }
    }
};

// LAYER: layer norms; A: B and a full gate are bfloat16; S: the stream and its gradients are; G: dZ,
// dB and a full gate's gradient are.  The workgroups are few and keep their column sums over all their
// rows, so that the partial sums are small beside the rows.
// Measured: 2^20 x 128 float32, RMS norms and a gate a feature, 3.2 GB in two parts of 289 to 300 us, 5.4 to 5.6 TB/s; 8,191 x
// 4,096 bfloat16 403 MB in 106 to 109 us, 3.8 TB/s, bound by the two reductions of each row of which a workgroup of 1,024 threads
// has one at work and one on its way; 20,001 x 99 with layer norms and a sigmoid gate 55 MB in 23 us: five rounds of
// latency, and the columns' sums joined at the end.
template <int TPR, int Q, bool LAYER, bool A, bool S, bool G>
__global__ __launch_bounds__((Shape<TPR, Q>::kBlock)) void norm_backward_kernel(BackwardArgs a) {
    constexpr bool TINY = TPR == 1;
    // One quad a thread: the weights and the column sums stay in registers over the rows.  More: the
    // weights are read again from the cache, and the sums of w1, b1, w2, b2 are kept in LDS, each thread
    // at its own places (6 accesses of 16 bytes a quad, a small part of LDS's rate).
    constexpr bool kHold = Q <= 1;
    constexpr bool kAhead = Q < 4;                   // registers for the next row's operands
    extern __shared__ row_f32x4 kept[];              // !kHold: [slots wanted of the four][Q][kBlock]
    constexpr int kBlock = Shape<TPR, Q>::kBlock, kGroups = Shape<TPR, Q>::kGroups;
    __shared__ row_f32x4 sh[row_reduce_quads<TPR>()];
    __shared__ row_f32x4 join[kGroups > 1 ? kBlock : 1];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int F = a.F;
    const bool odd = F & 3, ragged = F != 4 * TPR * Q;
    const float inv_f = 1.f / static_cast<float>(F);
    const bool post = a.flags & DUALGCN_NORM_POST, sig = a.flags & DUALGCN_GATE_SIGMOID;
    const bool pre = a.dZ != nullptr, block = a.B != nullptr;
    QuadPlace at[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) at[q].set(static_cast<uint32_t>(g) * F, 4 * (l + q * TPR), F);

    row_f32x4 w1[Q], b1[Q], w2[Q], gc[Q];
    auto vector_of_pre = [&]() {
        if (pre) Vector(a.w2, F, 1.f).load<Q, TINY>(at, odd, w2);
    };
    auto vectors_of_post = [&]() {
        if (post) {
            Vector(a.w1, F, 1.f).load<Q, TINY>(at, odd, w1);
            if constexpr (LAYER) Vector(a.b1, F, 0.f).load<Q, TINY>(at, odd, b1);
        }
        if (a.flags & DUALGCN_GATE_FEATURE) {
            Vector(a.gate, F, 1.f).load<Q, TINY>(at, odd, gc);
            if (sig)
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) gc[q][i] = sigmoid(gc[q][i]);
        }
    };
    if constexpr (kHold) {
        vector_of_pre();
        vectors_of_post();
    }

    row_f32x4 acc[kHold ? 4 : 1][Q], acc_gate[Q];
    // slot s's place among the wanted ones
    auto place = [&](int s, int q) { return (__popc(a.want & ((1u << s) - 1u)) * Q + q) * kBlock + static_cast<int>(threadIdx.x); };
    auto add = [&](int s, int q, row_f32x4 v) {
        if constexpr (kHold) acc[s][q] += v;
        else if (a.want >> s & 1) kept[place(s, q)] += v;
    };
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        acc_gate[q] = row_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if constexpr (kHold) acc[s][q] = acc_gate[q];
            else if (a.want >> s & 1) kept[place(s, q)] = acc_gate[q];
        }
    }

    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    int64_t row0 = static_cast<int64_t>(blockIdx.x) * kGroups;
    RowIn<Q, TINY, A, S, G> in, next;
    if constexpr (kAhead) in.load(a, row0, kGroups, g, at);
    for (; row0 < a.n; row0 += step) {
        const int rows = static_cast<int>(min(static_cast<int64_t>(kGroups), a.n - row0));
        const int64_t first = row0 * F, elems = static_cast<int64_t>(rows) * F;
        // the next rows are on their way while these are worked on
        if constexpr (kAhead) next.load(a, row0 + step, kGroups, g, at);
        else in.load(a, row0, kGroups, g, at);
        if constexpr (!kHold) vector_of_pre();

        row_f32x4 x[Q], t[Q], b[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            x[q] = pre ? in.r[q].get(at[q], odd) : row_f32x4{0.f, 0.f, 0.f, 0.f};
            t[q] = pre ? in.z[q].get(at[q], odd) : row_f32x4{0.f, 0.f, 0.f, 0.f};
            b[q] = block ? in.b[q].get(at[q], odd) : row_f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // Behind a row's end, and in rows behind the last, every operand and weight is zero.
        // Both norms' statistics, in two reductions (one for RMS norms); the second takes the
        // sums of t w2 and t w2 (x - m2) along
        if constexpr (LAYER) {
            float m[2] = {sum_of(x), sum_of(b)};
            row_reduce<TPR>(m, AddOp(), sh, turn);
            if (pre) centre(x, m[0] * inv_f, at, ragged);
            if (post) centre(b, m[1] * inv_f, at, ragged);
        }
        row_f32x4 tw[Q];
        float s2 = 0.f, s3 = 0.f;
        if (pre) {
#pragma unroll
            for (int q = 0; q < Q; ++q) tw[q] = t[q] * w2[q];
            s2 = dot_of(tw, x);
            if constexpr (LAYER) s3 = sum_of(tw);
        }
        float st[LAYER ? 4 : 3];
        st[0] = dot_of(x, x);
        st[1] = dot_of(b, b);
        st[2] = s2;
        if constexpr (LAYER) st[3] = s3;
        row_reduce<TPR>(st, AddOp(), sh, turn);

        // the stream's gradient
        row_f32x4 d[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q)
            d[q] = a.dRn ? in.d[q].get(at[q], odd) : row_f32x4{0.f, 0.f, 0.f, 0.f};
        if (pre) {
            const float r2 = __builtin_amdgcn_rsqf(fmaf(st[0], inv_f, a.eps));
            const float mtu = r2 * st[2] * inv_f;
            if constexpr (LAYER) centre(tw, st[3] * inv_f, at, ragged);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                x[q] *= r2;
                add(kW2, q, t[q] * x[q]);
                if constexpr (LAYER) add(kB2, q, t[q]);
                d[q] += r2 * (tw[q] - x[q] * mtu);
            }
        }
        if constexpr (!kHold) vectors_of_post();
        if (a.dR) {
            const __amdgpu_buffer_rsrc_t w = row_window<S>(a.dR, first, elems);
#pragma unroll
            for (int q = 0; q < Q; ++q) store_row_quad<S, TINY>(w, at[q], d[q], odd, a.streaming);
        }
        if (block) {
            const float r1 = post ? __builtin_amdgcn_rsqf(fmaf(st[1], inv_f, a.eps)) : 1.f;
            row_f32x4 v[Q];                            // scale * d * gate, the gradient of post(B)
            float sums[3] = {0.f, 0.f, 0.f};
            const float gnode = sig ? sigmoid(in.gn) : in.gn;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                b[q] *= r1;
                row_f32x4 p = b[q];
                if (post) p = LAYER ? b[q] * w1[q] + b1[q] : b[q] * w1[q];
                d[q] *= a.scale;
                row_f32x4 dg = d[q] * p;               // the gate's gradient
                if (a.flags & (DUALGCN_GATE_FEATURE | DUALGCN_GATE_FULL)) {
                    row_f32x4 gate;
                    if (a.flags & DUALGCN_GATE_FEATURE) {
                        gate = gc[q];
                    } else {
                        gate = in.g[q].get(at[q], odd);
                        if (sig)
#pragma unroll
                            for (int i = 0; i < 4; ++i) gate[i] = sigmoid(gate[i]);
                    }
                    v[q] = d[q] * gate;
                    if (sig) dg *= gate * (1.f - gate);
                } else if (a.flags & DUALGCN_GATE_NODE) {
                    v[q] = d[q] * gnode;
                    if (sig) dg *= gnode * (1.f - gnode);
                } else {
                    v[q] = d[q];
                }
                acc_gate[q] += dg;
                sums[2] += (dg[0] + dg[1]) + (dg[2] + dg[3]);
                if (a.dgate && (a.flags & DUALGCN_GATE_FULL))
                    store_row_quad<G, TINY>(row_window<G>(a.dgate, first, elems), at[q], dg, odd, a.streaming);
            }
            if (post) {
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    add(kW1, q, v[q] * b[q]);
                    if constexpr (LAYER) add(kB1, q, v[q]);
                    v[q] *= w1[q];
                }
                sums[0] = dot_of(v, b);
                if constexpr (LAYER) sums[1] = sum_of(v);
            }
            if (post || (a.flags & DUALGCN_GATE_NODE)) row_reduce<TPR>(sums, AddOp(), sh, turn);
            if (post) {
                const float msu = sums[0] * inv_f, ms = sums[1] * inv_f;
#pragma unroll
                for (int q = 0; q < Q; ++q) v[q] = r1 * (LAYER ? v[q] - ms - b[q] * msu : v[q] - b[q] * msu);
            }
            if (a.dgate && (a.flags & DUALGCN_GATE_NODE) && l == 0 && g < rows)
                static_cast<float *>(a.dgate)[row0 + g] = sums[2];
            if (a.dB) {
                const __amdgpu_buffer_rsrc_t w = row_window<G>(a.dB, first, elems);
#pragma unroll
                for (int q = 0; q < Q; ++q) store_row_quad<G, TINY>(w, at[q], v[q], odd, a.streaming);
            }
        }
        if constexpr (kAhead) in = next;
    }

    // this workgroup's column sums: over its groups in order, then one row of partials a slot
    const int wanted = __popc(a.want);
    int k = 0;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
        if (!(a.want >> s & 1)) continue;              // uniform
        const int64_t p0 = (static_cast<int64_t>(blockIdx.x) * wanted + k++) * F;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            row_f32x4 sum = acc_gate[q];
            if (s < 4) sum = kHold ? acc[kHold ? s & 3 : 0][q] : kept[place(s & 3, q)];
            if constexpr (kGroups > 1) {
                __syncthreads();
                join[threadIdx.x] = sum;
                __syncthreads();
                if (g == 0) {
                    for (int j = 1; j < kGroups; ++j) sum += join[j * TPR + l];
                }
            }
            if (g == 0) store_quad<false>(a.partial, p0 + 4 * (l + q * TPR), at[q].count, sum);
        }
    }
}

// out[slot][c] = the sum over workgroups of the partial sums of column c: 32 threads sum
// consecutive parts in order, in float64, and the parts are added in order.  A pass in parts keeps the sum of those
// before in `before` (float64, [slots][F]; not read by the first, not written by the last).  Measured: 512 partial sums
// of 3 x 128 columns 4.6 us, 256 of 2 x 4,096 6.2 us, bound by the loads' latency: 16 are in flight.
constexpr int kSumSegs = 32;
constexpr int kSumCols = kThreads / kSumSegs;
struct SumOut {
    float *to[kSlots];               // the wanted slots, in order
};
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(const float *__restrict__ partial, int32_t count,
                                                                int32_t wanted, int32_t F, double *before, bool first,
                                                                bool last, SumOut out) {
    __shared__ double sh[kSumSegs][kSumCols];
    const int el = threadIdx.x % kSumCols, seg = threadIdx.x / kSumCols;
    const int c = blockIdx.x * kSumCols + el, slot = blockIdx.y;
    const int per = (count + kSumSegs - 1) / kSumSegs;
    double s = 0.0;
    if (c < F) {
        const int64_t step = static_cast<int64_t>(wanted) * F;
        const float *p = partial + static_cast<int64_t>(slot) * F + c;
        const int b1 = min(count, (seg + 1) * per);
        int b = seg * per;
        for (; b + 16 <= b1; b += 16) {
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = p[(b + j) * step];
#pragma unroll
            for (int j = 0; j < 16; ++j) s += static_cast<double>(v[j]);
        }
        for (; b < b1; ++b) s += static_cast<double>(p[b * step]);
    }
    sh[seg][el] = s;
    __syncthreads();
    if (seg == 0 && c < F) {
        double t = 0.0;
#pragma unroll
        for (int k = 0; k < kSumSegs; ++k) t += sh[k][el];
        double *const b = before + static_cast<int64_t>(slot) * F + c;
        if (!first) t += *b;
        if (last) out.to[slot][c] = static_cast<float>(t);
        else *b = t;
    }
}

// ------------------------------------------------------------------ dispatch

// f(threads of a row, quads of each) for rows of F.  Few threads with two or three quads each
// work on more rows at a time than many with one (a wavefront's lifetime is mostly latency), and
// the fewer places a row leaves empty the better; past that the registers bound the quads.
// Forward of 2^27 elements, us, float32 / bfloat16 (floor 324 / 185): F = 192 (16, 3) 320 / 204, (64, 1)
// 379 / 318; F = 300 (32, 3) 388 / 268, (128, 1) 411 / 402; F = 3,000 (256, 3) 343 / 215, (1024, 1) 498 / 489;
// 65 to 128 features by the rows' lines: F = 96 (16, 2) 335 / 246, (32, 1) 382 / 319; F = 100 445 / 285, 373 / 304.
template <int T, int Q, class Fn>
void shape(Fn f) { f(std::integral_constant<int, T>(), std::integral_constant<int, Q>()); }

template <class Fn>
void with_forward_shape(int32_t F, Fn f) {
    if (F < 4) shape<1, 1>(f);
    else if (F <= 32) shape<8, 1>(f);
    else if (F <= 64) shape<16, 1>(f);
    else if (F <= 128 && F % 32) shape<32, 1>(f);
    else if (F <= 128) shape<16, 2>(f);
    else if (F <= 192) shape<16, 3>(f);
    else if (F <= 256) shape<32, 2>(f);
    else if (F <= 384) shape<32, 3>(f);
    else if (F <= 512) shape<64, 2>(f);
    else if (F <= 768) shape<64, 3>(f);
    else if (F <= 1024) shape<128, 2>(f);
    else if (F <= 1536) shape<128, 3>(f);
    else if (F <= 2048) shape<256, 2>(f);
    else if (F <= 4 * 256 * 3) shape<256, 3>(f);
    else if (F <= 4096) shape<512, 2>(f);
    else if (F <= 6144) shape<512, 3>(f);
    else shape<512, 4>(f);
}

// Float64 sums, bound by the vector unit (conversions, and a row's statistics): the widths by powers of two, so that
// fewer instances do.  2^27 elements, bfloat16 in, float32 Z, RMS and a gate a feature, us: F = 64 272, 128 269, 256 270, 1,024
// 292, 4,096 345; 192 358, 700 398 (float32 sums of all widths, whose stream was not the formula's: 226 to 293).
template <class Fn>
void with_exact_shape(int32_t F, Fn f) {
    if (F < 4) shape<1, 1>(f);
    else if (F <= 32) shape<8, 1>(f);
    else if (F <= 64) shape<8, 2>(f);
    else if (F <= 128) shape<16, 2>(f);
    else if (F <= 256) shape<32, 2>(f);
    else if (F <= 512) shape<64, 2>(f);
    else if (F <= 1024) shape<128, 2>(f);
    else if (F <= 2048) shape<256, 2>(f);
    else if (F <= 4096) shape<512, 2>(f);
    else shape<1024, 2>(f);
}

// The backward pass has about twice the registers a quad.  2^26 elements, us, float32 / bfloat16 (floor
// 278 / 139): F = 256 (64, 1) 285 / 163, (32, 2) 305 / 165; F = 600 (64, 3) 339 / 240, (256, 1) 340 / 307;
// F = 3,000 (256, 3) 335 / 229, (1024, 1) 418 / 330.
template <class Fn>
void with_backward_shape(int32_t F, Fn f) {
    if (F < 4) shape<1, 1>(f);
    else if (F <= 32) shape<8, 1>(f);
    else if (F <= 64) shape<16, 1>(f);
    else if (F <= 128) shape<32, 1>(f);
    else if (F <= 256) shape<64, 1>(f);
    else if (F <= 384) shape<32, 3>(f);
    else if (F <= 512) shape<64, 2>(f);
    else if (F <= 768) shape<64, 3>(f);
    else if (F <= 1024) shape<256, 1>(f);
    else if (F <= 1536) shape<128, 3>(f);
    else if (F <= 2048) shape<256, 2>(f);
    else if (F <= 4 * 256 * 3) shape<256, 3>(f);
    else if (F <= 4096) shape<1024, 1>(f);
    else if (F <= 6144) shape<512, 3>(f);
    else shape<512, 4>(f);
}

// f of up to four truth values as compile-time constants.
template <class Fn>
void with_flags(Fn f) { f(); }
template <class Fn, class... More>
void with_flags(Fn f, bool b, More... more) {
    if (b) with_flags([&](auto... rest) { f(std::true_type(), rest...); }, more...);
    else with_flags([&](auto... rest) { f(std::false_type(), rest...); }, more...);
}

// Workgroups of a backward pass, each with a partial sum of every column.  Its wavefronts have two
// rows in flight each, so two workgroups a CU fill the memory's queues with float32 operands
// (us at 2, 3, 4 a CU: 20,001 x 99 20.7, 20.4, 20.6; 50,000 x 64 20.4, 21.7, 20.4; 30,000 x 256 36.7, 38.6, 36.7; 100,000 x 256 112,
// 121, 123; 60,000 x 512 139, 143, 157; 2^20 x 128 606, 592, 672), and four where every operand is bfloat16 (226, 179, 159).
int backward_blocks(int64_t n, int32_t F, bool all_bf16, int &groups) {
    int per_cu = 1, most = 1;
    with_backward_shape(F, [&](auto tpr, auto quads) {
        constexpr int T = decltype(tpr)::value, Q = decltype(quads)::value;
        groups = Shape<T, Q>::kGroups;
        per_cu = T > 256 ? 1 : T == 128 ? 4 : all_bf16 ? 5 - Q : 2;
        most = kMostBlocks<T>;
    });
    return static_cast<int>(std::min<int64_t>((n + groups - 1) / groups, std::min(most, per_cu * device_cus())));
}

// Outputs the L2s (8 x 4 MiB) would not keep for the next launch are stored past them (us so and without the
// hint, forward of n x 256: 8,192 14.1, 13.5; 65,536 39.5, 51.4; 2^20 636, 668; backward of n x 128: 8,192 26.1, 24.4; 65,536 41.4,
// 43.7; 2^20 592, 609).
bool past_l2(int64_t elems) { return elems * 4 > int64_t{32} << 20; }

}  // namespace

int launch_norm_residual(const dualgcn_norm &p, const void *R, const void *B, void *Rn, void *Z, int32_t n,
                         int32_t F, hipStream_t s) {
    const ForwardArgs a{R, B, p.gate, Rn, Z, p.post_weight, p.post_bias, p.pre_weight, p.pre_bias, n, F,
                        static_cast<float>(p.eps), static_cast<float>(p.scale), p.flags, past_l2(static_cast<int64_t>(n) * F),
                        1.0 / F, p.eps, p.scale};
    const bool exact = B && Z && (p.flags & DUALGCN_STREAM_BF16) && !(p.flags & DUALGCN_OUT_BF16);
    const bool layer = p.flags & DUALGCN_NORM_LAYER, act = p.flags & DUALGCN_IN_BF16;
    auto launch = [&](auto tpr, auto quads, auto exactly, auto l, auto b, auto st) {
        constexpr int T = decltype(tpr)::value, Q = decltype(quads)::value;
        const int64_t need = (static_cast<int64_t>(n) + Shape<T, Q>::kGroups - 1) / Shape<T, Q>::kGroups;
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>(need, kMaxForwardBlocks)));
        hipLaunchKernelGGL((norm_residual_kernel<T, Q, decltype(l)::value, decltype(b)::value, decltype(st)::value, decltype(exactly)::value>),
                           grid, dim3(Shape<T, Q>::kBlock), 0, s, a);
    };
    if (exact)
        with_exact_shape(F, [&](auto tpr, auto quads) {
            with_flags([&](auto l, auto b) { launch(tpr, quads, std::true_type(), l, b, std::true_type()); }, layer, act);
        });
    else
        with_forward_shape(F, [&](auto tpr, auto quads) {
            with_flags([&](auto l, auto b, auto st) { launch(tpr, quads, std::false_type(), l, b, st); }, layer, act,
                       (p.flags & DUALGCN_STREAM_BF16) != 0);
        });
    return hip_status(hipGetLastError());
}

size_t norm_backward_workspace_bytes(int32_t n, int32_t F) {
    int groups = 1, most = 1;
    with_backward_shape(F, [&](auto tpr, auto quads) {
        groups = Shape<decltype(tpr)::value, decltype(quads)::value>::kGroups;
        most = kMostBlocks<decltype(tpr)::value>;
    });
    const int64_t need = (static_cast<int64_t>(n) + groups - 1) / groups;
    // the sums of the parts before, then the partial sums
    return kSlots * static_cast<size_t>(F) * (sizeof(double) + static_cast<size_t>(std::min<int64_t>(need, most)) * sizeof(float));
}

int launch_norm_backward(const dualgcn_norm &p, const void *Rn, const void *B, const void *dZ, const void *dRn,
                         void *dR, void *dB, const dualgcn_norm_grads &g, int32_t n, int32_t F, void *workspace,
                         hipStream_t s) {
    double *const before = static_cast<double *>(workspace);
    BackwardArgs a{Rn, B, p.gate, dZ, dRn, dR, dB, g.gate, p.post_weight, p.post_bias, p.pre_weight,
                   reinterpret_cast<float *>(before + kSlots * static_cast<size_t>(F)), n, F, static_cast<float>(p.eps),
                   static_cast<float>(p.scale), p.flags, 0u,
                   past_l2(static_cast<int64_t>(n) * F)};
    SumOut out{};
    int wanted = 0;
    float *const to[kSlots] = {g.post_weight, g.post_bias, g.pre_weight, g.pre_bias,
                               p.flags & DUALGCN_GATE_FEATURE ? static_cast<float *>(g.gate) : nullptr};
    for (int k = 0; k < kSlots; ++k)
        if (to[k]) {
            a.want |= 1u << k;
            out.to[wanted++] = to[k];
        }
    const bool act = p.flags & DUALGCN_IN_BF16, str = p.flags & DUALGCN_STREAM_BF16, grd = p.flags & DUALGCN_GRAD_BF16;
    int groups = 1;
    const int most = backward_blocks(n, F, act && str && grd, groups);
    // parts of equal numbers of rows, whole steps of all workgroups
    const int64_t step = static_cast<int64_t>(most) * groups, steps = (n + step - 1) / step;
    const int64_t parts = wanted ? (steps + kChain - 1) / kChain : 1, rows = (steps + parts - 1) / parts * step;
    // a pointer moved by `count` elements of four or (bf16) two bytes
    auto moved = [](auto *x, int64_t count, bool bf16) {
        using P = decltype(x);
        return x ? (P)((char *)x + count * (bf16 ? 2 : 4)) : x;
    };
    int st = DUALGCN_OK;
    for (int64_t row = 0; row < n && !st; row += rows) {
        const int64_t at = row * F;
        BackwardArgs part = a;
        part.n = static_cast<int32_t>(std::min(rows, n - row));
        part.Rn = moved(Rn, at, str);
        part.B = moved(B, at, act);
        part.dZ = moved(dZ, at, grd);
        part.dRn = moved(dRn, at, str);
        part.dR = moved(dR, at, str);
        part.dB = moved(dB, at, grd);
        if (p.flags & DUALGCN_GATE_FULL) {
            part.gate = moved(p.gate, at, act);
            part.dgate = moved(g.gate, at, grd);
        } else if (p.flags & DUALGCN_GATE_NODE) {
            part.gate = moved(p.gate, row, false);
            part.dgate = moved(g.gate, row, false);
        }
        const int blocks = static_cast<int>(std::min<int64_t>((part.n + groups - 1) / groups, most));
        with_backward_shape(F, [&](auto tpr, auto quads) {
            constexpr int T = decltype(tpr)::value, Q = decltype(quads)::value;
            const size_t lds = Q > 1 ? sizeof(row_f32x4) * Q * Shape<T, Q>::kBlock * __builtin_popcount(a.want & 15u) : 0;
            with_flags([&](auto layer, auto bf, auto stream, auto grad) {
                const auto kernel = &norm_backward_kernel<T, Q, decltype(layer)::value, decltype(bf)::value,
                                                          decltype(stream)::value, decltype(grad)::value>;
                if (lds > 48 * 1024 && (st = hip_status(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                                             hipFuncAttributeMaxDynamicSharedMemorySize,
                                                                             static_cast<int>(lds)))))
                    return;
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(Shape<T, Q>::kBlock), lds, s, part);
            }, (p.flags & DUALGCN_NORM_LAYER) != 0, act, str, grd);
        });
        if (!st) st = hip_status(hipGetLastError());
        if (st || !wanted) continue;
        hipLaunchKernelGGL(norm_columns_kernel, dim3((F + kSumCols - 1) / kSumCols, wanted), dim3(kThreads), 0, s,
                           a.partial, blocks, wanted, F, before, row == 0, row + rows >= n, out);
        st = hip_status(hipGetLastError());
    }
    return st;
}

}  // namespace dgc
