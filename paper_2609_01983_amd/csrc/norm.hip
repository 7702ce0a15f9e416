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
// Both passes are bound by memory (about one flop a byte): a row stays in the registers of
// its threads from the load to the store, so every operand is read and every output written
// once.  The threads of a row are as many as hold it in few quads: 8 to 64 lanes of a
// wavefront up to 1,024 features, 256 or 512 threads up to 8,192.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 1024;                     // workgroups, hence partial column sums, of a backward pass

// ------------------------------------------------------------------ shared by both directions

template <int TPR, int Q>
struct Shape {
    static constexpr int kBlock = TPR > kThreads ? TPR : kThreads;   // threads of a workgroup
    static constexpr int kGroups = kBlock / TPR;                     // rows it works on at a time
};

// rows whose threads hold more than they have: the row's columns past F are zeros
template <int TPR, int Q>
__device__ __forceinline__ bool is_ragged(int F) {
    return F != 4 * TPR * Q;
}

template <int Q, bool TINY>
__device__ __forceinline__ void load_vector(const float *w, float missing, const QuadPlace (&at)[Q],
                                            bool ragged, row_f32x4 (&out)[Q]) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (w) {
            RawRowQuad<false, TINY> raw;
            raw.load(w, 0, at[q]);
            out[q] = raw.get(at[q], ragged);
        } else {
            out[q] = row_f32x4{missing, missing, missing, missing};
        }
    }
}

// x - mean on the row's columns, zeros behind them
template <int Q>
__device__ __forceinline__ void centre(row_f32x4 (&x)[Q], float mean, const QuadPlace (&at)[Q], bool ragged) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = x[q][i] - mean;
            x[q][i] = ragged && i >= at[q].count ? 0.f : c;
        }
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
template <int TPR, int Q>
__device__ __forceinline__ void normalise(row_f32x4 (&x)[Q], const QuadPlace (&at)[Q], bool ragged, bool layer,
                                          float inv_f, float eps, float *sh, int &turn) {
    if (layer) {
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

// ------------------------------------------------------------------ forward

struct ForwardArgs {
    const void *R, *B, *gate;
    void *Rn, *Z;
    const float *w1, *b1, *w2, *b2;
    int32_t n, F;
    float eps, scale;
    uint32_t flags;
};

// A: B and a full gate are bfloat16; S: the stream is.
template <int TPR, int Q, bool A, bool S>
__global__ __launch_bounds__((Shape<TPR, Q>::kBlock)) void norm_residual_kernel(ForwardArgs a) {
    constexpr bool TINY = TPR == 1;
    constexpr bool kHold = Q <= 2;                   // the weights stay in registers over the rows
    constexpr int kGroups = Shape<TPR, Q>::kGroups;
    __shared__ float sh[row_reduce_floats<TPR>()];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int F = a.F;
    const bool ragged = is_ragged<TPR, Q>(F);
    const float inv_f = 1.f / static_cast<float>(F);
    const bool layer = a.flags & DUALGCN_NORM_LAYER, post = a.flags & DUALGCN_NORM_POST;
    const bool sig = a.flags & DUALGCN_GATE_SIGMOID;
    QuadPlace at[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) at[q].set(4 * (l + q * TPR), F);

    row_f32x4 w1[Q], b1[Q], w2[Q], b2[Q], gc[Q];
    auto vectors = [&]() {
        if (post) {
            load_vector<Q, TINY>(a.w1, 1.f, at, ragged, w1);
            load_vector<Q, TINY>(a.b1, 0.f, at, ragged, b1);
        }
        if (a.Z) {
            load_vector<Q, TINY>(a.w2, 1.f, at, ragged, w2);
            load_vector<Q, TINY>(a.b2, 0.f, at, ragged, b2);
        }
        if (a.flags & DUALGCN_GATE_FEATURE) {
            load_vector<Q, TINY>(static_cast<const float *>(a.gate), 1.f, at, ragged, gc);
            if (sig)
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) gc[q][i] = sigmoid(gc[q][i]);
        }
    };
    if constexpr (kHold) vectors();

    for (int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + g; row < a.n;
         row += static_cast<int64_t>(gridDim.x) * kGroups) {
        const int64_t r0 = row * F;
        RawRowQuad<S, TINY> rr[Q];
        RawRowQuad<A, TINY> rb[Q], rg[Q];
        float gn = 1.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) rr[q].load(a.R, r0, at[q]);
        if (a.B) {
#pragma unroll
            for (int q = 0; q < Q; ++q) rb[q].load(a.B, r0, at[q]);
            if (a.flags & DUALGCN_GATE_FULL)
#pragma unroll
                for (int q = 0; q < Q; ++q) rg[q].load(a.gate, r0, at[q]);
            if (a.flags & DUALGCN_GATE_NODE) gn = static_cast<const float *>(a.gate)[row];
        }
        if constexpr (!kHold) vectors();
        row_f32x4 x[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) x[q] = rr[q].get(at[q], ragged);
        if (a.B) {
            row_f32x4 v[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) v[q] = rb[q].get(at[q], ragged);
            if (post) {
                normalise<TPR, Q>(v, at, ragged, layer, inv_f, a.eps, sh, turn);
#pragma unroll
                for (int q = 0; q < Q; ++q) v[q] = v[q] * w1[q] + b1[q];
            }
            if (a.flags & DUALGCN_GATE_FEATURE) {
#pragma unroll
                for (int q = 0; q < Q; ++q) v[q] *= gc[q];
            }
            if (a.flags & DUALGCN_GATE_FULL) {
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    row_f32x4 gate = rg[q].get(at[q], ragged);
                    if (sig)
#pragma unroll
                        for (int i = 0; i < 4; ++i) gate[i] = sigmoid(gate[i]);
                    v[q] *= gate;
                }
            }
            const float scale = a.scale * (sig && (a.flags & DUALGCN_GATE_NODE) ? sigmoid(gn) : gn);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[q][i] = fmaf(scale, v[q][i], x[q][i]);
                    // the next norm (and the backward pass) take the stream as it is stored
                    if constexpr (S) x[q][i] = through_bf16(x[q][i]);
                    if (ragged && i >= at[q].count) x[q][i] = 0.f;     // b1 may have left the row's end
                }
                store_quad<S>(a.Rn, r0 + 4 * (l + q * TPR), at[q].count, x[q]);
            }
        }
        if (a.Z) {
            normalise<TPR, Q>(x, at, ragged, layer, inv_f, a.eps, sh, turn);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const row_f32x4 z = x[q] * w2[q] + b2[q];
                if (a.flags & DUALGCN_OUT_BF16) store_quad<true>(a.Z, r0 + 4 * (l + q * TPR), at[q].count, z);
                else store_quad<false>(a.Z, r0 + 4 * (l + q * TPR), at[q].count, z);
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
};

// A: B and a full gate are bfloat16; S: the stream and its gradients are; G: dZ, dB and a full
// gate's gradient are.
template <int TPR, int Q, bool A, bool S, bool G>
__global__ __launch_bounds__((Shape<TPR, Q>::kBlock)) void norm_backward_kernel(BackwardArgs a) {
    constexpr bool TINY = TPR == 1;
    constexpr bool kHold = Q <= 1;
    constexpr int kBlock = Shape<TPR, Q>::kBlock, kGroups = Shape<TPR, Q>::kGroups;
    __shared__ float sh[row_reduce_floats<TPR>()];
    __shared__ row_f32x4 join[kGroups > 1 ? kBlock : 1];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int F = a.F;
    const bool ragged = is_ragged<TPR, Q>(F);
    const float inv_f = 1.f / static_cast<float>(F);
    const bool layer = a.flags & DUALGCN_NORM_LAYER, post = a.flags & DUALGCN_NORM_POST;
    const bool sig = a.flags & DUALGCN_GATE_SIGMOID;
    const bool pre = a.dZ != nullptr, block = a.B != nullptr;
    QuadPlace at[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) at[q].set(4 * (l + q * TPR), F);

    row_f32x4 w1[Q], b1[Q], w2[Q], gc[Q];
    auto vectors = [&]() {
        if (post) {
            load_vector<Q, TINY>(a.w1, 1.f, at, ragged, w1);
            load_vector<Q, TINY>(a.b1, 0.f, at, ragged, b1);
        }
        if (pre) load_vector<Q, TINY>(a.w2, 1.f, at, ragged, w2);
        if (a.flags & DUALGCN_GATE_FEATURE) {
            load_vector<Q, TINY>(static_cast<const float *>(a.gate), 1.f, at, ragged, gc);
            if (sig)
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) gc[q][i] = sigmoid(gc[q][i]);
        }
    };
    if constexpr (kHold) vectors();

    row_f32x4 acc[kSlots][Q];
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
#pragma unroll
        for (int q = 0; q < Q; ++q) acc[s][q] = row_f32x4{0.f, 0.f, 0.f, 0.f};

    for (int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + g; row < a.n;
         row += static_cast<int64_t>(gridDim.x) * kGroups) {
        const int64_t r0 = row * F;
        RawRowQuad<S, TINY> raw_r[Q], raw_d[Q];
        RawRowQuad<G, TINY> raw_z[Q];
        RawRowQuad<A, TINY> raw_b[Q], raw_g[Q];
        float gn = 1.f;
        if (pre) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                raw_r[q].load(a.Rn, r0, at[q]);
                raw_z[q].load(a.dZ, r0, at[q]);
            }
        }
        if (a.dRn) {
#pragma unroll
            for (int q = 0; q < Q; ++q) raw_d[q].load(a.dRn, r0, at[q]);
        }
        if (block) {
#pragma unroll
            for (int q = 0; q < Q; ++q) raw_b[q].load(a.B, r0, at[q]);
            if (a.flags & DUALGCN_GATE_FULL)
#pragma unroll
                for (int q = 0; q < Q; ++q) raw_g[q].load(a.gate, r0, at[q]);
            if (a.flags & DUALGCN_GATE_NODE) gn = static_cast<const float *>(a.gate)[row];
        }
        if constexpr (!kHold) vectors();

        row_f32x4 x[Q], t[Q], b[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            x[q] = pre ? raw_r[q].get(at[q], ragged) : row_f32x4{0.f, 0.f, 0.f, 0.f};
            t[q] = pre ? raw_z[q].get(at[q], ragged) : row_f32x4{0.f, 0.f, 0.f, 0.f};
            b[q] = block ? raw_b[q].get(at[q], ragged) : row_f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // both norms' statistics, in two reductions (one for RMS norms); the second takes the
        // sums of t w2 and t w2 (x - m2) along
        if (layer) {
            float m[2] = {sum_of(x), sum_of(b)};
            row_reduce<TPR>(m, AddOp(), sh, turn);
            if (pre) centre(x, m[0] * inv_f, at, ragged);
            if (post) centre(b, m[1] * inv_f, at, ragged);
        }
        float st[4] = {dot_of(x, x), dot_of(b, b), 0.f, 0.f};
        row_f32x4 tw[Q];
        if (pre) {
#pragma unroll
            for (int q = 0; q < Q; ++q) tw[q] = t[q] * w2[q];
            st[2] = sum_of(tw);
            st[3] = dot_of(tw, x);
        }
        row_reduce<TPR>(st, AddOp(), sh, turn);

        // the stream's gradient
        row_f32x4 d[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q)
            d[q] = a.dRn ? raw_d[q].get(at[q], ragged) : row_f32x4{0.f, 0.f, 0.f, 0.f};
        if (pre) {
            const float r2 = __builtin_amdgcn_rsqf(fmaf(st[0], inv_f, a.eps));
            const float mt = layer ? st[2] * inv_f : 0.f;
            const float mtu = r2 * st[3] * inv_f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                x[q] *= r2;
                acc[kW2][q] += t[q] * x[q];
                acc[kB2][q] += t[q];
                d[q] += r2 * (tw[q] - mt - x[q] * mtu);
            }
        }
        if (a.dR) {
#pragma unroll
            for (int q = 0; q < Q; ++q) store_quad<S>(a.dR, r0 + 4 * (l + q * TPR), at[q].count, d[q]);
        }
        if (block) {
            const float r1 = post ? __builtin_amdgcn_rsqf(fmaf(st[1], inv_f, a.eps)) : 1.f;
            row_f32x4 v[Q];                            // scale * d * gate, the gradient of post(B)
            float sums[3] = {0.f, 0.f, 0.f};
            const float gnode = a.flags & DUALGCN_GATE_NODE ? (sig ? sigmoid(gn) : gn) : 1.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                b[q] *= r1;
                const row_f32x4 p = post ? b[q] * w1[q] + b1[q] : b[q];
                row_f32x4 gate = row_f32x4{gnode, gnode, gnode, gnode};
                if (a.flags & DUALGCN_GATE_FEATURE) gate = gc[q];
                if (a.flags & DUALGCN_GATE_FULL) {
                    gate = raw_g[q].get(at[q], ragged);
                    if (sig)
#pragma unroll
                        for (int i = 0; i < 4; ++i) gate[i] = sigmoid(gate[i]);
                }
                d[q] *= a.scale;
                v[q] = d[q] * gate;
                row_f32x4 dg = d[q] * p;               // the gate's gradient
                if (sig) dg *= gate * (1.f - gate);
                if (ragged) {                          // p and gate are not zero behind the row's end
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i >= at[q].count) {
                            dg[i] = 0.f;
                            v[q][i] = 0.f;
                        }
                    }
                }
                acc[kGate][q] += dg;
                sums[2] += (dg[0] + dg[1]) + (dg[2] + dg[3]);
                if (a.dgate && (a.flags & DUALGCN_GATE_FULL))
                    store_quad<G>(a.dgate, r0 + 4 * (l + q * TPR), at[q].count, dg);
            }
            if (post) {
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    acc[kW1][q] += v[q] * b[q];
                    acc[kB1][q] += v[q];
                    v[q] *= w1[q];
                }
                sums[0] = sum_of(v);
                sums[1] = dot_of(v, b);
            }
            if (post || (a.flags & DUALGCN_GATE_NODE)) row_reduce<TPR>(sums, AddOp(), sh, turn);
            if (post) {
                const float ms = layer ? sums[0] * inv_f : 0.f, msu = sums[1] * inv_f;
#pragma unroll
                for (int q = 0; q < Q; ++q) v[q] = r1 * (v[q] - ms - b[q] * msu);
            }
            if (a.dgate && (a.flags & DUALGCN_GATE_NODE) && l == 0) static_cast<float *>(a.dgate)[row] = sums[2];
            if (a.dB) {
#pragma unroll
                for (int q = 0; q < Q; ++q) store_quad<G>(a.dB, r0 + 4 * (l + q * TPR), at[q].count, v[q]);
            }
        }
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
            row_f32x4 sum = acc[s][q];
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

// out[slot][c] = the sum over workgroups of the partial sums of column c: eight threads sum
// consecutive eighths in order, in float64, and the eighths are added in order.
constexpr int kSumSegs = 8;
constexpr int kSumCols = kThreads / kSumSegs;
struct SumOut {
    float *to[kSlots];               // the wanted slots, in order
};
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(const float *__restrict__ partial, int32_t count,
                                                                int32_t wanted, int32_t F, SumOut out) {
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
        out.to[slot][c] = static_cast<float>(t);
    }
}

// ------------------------------------------------------------------ dispatch

// Rows a workgroup works on at a time (the groups of launch_norm_* for this width).
int rows_per_step(int32_t F) {
    return F < 4 ? kThreads : F <= 32 ? kThreads / 8 : F <= 64 ? kThreads / 16 : F <= 128 ? kThreads / 32
                                                     : F <= 512 ? kThreads / 64 : 1;
}

int backward_blocks(int32_t n, int32_t F) {
    const int64_t need = (static_cast<int64_t>(n) + rows_per_step(F) - 1) / rows_per_step(F);
    return static_cast<int>(std::min<int64_t>(need, kMaxBlocks));
}

template <int TPR, int Q>
void launch_forward(const ForwardArgs &a, bool act, bool stream, hipStream_t s) {
    const int64_t need = (static_cast<int64_t>(a.n) + Shape<TPR, Q>::kGroups - 1) / Shape<TPR, Q>::kGroups;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(need, static_cast<int64_t>(device_cus()) * 8)));
    const dim3 block(Shape<TPR, Q>::kBlock);
    if (act && stream) hipLaunchKernelGGL((norm_residual_kernel<TPR, Q, true, true>), grid, block, 0, s, a);
    else if (act) hipLaunchKernelGGL((norm_residual_kernel<TPR, Q, true, false>), grid, block, 0, s, a);
    else if (stream) hipLaunchKernelGGL((norm_residual_kernel<TPR, Q, false, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((norm_residual_kernel<TPR, Q, false, false>), grid, block, 0, s, a);
}

template <int TPR, int Q, bool A, bool S>
void launch_backward_g(const BackwardArgs &a, bool grad, dim3 grid, hipStream_t s) {
    const dim3 block(Shape<TPR, Q>::kBlock);
    if (grad) hipLaunchKernelGGL((norm_backward_kernel<TPR, Q, A, S, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((norm_backward_kernel<TPR, Q, A, S, false>), grid, block, 0, s, a);
}

template <int TPR, int Q>
void launch_backward(const BackwardArgs &a, bool act, bool stream, bool grad, int blocks, hipStream_t s) {
    const dim3 grid(static_cast<unsigned>(blocks));
    if (act && stream) launch_backward_g<TPR, Q, true, true>(a, grad, grid, s);
    else if (act) launch_backward_g<TPR, Q, true, false>(a, grad, grid, s);
    else if (stream) launch_backward_g<TPR, Q, false, true>(a, grad, grid, s);
    else launch_backward_g<TPR, Q, false, false>(a, grad, grid, s);
}

}  // namespace

int launch_norm_residual(const dualgcn_norm &p, const void *R, const void *B, void *Rn, void *Z, int32_t n,
                         int32_t F, hipStream_t s) {
    const ForwardArgs a{R, B, p.gate, Rn, Z, p.post_weight, p.post_bias, p.pre_weight, p.pre_bias, n, F,
                        p.eps, p.scale, p.flags};
    const bool act = p.flags & DUALGCN_IN_BF16, stream = p.flags & DUALGCN_STREAM_BF16;
    if (F < 4) launch_forward<1, 1>(a, act, stream, s);
    else if (F <= 32) launch_forward<8, 1>(a, act, stream, s);
    else if (F <= 64) launch_forward<16, 1>(a, act, stream, s);
    else if (F <= 128) launch_forward<32, 1>(a, act, stream, s);
    else if (F <= 256) launch_forward<64, 1>(a, act, stream, s);
    else if (F <= 512) launch_forward<64, 2>(a, act, stream, s);
    else if (F <= 1024) launch_forward<256, 1>(a, act, stream, s);
    else if (F <= 2048) launch_forward<256, 2>(a, act, stream, s);
    else if (F <= 4096) launch_forward<512, 2>(a, act, stream, s);
    else launch_forward<1024, 2>(a, act, stream, s);
    return hip_status(hipGetLastError());
}

size_t norm_backward_workspace_bytes(int32_t n, int32_t F) {
    return static_cast<size_t>(backward_blocks(n, F)) * kSlots * F * sizeof(float);
}

int launch_norm_backward(const dualgcn_norm &p, const void *Rn, const void *B, const void *dZ, const void *dRn,
                         void *dR, void *dB, const dualgcn_norm_grads &g, int32_t n, int32_t F, void *workspace,
                         hipStream_t s) {
    BackwardArgs a{Rn, B, p.gate, dZ, dRn, dR, dB, g.gate, p.post_weight, p.post_bias, p.pre_weight,
                   static_cast<float *>(workspace), n, F, p.eps, p.scale, p.flags, 0u};
    SumOut out{};
    int wanted = 0;
    float *const to[kSlots] = {g.post_weight, g.post_bias, g.pre_weight, g.pre_bias,
                               p.flags & DUALGCN_GATE_FEATURE ? static_cast<float *>(g.gate) : nullptr};
    for (int k = 0; k < kSlots; ++k)
        if (to[k]) {
            a.want |= 1u << k;
            out.to[wanted++] = to[k];
        }
    const bool act = p.flags & DUALGCN_IN_BF16, stream = p.flags & DUALGCN_STREAM_BF16;
    const bool grad = p.flags & DUALGCN_GRAD_BF16;
    const int blocks = backward_blocks(n, F);
    if (F < 4) launch_backward<1, 1>(a, act, stream, grad, blocks, s);
    else if (F <= 32) launch_backward<8, 1>(a, act, stream, grad, blocks, s);
    else if (F <= 64) launch_backward<16, 1>(a, act, stream, grad, blocks, s);
    else if (F <= 128) launch_backward<32, 1>(a, act, stream, grad, blocks, s);
    else if (F <= 256) launch_backward<64, 1>(a, act, stream, grad, blocks, s);
    else if (F <= 512) launch_backward<64, 2>(a, act, stream, grad, blocks, s);
    else if (F <= 1024) launch_backward<256, 1>(a, act, stream, grad, blocks, s);
    else if (F <= 2048) launch_backward<256, 2>(a, act, stream, grad, blocks, s);
    else if (F <= 4096) launch_backward<512, 2>(a, act, stream, grad, blocks, s);
    else launch_backward<1024, 2>(a, act, stream, grad, blocks, s);
    const int st = hip_status(hipGetLastError());
    if (st || !wanted) return st;
    hipLaunchKernelGGL(norm_columns_kernel, dim3((F + kSumCols - 1) / kSumCols, wanted), dim3(kThreads), 0, s,
                       a.partial, blocks, wanted, F, out);
    return hip_status(hipGetLastError());
}

}  // namespace dgc
