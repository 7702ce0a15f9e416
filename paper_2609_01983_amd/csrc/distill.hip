// Distillation of a node classifier from a teacher's top logits, with the labels' cross-entropy
// beside it: the loss and its gradient in one pass over the student's logits.
//
// Row v keeps K entries (id, t) of its teacher; an entry counts if its id is in [0, C) and its
// logit is not -inf.  With Q = softmax(Y_v / T) over all C classes and
//   p_k = exp(t_k / T) / sum over the row's entries      (the teacher on what it kept)
// the row adds, if it has an entry,  soft T^2 sum_k p_k (log p_k - log Q[id_k])  to the loss and
//   soft T (Q_j - P_j),  P_j = sum of the p_k with id_k = j,   to G_j,
// and, if its label is in [0, C), hard (-log softmax(Y_v)[label]) and hard (softmax(Y_v)_j - e_j).
//
// Bound by memory: Y is read once and G written once, about 30 operations an element.  Exponentials
// are base 2, exp2((y - m) a) with a = log2(e) / T: the difference first, so that a row whose
// every logit is the type's lowest value is still a uniform distribution.
//
// P is scattered to LDS by an exchange for each entry: the value that comes back is zero unless
// another entry has the same id, and such a row is summed again entry by entry in order, so that
// the result does not depend on timing.  The cross term of the loss, sum_j P_j (y_j - m), is
// formed where the gradient reads P, with no gathers from Y.
#include "rows.h"

#include <algorithm>
#include <cfloat>

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 8192;                     // workgroups, hence partial sums of the loss
constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.69314718055994530942;

struct Args {
    const void *Y, *teacher;
    const int32_t *ids, *labels;
    void *G;
    double *partial;                 // [workgroups][2]: soft and hard sums, in nats
    float *stats;                    // of split rows: [n][splits][3]
    int32_t n, C, K;
    float temp_a;                    // log2(e) / T
    float soft, hard;                // coefficients of the gradient: soft T, hard
    bool g_bf16, streaming;          // G is bfloat16; G is past the L2s
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <bool TBF>
__device__ __forceinline__ float teacher_at(const void *t, int64_t at) {
    if constexpr (TBF) return bf16_to_float(static_cast<const unsigned short *>(t)[at]);
    else return static_cast<const float *>(t)[at];
}

// Lanes of one row up to a wavefront: LDS operations of a wavefront are done in order, so only
// the compiler has to be told; above that the workgroup meets.
template <int TPR>
__device__ __forceinline__ void row_sync() {
    if constexpr (TPR > 64) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// A row's entries: the first kHeld of each thread in registers, any others read again from the
// cache on each use.  Threads of the row take entries l, l + TPR, ...
template <int TPR, bool TBF>
struct Entries {
    static constexpr int kHeld = 2;
    const int32_t *ids;
    const void *teacher;
    int64_t at;
    int K, C, l;
    int id[kHeld];
    float t[kHeld];                  // the logit, -inf: none; its exponential from local_sum on, 0: none
    float m, inv;                    // largest logit; 1 / sum of the exponentials
    float entropy;                   // this thread's share of sum p log2(p sum)
    bool taught;

    // no entry: class -1 and logit -inf
    __device__ __forceinline__ void fetch(int64_t k, int &i, float &x) const {
        i = ids[at + k];
        x = teacher_at<TBF>(teacher, at + k);
        if (i < 0 || i >= C || x == -INFINITY) {
            i = -1;
            x = -INFINITY;
        }
    }
    __device__ __forceinline__ void load(const Args &a, int64_t row, int lane) {
        ids = a.ids;
        teacher = a.teacher;
        at = row * a.K;
        K = row < a.n ? a.K : 0;                         // a row behind the last has no entries
        C = a.C;
        l = lane;
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            id[h] = -1;
            t[h] = -INFINITY;
            if (l + h * TPR < K) fetch(l + h * TPR, id[h], t[h]);
        }
    }
    // f of the entries that are not held: their classes and logits
    template <class F>
    __device__ __forceinline__ void others(F f) const {
        for (int k = l + kHeld * TPR; k < K; k += TPR) {
            int i;
            float x;
            fetch(k, i, x);
            f(i, x);
        }
    }
    // f of the classes and exponentials (0: none) of all entries, after local_sum
    template <class F>
    __device__ __forceinline__ void each(float a, F f) const {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) f(id[h], t[h]);
        others([&](int i, float x) { f(i, exponential(x, a)); });
    }
    __device__ __forceinline__ float exponential(float x, float a) const {
        return x == -INFINITY ? 0.f : exp2_fast((x - m) * a);
    }

    // The row's largest logit and the sum of its exponentials, in two steps around the reductions that
    // the row's own logits need too: v[0] and v[1] join `max`, v[0] joins `sum`.
    __device__ __forceinline__ void local_max(float *v) const {
        v[0] = -INFINITY;
        v[1] = 0.f;                                      // does an entry count? (NaN does)
        auto one = [&](int, float x) {
            v[0] = fmaxf(v[0], x);
            if (!(x == -INFINITY)) v[1] = 1.f;
        };
#pragma unroll
        for (int h = 0; h < kHeld; ++h) one(id[h], t[h]);
        others(one);
    }
    __device__ __forceinline__ void local_sum(const float *max, float a, float *v) {
        m = max[0];
        taught = max[1] > 0.f;
        v[0] = 0.f;
        entropy = 0.f;
        auto one = [&](float x) {
            const float e = exponential(x, a);
            v[0] += e;
            entropy = fmaf(e, e == 0.f ? 0.f : (x - m) * a, entropy);    // no 0 * infinity
            return e;
        };
#pragma unroll
        for (int h = 0; h < kHeld; ++h) t[h] = one(t[h]);
        others([&](int, float x) { one(x); });
    }
    __device__ __forceinline__ void have(float sum) {
        inv = __builtin_amdgcn_rcpf(sum);
        entropy *= inv;
    }

    // P of the classes [c0, c1) into tile[id - c0] (zeros before); clear() undoes it.  have() first.
    __device__ __forceinline__ void scatter(float *tile, int c0, int c1, float a, int *flag) const {
        bool twice = false;
        each(a, [&](int i, float e) {
            const float v = e * inv;
            if (!(v == 0.f) && static_cast<uint32_t>(i - c0) < static_cast<uint32_t>(c1 - c0))
                twice |= __hip_atomic_exchange(tile + (i - c0), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) != 0.f;
        });
        if constexpr (TPR > 64) {
            // the flag is set again only after the next row's reductions, which all threads reach
            // after they have read it here
            if (twice) *flag = 1;
            __syncthreads();
            twice = *flag != 0;
        } else {
            row_sync<TPR>();
            const uint64_t all = __ballot(twice);
            const int first = (threadIdx.x & 63) / TPR * TPR;
            twice = (TPR == 64 ? all : all >> first & ((uint64_t{1} << (TPR & 63)) - 1)) != 0;
        }
        if (twice) {                                     // the same for all threads of the row
            clear(tile, c0, c1);
            row_sync<TPR>();
            if (l == 0) {
                for (int k = 0; k < K; ++k) {
                    int i;
                    float x;
                    fetch(k, i, x);
                    if (i >= c0 && i < c1) tile[i - c0] += exponential(x, a) * inv;
                }
                if constexpr (TPR > 64) *flag = 0;
            }
            row_sync<TPR>();
        }
    }
    __device__ __forceinline__ void clear(float *tile, int c0, int c1) const {
        // whatever the p: a row with an infinity or a NaN has NaN where the exponential is 0
        auto one = [&](int i) {
            if (static_cast<uint32_t>(i - c0) < static_cast<uint32_t>(c1 - c0)) tile[i - c0] = 0.f;
        };
#pragma unroll
        for (int h = 0; h < kHeld; ++h) one(id[h]);
        others([&](int i, float) { one(i); });
    }
};

// Has a quad of P anything?  (P is never negative, and a NaN's bits are not zero.)
__device__ __forceinline__ bool some(row_f32x4 P) {
    return (__float_as_uint(P[0]) | __float_as_uint(P[1]) | __float_as_uint(P[2]) | __float_as_uint(P[3])) != 0;
}

// A thread's sums of the loss over its rows, joined over the workgroup in a fixed order.
template <int BLOCK>
__device__ __forceinline__ void write_partial(double soft, double hard, double *partial) {
    __shared__ double sh[2][BLOCK / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        soft += __shfl_xor(soft, o);
        hard += __shfl_xor(hard, o);
    }
    if ((threadIdx.x & 63) == 0) {
        sh[0][threadIdx.x >> 6] = soft;
        sh[1][threadIdx.x >> 6] = hard;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        double s = 0.0;
        for (int w = 0; w < BLOCK / 64; ++w) s += sh[threadIdx.x][w];
        partial[threadIdx.x] = s;
    }
}

// Rows whose logits stay in the registers of their TPR threads, Q quads each.  YBF, TBF: the
// logits, the teacher's are bfloat16.  Measured: 2^22 x 64 with 16 entries a row, T = 4 and labels, 2.7 GB in 526 us a call
// (536 to 556 in a trace), 5.1 TB/s; 30,007 x 47 with 8 entries 13 MB in 7.4 us.  Short rows are bound by the vector unit as much
// as by memory: two exponentials a logit, three reductions a row and the entries' own work.
template <int TPR, int Q, bool YBF, bool TBF>
__global__ __launch_bounds__((TPR > 64 ? TPR : kThreads)) void distill_rows_kernel(Args a) {
    constexpr bool TINY = TPR == 1;
    constexpr int kBlock = TPR > 64 ? TPR : kThreads, kGroups = kBlock / TPR;
    __shared__ row_f32x4 sh[row_reduce_quads<TPR>()];
    __shared__ row_f32x4 tiles[kGroups][TPR * Q];
    __shared__ int flag;
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int C = a.C;
    const bool odd = C & 3, ragged = C != 4 * TPR * Q;
    float *tile = reinterpret_cast<float *>(tiles[g]);
    QuadPlace at[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        at[q].set(static_cast<uint32_t>(g) * C, 4 * (l + q * TPR), C);
        tiles[g][l + q * TPR] = row_f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (threadIdx.x == 0) flag = 0;
    row_sync<TPR>();
    const bool same = a.temp_a == kLog2e;                // T = 1: one softmax serves both
    double soft = 0.0, hard = 0.0;

    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kGroups; row0 < a.n;
         row0 += static_cast<int64_t>(gridDim.x) * kGroups) {
        const int64_t row = row0 + g;
        const int64_t elems = min(static_cast<int64_t>(kGroups), a.n - row0) * C;
        const __amdgpu_buffer_rsrc_t wy = row_window<YBF>(a.Y, row0 * C, elems);
        RawRowQuad<YBF, TINY> raw[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) raw[q].load(wy, at[q].at, at[q].count);
        Entries<TPR, TBF> en;
        en.load(a, row, l);
        const int lab = a.labels && row < a.n ? a.labels[row] : -1;
        const bool labeled = lab >= 0 && lab < C;
        float top[3];
        en.local_max(top);
        top[2] = -FLT_MAX;                               // all of the row -inf: the sums are 0, G NaN
        row_f32x4 y[Q], o[Q], e1[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            y[q] = raw[q].get(at[q], odd);
            if (ragged)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= at[q].count) y[q][i] = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) top[2] = fmaxf(top[2], y[q][i]);
        }
        row_reduce<TPR>(top, MaxOp(), sh, turn);
        float s[3];                                      // the entries', at T, at 1
        en.local_sum(top, a.temp_a, s);
        s[1] = s[2] = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[q][i] -= top[2];
                o[q][i] = exp2_fast(y[q][i] * a.temp_a);
                s[1] += o[q][i];
            }
        if (labeled && !same)
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e1[q][i] = exp2_fast(y[q][i] * kLog2e);
                    s[2] += e1[q][i];
                }
        row_reduce<TPR>(s, AddOp(), sh, turn);
        if (same) s[2] = s[1];
        const float ct = en.taught ? a.soft : 0.f;
        // at T = 1 the label's share of the softmax joins the teacher's
        const float it = (same && labeled ? ct + a.hard : ct) * __builtin_amdgcn_rcpf(s[1]);
#pragma unroll
        for (int q = 0; q < Q; ++q) o[q] *= it;
        float loss_s = 0.f, loss_h = 0.f;                // this thread's share, in powers of two
        if (labeled) {
            const float i1 = a.hard * __builtin_amdgcn_rcpf(s[2]);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                if (!same) o[q] += e1[q] * i1;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (4 * (l + q * TPR) + i == lab) {
                        o[q][i] -= a.hard;
                        loss_h = y[q][i];
                    }
            }
        }
        if (en.taught) {
            en.have(s[0]);
            en.scatter(tile, 0, C, a.temp_a, &flag);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const row_f32x4 P = tiles[g][l + q * TPR];
                if (some(P)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // no 0 * infinity where the class has no P
                        loss_s = fmaf(P[i], P[i] == 0.f ? 0.f : y[q][i], loss_s);
                        o[q][i] = fmaf(-ct, P[i], o[q][i]);
                    }
                }
            }
            row_sync<TPR>();                             // P is read before it is cleared
            en.clear(tile, 0, C);
            if constexpr (TPR <= 64) row_sync<TPR>();    // else the next row's reductions come between
            soft += en.entropy - static_cast<double>(a.temp_a) * loss_s;
            if (l == 0) soft += __builtin_amdgcn_logf(s[1]) - __builtin_amdgcn_logf(s[0]);
        }
        if (labeled) {
            hard -= static_cast<double>(kLog2e) * loss_h;
            if (l == 0) hard += __builtin_amdgcn_logf(s[2]);
        }
        if (!en.taught && !labeled)                      // zeros, whatever the logits
#pragma unroll
            for (int q = 0; q < Q; ++q) o[q] = row_f32x4{0.f, 0.f, 0.f, 0.f};
        if (a.g_bf16) {
            const __amdgpu_buffer_rsrc_t w = row_window<true>(a.G, row0 * C, elems);
#pragma unroll
            for (int q = 0; q < Q; ++q) store_row_quad<true, TINY>(w, at[q], o[q], odd, a.streaming);
        } else {
            const __amdgpu_buffer_rsrc_t w = row_window<false>(a.G, row0 * C, elems);
#pragma unroll
            for (int q = 0; q < Q; ++q) store_row_quad<false, TINY>(w, at[q], o[q], odd, a.streaming);
        }
    }
    write_partial<kBlock>(soft, hard, a.partial + 2 * static_cast<int64_t>(blockIdx.x));
}

// ------------------------------------------------------------------ long rows
//
// A workgroup takes a row, and its P is scattered to LDS piece by piece.  Up to 32,768 logits stay in
// the workgroup's registers as they are stored, so that they are read once.  Longer rows are swept twice: a running
// maximum and sums, then the gradient.  Where there are few rows, `splits` workgroups share each: a
// first launch leaves their maxima and sums in `stats`, the second joins them.
constexpr int kSweep = 512;                          // threads of a sweep
constexpr int kSweepQ = 8;                           // quads a thread and piece
constexpr int kHeldQ = 4;                            // the same where the row is held

struct RowStats {
    float m, st, s1;
};

// Quad q of this thread in the piece at class c, none from class c1 on (a whole number of quads, or
// the row's end).  Behind the row's end the window needs no compare.  ODD: C is no multiple of four.
template <int THREADS, bool ODD>
__device__ __forceinline__ QuadPlace place(int thread, int c, int q, int c1, int C) {
    const int first = c + 4 * (thread + q * THREADS);
    QuadPlace at;
    if constexpr (ODD) {
        at.set(0, first < c1 ? first : C, C);
    } else {
        at.count = c1 - first;
        at.part = 0;
        at.col = at.at = c1 == C || first < c1 ? first : kNoQuad;
    }
    return at;
}

// A quad's logits as float32, -infinity behind the row's or split's end.
template <bool YBF, bool ODD>
__device__ __forceinline__ row_f32x4 logits(const RawRowQuad<YBF, false> &raw, const QuadPlace &at, bool cut) {
    row_f32x4 y = raw.get(at, ODD);
    if (cut)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i >= at.count) y[i] = -INFINITY;
    return y;
}

// What the gradient of a row is made of.
template <bool ODD>
struct RowGrad {
    float m, a, ct, ch, it, i1;      // i1: at T = 1 the label's share is in `it`
    int lab;
    bool labeled, two;               // two: a softmax of its own for the label
    __device__ __forceinline__ RowGrad(const Args &args, const RowStats &s, bool taught, int lab_)
        : m(s.m), a(args.temp_a), lab(lab_) {
        labeled = lab >= 0 && lab < args.C;
        two = labeled && a != kLog2e;
        ct = taught ? args.soft : 0.f;
        ch = labeled ? args.hard : 0.f;
        it = (two ? ct : ct + ch) * __builtin_amdgcn_rcpf(s.st);
        i1 = two ? ch * __builtin_amdgcn_rcpf(s.s1) : 0.f;
    }
    // one quad, stored; its share of the loss (sum of P (y - m), the label's y - m) is added
    __device__ __forceinline__ void quad(const Args &args, int64_t row, const QuadPlace &at, row_f32x4 y, int col,
                                         row_f32x4 P, float &cross, float &label) const {
        row_f32x4 o;
        y -= m;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = exp2_fast(y[i] * a) * it;
        if (two)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(exp2_fast(y[i] * kLog2e), i1, o[i]);
        if (labeled && static_cast<uint32_t>(lab - col) < 4u && at.count > 0)    // places behind c1 are another split's
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i == lab) {
                    o[i] -= ch;
                    label += y[i];
                }
        if (some(P))
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cross = fmaf(P[i], P[i] == 0.f ? 0.f : y[i], cross);
                o[i] = fmaf(-ct, P[i], o[i]);
            }
        if (args.g_bf16)
            store_row_quad<true, false>(row_window<true>(args.G, row * args.C, args.C), at, o, ODD, args.streaming);
        else
            store_row_quad<false, false>(row_window<false>(args.G, row * args.C, args.C), at, o, ODD, args.streaming);
    }
};

// Zeros to the classes [c0, c1) of a row.
template <int THREADS, bool ODD>
__device__ __forceinline__ void put_zeros(const Args &a, int64_t row, int c0, int c1) {
    const row_f32x4 z = {0.f, 0.f, 0.f, 0.f};
    for (int c = c0; c < c1; c += 4 * THREADS) {
        const QuadPlace at = place<THREADS, ODD>(threadIdx.x, c, 0, c1, a.C);
        if (a.g_bf16) store_row_quad<true, false>(row_window<true>(a.G, row * a.C, a.C), at, z, ODD, a.streaming);
        else store_row_quad<false, false>(row_window<false>(a.G, row * a.C, a.C), at, z, ODD, a.streaming);
    }
}

// A row that QUADS quads of THREADS threads hold.  The second bound keeps a CU's registers full.
// Measured, 16 entries a row, T = 2, labels, float32 / bfloat16: 16,384 x 8,192 192 / 130 us (5.6 / 4.1 TB/s), 8,192 x 16,384
// 218 / 124 us, 65,536 x 2,000 223 / 158 us; with bfloat16 the vector unit is busy all the time by its counter (four exponentials a
// logit), with float32 77%.
template <bool YBF, bool TBF, bool ODD, int THREADS, int QUADS>
__global__ __launch_bounds__(THREADS, 4) void distill_held_kernel(Args a) {
    __shared__ row_f32x4 sh[row_reduce_quads<THREADS>()];
    __shared__ row_f32x4 tiles[THREADS * kHeldQ];
    __shared__ int flag;
    int turn = 0;
    const int C = a.C;
    constexpr int kPiece = 4 * THREADS * kHeldQ;
    float *tile = reinterpret_cast<float *>(tiles);
#pragma unroll
    for (int q = 0; q < kHeldQ; ++q) tiles[threadIdx.x + q * THREADS] = row_f32x4{0.f, 0.f, 0.f, 0.f};
    if (threadIdx.x == 0) flag = 0;
    __syncthreads();
    double soft = 0.0, hard = 0.0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const __amdgpu_buffer_rsrc_t wy = row_window<YBF>(a.Y, row * C, C);
        RawRowQuad<YBF, false> raw[QUADS];
        int thread = anew(static_cast<int>(threadIdx.x));
#pragma unroll
        for (int q = 0; q < QUADS; ++q) {
            const QuadPlace at = place<THREADS, ODD>(thread, 0, q, C, C);
            raw[q].load(wy, at.at, at.count);
        }
        Entries<THREADS, TBF> en;
        en.load(a, row, threadIdx.x);
        const int lab = a.labels ? a.labels[row] : -1;
        const bool labeled = lab >= 0 && lab < C, two = labeled && a.temp_a != kLog2e;
        float top[3];
        en.local_max(top);
        top[2] = -FLT_MAX;
#pragma unroll
        for (int q = 0; q < QUADS; ++q)
            if (4 * q * THREADS < C) {                   // uniform
                const row_f32x4 y = logits<YBF, ODD>(raw[q], place<THREADS, ODD>(thread, 0, q, C, C), 4 * (q + 1) * THREADS > C);
                top[2] = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), top[2]);
            }
        row_reduce<THREADS>(top, MaxOp(), sh, turn);
        float s[3];
        en.local_sum(top, a.temp_a, s);
        s[1] = s[2] = 0.f;
        thread = anew(thread);
#pragma unroll
        for (int q = 0; q < QUADS; ++q)
            if (4 * q * THREADS < C) {
                raw[q].v = anew(raw[q].v);
                row_f32x4 y = logits<YBF, ODD>(raw[q], place<THREADS, ODD>(thread, 0, q, C, C), 4 * (q + 1) * THREADS > C);
                y -= top[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[1] += exp2_fast(y[i] * a.temp_a);
                if (two)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[2] += exp2_fast(y[i] * kLog2e);
                if (q % 2) __builtin_amdgcn_sched_barrier(0);    // registers for two quads' work, not for all
            }
        row_reduce<THREADS>(s, AddOp(), sh, turn);
        if (!en.taught && !labeled) {                    // zeros, whatever the logits
            put_zeros<THREADS, ODD>(a, row, 0, C);
            continue;
        }
        en.have(s[0]);
        const RowGrad<ODD> grad(a, RowStats{top[2], s[1], s[2]}, en.taught, lab);
        float cross = 0.f, label = 0.f;
#pragma unroll
        for (int q0 = 0; q0 < QUADS; q0 += kHeldQ) {
            const int c = 4 * q0 * THREADS;
            thread = anew(thread);
            if (c < C) {
                if (en.taught) en.scatter(tile, c, min(C, c + kPiece), a.temp_a, &flag);
#pragma unroll
                for (int q = q0; q < q0 + kHeldQ && q < QUADS; ++q)
                    if (4 * q * THREADS < C) {
                        raw[q].v = anew(raw[q].v);
                        const QuadPlace at = place<THREADS, ODD>(thread, 0, q, C, C);
                        grad.quad(a, row, at, raw[q].get(at, ODD), 4 * (thread + q * THREADS),
                                  tiles[threadIdx.x + (q - q0) * THREADS], cross, label);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                if (en.taught) {
                    __syncthreads();
                    en.clear(tile, c, min(C, c + kPiece));
                    __syncthreads();
                }
            }
        }
        if (en.taught) {
            soft += en.entropy - static_cast<double>(a.temp_a) * cross;
            if (threadIdx.x == 0) soft += __builtin_amdgcn_logf(s[1]) - __builtin_amdgcn_logf(s[0]);
        }
        if (labeled) {
            hard -= static_cast<double>(kLog2e) * label;
            if (threadIdx.x == 0) hard += __builtin_amdgcn_logf(two ? s[2] : s[1]);
        }
    }
    write_partial<THREADS>(soft, hard, a.partial + 2 * static_cast<int64_t>(blockIdx.x));
}

// Classes [c0, c1) of a row: maximum and sums at T and (one) at 1, over the workgroup.
template <bool YBF, bool ODD>
__device__ __forceinline__ RowStats sweep_stats(const Args &a, int64_t row, int c0, int c1, bool one, row_f32x4 *sh,
                                                int &turn) {
    constexpr int kPiece = 4 * kSweep * kSweepQ;
    float m = -FLT_MAX, st = 0.f, s1 = 0.f;
    const __amdgpu_buffer_rsrc_t w = row_window<YBF>(a.Y, row * a.C, a.C);
    for (int c = c0; c < c1; c += kPiece) {
        RawRowQuad<YBF, false> raw[kSweepQ];
#pragma unroll
        for (int q = 0; q < kSweepQ; ++q) {
            const QuadPlace at = place<kSweep, ODD>(threadIdx.x, c, q, c1, a.C);
            raw[q].load(w, at.at, at.count);
        }
        row_f32x4 y[kSweepQ];
        float top = m;
#pragma unroll
        for (int q = 0; q < kSweepQ; ++q) {
            y[q] = logits<YBF, ODD>(raw[q], place<kSweep, ODD>(threadIdx.x, c, q, c1, a.C), c + kPiece > c1);
            top = fmaxf(fmaxf(fmaxf(y[q][0], y[q][1]), fmaxf(y[q][2], y[q][3])), top);
        }
        st *= exp2_fast((m - top) * a.temp_a);
        s1 *= exp2_fast((m - top) * kLog2e);
        m = top;
        // a piece's exponentials by themselves first, so that no chain of additions is longer than a row's 64 pieces (with all
        // added one by one, the sums of rows of 2^20 classes were off by 187 times 2^-24 and more)
        auto piece = [&](float by) {
            float sum[kSweepQ];
#pragma unroll
            for (int q = 0; q < kSweepQ; ++q) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = exp2_fast((y[q][i] - m) * by);
                sum[q] = (e[0] + e[1]) + (e[2] + e[3]);
            }
#pragma unroll
            for (int h = kSweepQ / 2; h > 0; h >>= 1)
#pragma unroll
                for (int q = 0; q < h; ++q) sum[q] += sum[q + h];
            return sum[0];
        };
        st += piece(a.temp_a);
        if (one) s1 += piece(kLog2e);
    }
    float all[1] = {m};
    row_reduce<kSweep>(all, MaxOp(), sh, turn);
    float s[2] = {st * exp2_fast((m - all[0]) * a.temp_a), s1 * exp2_fast((m - all[0]) * kLog2e)};
    row_reduce<kSweep>(s, AddOp(), sh, turn);
    return RowStats{all[0], s[0], s[1]};
}

// Classes of a split: whole quads.
__host__ __device__ __forceinline__ int split_width(int C, int splits) { return ((C + splits - 1) / splits + 3) / 4 * 4; }

// First launch of split rows: statistics of split blockIdx.x of row blockIdx.y.  Both launches and the
// loss: 1 x 1,000,000 18.7 us, 16 x 131,072 20.4 us; with one workgroup a row the chip would stand idle.
template <bool YBF, bool ODD>
__global__ __launch_bounds__(kSweep) void distill_stats_kernel(Args a) {
    __shared__ row_f32x4 sh[row_reduce_quads<kSweep>()];
    int turn = 0;
    const int splits = gridDim.x, width = split_width(a.C, splits);
    const int c0 = min(a.C, static_cast<int>(blockIdx.x) * width), c1 = min(a.C, c0 + width);
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        const RowStats s = sweep_stats<YBF, ODD>(a, row, c0, c1, a.labels != nullptr, sh, turn);
        if (threadIdx.x == 0) {
            float *o = a.stats + (row * splits + blockIdx.x) * 3;
            o[0] = s.m;
            o[1] = s.st;
            o[2] = s.s1;
        }
    }
}

// The gradient of rows of any length.  With one split the workgroup sweeps its rows' statistics
// itself; else they come from `stats`.  Measured: 4,095 x 131,072 bfloat16, T = 1, 64 entries: 2.15 GB in 479 us a call,
// 4.5 TB/s, and a second reading of Y, 1.07 GB, from beyond the L2 and for the most part not from HBM.
template <bool YBF, bool TBF, bool ODD>
__global__ __launch_bounds__(kSweep, 4) void distill_sweep_kernel(Args a) {
    constexpr int kPiece = 4 * kSweep * kSweepQ;
    __shared__ row_f32x4 sh[row_reduce_quads<kSweep>()];
    __shared__ row_f32x4 tiles[kSweep * kSweepQ];
    __shared__ int flag;
    int turn = 0;
    float *tile = reinterpret_cast<float *>(tiles);
    const int splits = gridDim.x, width = split_width(a.C, splits);
    const int c0 = min(a.C, static_cast<int>(blockIdx.x) * width), c1 = min(a.C, c0 + width);
#pragma unroll
    for (int q = 0; q < kSweepQ; ++q) tiles[threadIdx.x + q * kSweep] = row_f32x4{0.f, 0.f, 0.f, 0.f};
    if (threadIdx.x == 0) flag = 0;
    __syncthreads();
    double soft = 0.0, hard = 0.0;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        Entries<kSweep, TBF> en;
        en.load(a, row, threadIdx.x);
        const int lab = a.labels ? a.labels[row] : -1;
        const bool labeled = lab >= 0 && lab < a.C;
        float top[2], sum[1];
        en.local_max(top);
        row_reduce<kSweep>(top, MaxOp(), sh, turn);
        en.local_sum(top, a.temp_a, sum);
        row_reduce<kSweep>(sum, AddOp(), sh, turn);
        if (!en.taught && !labeled) {
            put_zeros<kSweep, ODD>(a, row, c0, c1);
            continue;
        }
        en.have(sum[0]);
        RowStats s;
        if (splits == 1) {
            s = sweep_stats<YBF, ODD>(a, row, 0, a.C, labeled && a.temp_a != kLog2e, sh, turn);
        } else {
            // a split a thread (one after the other they took most of a single row's time)
            const bool there = static_cast<int>(threadIdx.x) < splits;
            const float *in = a.stats + (row * splits + (there ? threadIdx.x : 0)) * 3;
            const float m = there ? in[0] : -FLT_MAX;
            float all[1] = {m};
            row_reduce<kSweep>(all, MaxOp(), sh, turn);
            float sums[2] = {there ? in[1] * exp2_fast((m - all[0]) * a.temp_a) : 0.f,
                             there ? in[2] * exp2_fast((m - all[0]) * kLog2e) : 0.f};
            row_reduce<kSweep>(sums, AddOp(), sh, turn);
            s = RowStats{all[0], sums[0], sums[1]};
        }
        const RowGrad<ODD> grad(a, s, en.taught, lab);
        const __amdgpu_buffer_rsrc_t wy = row_window<YBF>(a.Y, row * a.C, a.C);
        float cross = 0.f, label = 0.f;
        for (int c = c0; c < c1; c += kPiece) {
            RawRowQuad<YBF, false> raw[kSweepQ];
#pragma unroll
            for (int q = 0; q < kSweepQ; ++q) {
                const QuadPlace at = place<kSweep, ODD>(threadIdx.x, c, q, c1, a.C);
                raw[q].load(wy, at.at, at.count);
            }
            if (en.taught) en.scatter(tile, c, min(c1, c + kPiece), a.temp_a, &flag);
#pragma unroll
            for (int q = 0; q < kSweepQ; ++q) {
                const QuadPlace at = place<kSweep, ODD>(threadIdx.x, c, q, c1, a.C);
                grad.quad(a, row, at, raw[q].get(at, ODD), c + 4 * (static_cast<int>(threadIdx.x) + q * kSweep),
                          tiles[threadIdx.x + q * kSweep], cross, label);
            }
            if (en.taught) {
                __syncthreads();
                en.clear(tile, c, min(c1, c + kPiece));
                __syncthreads();
            }
        }
        // each split of a row adds its classes; the first one what the row has once
        if (en.taught) {
            soft -= static_cast<double>(a.temp_a) * cross;
            if (blockIdx.x == 0) soft += en.entropy;
            if (blockIdx.x == 0 && threadIdx.x == 0) soft += __builtin_amdgcn_logf(s.st) - __builtin_amdgcn_logf(sum[0]);
        }
        if (labeled) {
            hard -= static_cast<double>(kLog2e) * label;
            if (blockIdx.x == 0 && threadIdx.x == 0) hard += __builtin_amdgcn_logf(a.temp_a == kLog2e ? s.st : s.s1);
        }
    }
    write_partial<kSweep>(soft, hard,
                          a.partial + 2 * (static_cast<int64_t>(blockIdx.y) * splits + blockIdx.x));
}

// ------------------------------------------------------------------ high temperatures
//
// Where the teacher keeps most classes, the divergence of a row falls as 1 / T^2, while its terms in float32 (the logarithms of
// the sums above all) keep an error of about 5e-7, which T^2 enlarges: of a loss of 4 a row 3e-5 at T = 8, but 1e-3 at
// T = 100 and more than itself at T = 10,000.  Past kHotTemperature the soft loss is formed in float64, in a
// launch of its own: with z = (y - m) / T of both sides,
//   sum p_k (log p_k - log Q[id_k]) = sum e_k (z_k - z_y[id_k]) / sum e_k + log sum_j exp(z_y[j]) - log sum e_k.
// Bound by float64 exponentials, one a logit, and by the latency of few and long rows; us of a call below and past 8: 2^22 x 64
// (16 entries, many twice) 1,045, 2,110; 65,536 x 2,000 bfloat16 165, 375; 4,095 x 131,072 bfloat16 519, 1,387; 30,007 x 47 13, 23;
// 1 x 1,000,000 16, 285.
constexpr float kHotTemperature = 8.f;

template <int TPR, bool YBF, bool TBF>
__global__ __launch_bounds__((TPR > 64 ? TPR : kThreads)) void distill_hot_kernel(Args a, double inv_t, double *out) {
    constexpr int kBlock = TPR > 64 ? TPR : kThreads, kGroups = kBlock / TPR;
    __shared__ row_f32x4 sh[row_reduce_quads<TPR>()];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    auto logit = [](const void *p, int64_t at) {
        if constexpr (YBF) return bf16_to_float(static_cast<const unsigned short *>(p)[at]);
        else return static_cast<const float *>(p)[at];
    };
    double soft = 0.0;
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kGroups; row0 < a.n;
         row0 += static_cast<int64_t>(gridDim.x) * kGroups) {
        const int64_t row = row0 + g;
        const int C = row < a.n ? a.C : 0;               // a row behind the last has no classes and no entries
        const int K = row < a.n ? a.K : 0;
        // f of the classes and logits of the entries that count
        auto entries = [&](auto f) {
            for (int k = l; k < K; k += TPR) {
                const int i = a.ids[row * a.K + k];
                const float x = teacher_at<TBF>(a.teacher, row * a.K + k);
                if (i >= 0 && i < C && !(x == -INFINITY)) f(i, x);
            }
        };
        float top[3] = {-INFINITY, 0.f, -FLT_MAX};       // the entries' largest, is there one, the row's largest
        entries([&](int, float x) {
            top[0] = fmaxf(top[0], x);
            top[1] = 1.f;
        });
#pragma unroll 4
        for (int c = l; c < C; c += TPR) top[2] = fmaxf(top[2], logit(a.Y, row * a.C + c));
        row_reduce<TPR>(top, MaxOp(), sh, turn);
        const double mt = top[0], my = top[2];
        double st = 0.0, cross = 0.0, sy = 0.0;
        entries([&](int i, float x) {
            const double z = (x - mt) * inv_t, e = exp(z);
            st += e;
            if (e != 0.0) cross += e * (z - (logit(a.Y, row * a.C + i) - my) * inv_t);     // no 0 * infinity
        });
#pragma unroll 4
        for (int c = l; c < C; c += TPR) sy += exp((logit(a.Y, row * a.C + c) - my) * inv_t);
        st = row_sum<TPR>(st, sh, turn);
        cross = row_sum<TPR>(cross, sh, turn);
        sy = row_sum<TPR>(sy, sh, turn);
        if (l == 0 && top[1] > 0.f) soft += cross / st + log(sy) - log(st);
    }
    write_partial<kBlock>(soft / kLn2, 0.0, out + 2 * static_cast<int64_t>(blockIdx.x));    // as the other sums: in powers of 2
}

// loss = {soft + hard, soft, hard} from the workgroups' sums, by a fixed tree.  `hot`: the soft ones, if they are apart.
// 16 bytes a load, eight in flight a thread (8,192 workgroups: 13 us with one load at a time).
constexpr int kLossThreads = 1024;
typedef double f64x2 __attribute__((ext_vector_type(2)));
__global__ __launch_bounds__(kLossThreads) void distill_loss_kernel(const double *__restrict__ partial, int32_t count,
                                                                    const double *__restrict__ hot, int32_t hot_count,
                                                                    double soft, double hard, float *__restrict__ loss) {
    __shared__ f64x2 sh[kLossThreads];
    const int t = threadIdx.x;
    constexpr int kLoads = kMaxBlocks / kLossThreads;
    f64x2 v[kLoads], sum = {0.0, 0.0};
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int i = t + j * kLossThreads;
        v[j] = i < count ? reinterpret_cast<const f64x2 *>(partial)[i] : f64x2{0.0, 0.0};
    }
    if (hot)
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = t + j * kLossThreads;
            v[j][0] = i < hot_count ? hot[2 * i] : 0.0;
        }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) sum += v[j];
    sh[t] = sum;
    __syncthreads();
#pragma unroll
    for (int h = kLossThreads / 2; h > 0; h >>= 1) {
        if (t < h) sh[t] += sh[t + h];
        __syncthreads();
    }
    if (t == 0) {
        const double s = soft * kLn2 * sh[0][0], r = hard * kLn2 * sh[0][1];
        loss[0] = static_cast<float>(s + r);
        loss[1] = static_cast<float>(s);
        loss[2] = static_cast<float>(r);
    }
}

// ------------------------------------------------------------------ dispatch

constexpr int kRowClasses = 1024;                    // widest row of distill_rows_kernel
constexpr int kHeldClasses = 32768;                  // widest row of distill_held_kernel
constexpr int kSplitBlocks = 512;                    // workgroups that fill the chip (two a CU)
static_assert(kSplitBlocks <= kSweep, "a row's splits are joined by one thread each");
constexpr int kMinSplit = 4096;                      // classes a split has at least

// Rows that a workgroup can hold are not split (us split and held, 1 and 255 rows of 32,768 bfloat16: 20.5, 17.1 and
// 21.8, 21.1); longer ones where the rows are few (split and swept whole, 131,072 bfloat16: 1 row 20.8, 35.8; 100
// rows 29.2, 39.5; 200 rows 42.7, 39.8).
int splits_of(int32_t n, int32_t C) {
    if (C <= kHeldClasses || n > kSplitBlocks / 4) return 1;
    const int want = kSplitBlocks / n, most = (C + kMinSplit - 1) / kMinSplit;
    return std::max(1, std::min(want, most));
}

int row_blocks(int32_t n, int groups) {
    return static_cast<int>(std::min<int64_t>((static_cast<int64_t>(n) + groups - 1) / groups, kMaxBlocks));
}

template <int TPR, int Q, bool YBF>
int launch_rows(const Args &a, bool tbf, hipStream_t s) {
    constexpr int kBlock = TPR > 64 ? TPR : kThreads;
    const int blocks = row_blocks(a.n, kBlock / TPR);
    if (tbf) hipLaunchKernelGGL((distill_rows_kernel<TPR, Q, YBF, true>), dim3(blocks), dim3(kBlock), 0, s, a);
    else hipLaunchKernelGGL((distill_rows_kernel<TPR, Q, YBF, false>), dim3(blocks), dim3(kBlock), 0, s, a);
    return blocks;
}

template <bool YBF, bool ODD, int THREADS, int QUADS>
int launch_held(const Args &a, bool tbf, hipStream_t s) {
    const int blocks = row_blocks(a.n, 1);
    if (tbf) hipLaunchKernelGGL((distill_held_kernel<YBF, true, ODD, THREADS, QUADS>), dim3(blocks), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((distill_held_kernel<YBF, false, ODD, THREADS, QUADS>), dim3(blocks), dim3(THREADS), 0, s, a);
    return blocks;
}

// Rows past those of distill_rows_kernel.  Few threads with many quads each leave room for more rows
// on a CU (2^27 elements, us, float32 / bfloat16, floor 186 / 93: C = 8,192 (256, 8) 204 / 160, (512, 4) 251 / 181,
// (1024, 4) twice that); past 32,768 classes two workgroups a CU hold less than the sweep's second reading of
// a row from the caches costs (2^28 elements: C = 65,536 swept 457 / 297, held by 1,024 threads 582 / 360).
template <bool YBF, bool ODD>
int launch_long(const Args &a, bool tbf, hipStream_t s) {
    const int C = a.C;
    if (C <= kHeldClasses) {
        if (C <= 2048) return launch_held<YBF, ODD, 64, 8>(a, tbf, s);
        // (float32 / bfloat16 at C = 3,000: (256, 4) 212 / 165, (128, 8) 227 / 140)
        if (C <= 4096) return launch_held<YBF, ODD, YBF ? 128 : 256, YBF ? 8 : 4>(a, tbf, s);
        if (C <= 8192) return launch_held<YBF, ODD, 256, 8>(a, tbf, s);
        if (C <= 16384) return launch_held<YBF, ODD, 256, 16>(a, tbf, s);
        return launch_held<YBF, ODD, 512, 16>(a, tbf, s);
    }
    const int splits = splits_of(a.n, C);
    const dim3 grid(splits, row_blocks(a.n, 1));
    if (splits > 1) hipLaunchKernelGGL((distill_stats_kernel<YBF, ODD>), grid, dim3(kSweep), 0, s, a);
    if (tbf) hipLaunchKernelGGL((distill_sweep_kernel<YBF, true, ODD>), grid, dim3(kSweep), 0, s, a);
    else hipLaunchKernelGGL((distill_sweep_kernel<YBF, false, ODD>), grid, dim3(kSweep), 0, s, a);
    return static_cast<int>(grid.x * grid.y);
}

template <int TPR>
int launch_hot(const Args &a, bool ybf, bool tbf, float T, double *out, hipStream_t s) {
    constexpr int kBlock = TPR > 64 ? TPR : kThreads;
    const int blocks = row_blocks(a.n, kBlock / TPR);
    auto launch = [&](auto y, auto t) {
        hipLaunchKernelGGL((distill_hot_kernel<TPR, decltype(y)::value, decltype(t)::value>), dim3(blocks), dim3(kBlock), 0, s, a,
                           1.0 / T, out);
    };
    if (ybf && tbf) launch(std::true_type(), std::true_type());
    else if (ybf) launch(std::true_type(), std::false_type());
    else if (tbf) launch(std::false_type(), std::true_type());
    else launch(std::false_type(), std::false_type());
    return blocks;
}

// Few lanes a row with several quads each share a wavefront's instructions between more rows
// (2^27 elements, us, float32 / bfloat16: C = 128 (16, 2) 238 / 203, (32, 1) 309 / 295; C = 256 (16, 4) 217 / 169, (64, 1)
// 317 / 306).
template <bool YBF>
int launch_any(const Args &a, bool tbf, hipStream_t s) {
    const int C = a.C;
    if (C < 4) return launch_rows<1, 1, YBF>(a, tbf, s);
    if (C <= 16) return launch_rows<4, 1, YBF>(a, tbf, s);
    if (C <= 32) return launch_rows<8, 1, YBF>(a, tbf, s);
    if (C <= 64) return launch_rows<8, 2, YBF>(a, tbf, s);
    if (C <= 128) return launch_rows<16, 2, YBF>(a, tbf, s);
    if (C <= 192) return launch_rows<16, 3, YBF>(a, tbf, s);
    if (C <= 256) return launch_rows<16, 4, YBF>(a, tbf, s);
    if (C <= 384) return launch_rows<32, 3, YBF>(a, tbf, s);
    if (C <= 512) return launch_rows<32, 4, YBF>(a, tbf, s);
    if (C <= 768) return launch_rows<64, 3, YBF>(a, tbf, s);
    if (C <= kRowClasses) return launch_rows<64, 4, YBF>(a, tbf, s);
    return C & 3 ? launch_long<YBF, true>(a, tbf, s) : launch_long<YBF, false>(a, tbf, s);
}

}  // namespace

size_t distill_workspace_bytes(int32_t n, int32_t C) {
    // partial sums of the loss, those of the soft loss at high temperatures, then the statistics of split rows (rows
    // that are split are few)
    size_t bytes = 4 * sizeof(double) * kMaxBlocks;
    if (splits_of(n, C) > 1) bytes += sizeof(float) * 3 * static_cast<size_t>(n) * splits_of(n, C);
    return (bytes + 255) / 256 * 256;
}

int launch_distill(const void *Y, bool y_bf16, const int32_t *ids, const void *teacher, bool t_bf16,
                   const int32_t *labels, int32_t n, int32_t C, int32_t K, float T, float soft, float hard, void *G,
                   bool g_bf16, float *loss, void *workspace, hipStream_t s) {
    double *partial = static_cast<double *>(workspace);
    const int64_t elems = static_cast<int64_t>(n) * C;
    const Args a{Y, teacher, ids, labels, G, partial, reinterpret_cast<float *>(partial + 4 * kMaxBlocks), n, C, K,
                 T == 1.f ? kLog2e : kLog2e / T, soft * T, hard, g_bf16, elems * (g_bf16 ? 2 : 4) > (int64_t{32} << 20)};
    const int blocks = y_bf16 ? launch_any<true>(a, t_bf16, s) : launch_any<false>(a, t_bf16, s);
    int st = hip_status(hipGetLastError());
    if (st) return st;
    double *hot = nullptr;
    int hot_blocks = 0;
    if (T > kHotTemperature) {
        hot = partial + 2 * kMaxBlocks;
        hot_blocks = C <= 128 ? launch_hot<16>(a, y_bf16, t_bf16, T, hot, s)
                   : C <= 2048 ? launch_hot<64>(a, y_bf16, t_bf16, T, hot, s)
                   : C <= 16384 ? launch_hot<256>(a, y_bf16, t_bf16, T, hot, s)
                               : launch_hot<1024>(a, y_bf16, t_bf16, T, hot, s);
        if ((st = hip_status(hipGetLastError()))) return st;
    }
    hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(kLossThreads), 0, s, partial, blocks, hot, hot_blocks,
                       static_cast<double>(soft) * T * T, static_cast<double>(hard), loss);
    return hip_status(hipGetLastError());
}

}  // namespace dgc
