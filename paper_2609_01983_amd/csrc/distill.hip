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
    float t[kHeld];                  // the logit; -inf: none
    float m, inv;                    // largest logit; 1 / sum of the exponentials
    bool taught;

    __device__ __forceinline__ void fetch(int64_t k, int &i, float &x) const {
        i = ids[at + k];
        x = teacher_at<TBF>(teacher, at + k);
        if (i < 0 || i >= C) x = -INFINITY;
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
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) f(id[h], t[h]);
        for (int k = l + kHeld * TPR; k < K; k += TPR) {
            int i;
            float x;
            fetch(k, i, x);
            f(i, x);
        }
    }
    __device__ __forceinline__ float p(float x, float a) const { return exp2_fast((x - m) * a) * inv; }

    // The row's largest logit and the sum of its exponentials; `entropy` receives sum p log2 p.
    __device__ __forceinline__ void prepare(float a, float *sh, int &turn, float &entropy) {
        float top[2] = {-INFINITY, 0.f};                 // second: does an entry count? (NaN does)
        each([&](int, float x) {
            top[0] = fmaxf(top[0], x);
            if (!(x == -INFINITY)) top[1] = 1.f;
        });
        row_reduce<TPR>(top, MaxOp(), sh, turn);
        m = top[0];
        taught = top[1] > 0.f;
        entropy = 0.f;
        inv = 0.f;
        if (!taught) return;                             // the same for all threads of the row
        float s[2] = {0.f, 0.f};
        each([&](int, float x) {
            if (!(x == -INFINITY)) {
                const float z = (x - m) * a, e = exp2_fast(z);
                s[0] += e;
                if (!(e == 0.f)) s[1] = fmaf(e, z, s[1]);
            }
        });
        row_reduce<TPR>(s, AddOp(), sh, turn);
        inv = 1.f / s[0];
        entropy = s[1] * inv - __builtin_amdgcn_logf(s[0]);
    }

    // P of the classes [c0, c1) into tile[id - c0] (zeros before); clear() undoes it.
    __device__ __forceinline__ void scatter(float *tile, int c0, int c1, float a, int *flag) const {
        bool twice = false;
        each([&](int i, float x) {
            if (!(x == -INFINITY) && i >= c0 && i < c1) {
                const float v = p(x, a);
                if (!(v == 0.f))
                    twice |= __hip_atomic_exchange(tile + (i - c0), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) != 0.f;
            }
        });
        if constexpr (TPR > 64) {
            if (twice) *flag = 1;
            __syncthreads();
            twice = *flag != 0;
            __syncthreads();
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
                    if (!(x == -INFINITY) && i >= c0 && i < c1) tile[i - c0] += p(x, a);
                }
                if constexpr (TPR > 64) *flag = 0;
            }
        }
        row_sync<TPR>();
    }
    __device__ __forceinline__ void clear(float *tile, int c0, int c1) const {
        each([&](int i, float x) {
            if (!(x == -INFINITY) && i >= c0 && i < c1) tile[i - c0] = 0.f;
        });
    }
};

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
// logits, the teacher's are bfloat16.
template <int TPR, int Q, bool YBF, bool TBF>
__global__ __launch_bounds__((TPR > 64 ? TPR : kThreads)) void distill_rows_kernel(Args a) {
    constexpr bool TINY = TPR == 1;
    constexpr int kBlock = TPR > 64 ? TPR : kThreads, kGroups = kBlock / TPR;
    __shared__ float sh[row_reduce_floats<TPR>()];
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
        float entropy;
        en.prepare(a.temp_a, sh, turn, entropy);
        row_f32x4 o[Q];
        if (!en.taught && !labeled) {                    // zeros, whatever the logits
#pragma unroll
            for (int q = 0; q < Q; ++q) o[q] = row_f32x4{0.f, 0.f, 0.f, 0.f};
        } else {
            row_f32x4 y[Q];
            float m[1] = {-FLT_MAX};                     // all of the row -inf: the sums are 0, G NaN
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                y[q] = raw[q].get(at[q], odd);
                if (ragged)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i >= at[q].count) y[q][i] = -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) m[0] = fmaxf(m[0], y[q][i]);
            }
            row_reduce<TPR>(m, MaxOp(), sh, turn);
            row_f32x4 e1[Q];
            float s[3] = {0.f, 0.f, 0.f};                // at T, at 1, the label's y - m
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[q][i] -= m[0];
                    o[q][i] = exp2_fast(y[q][i] * a.temp_a);
                    s[0] += o[q][i];
                }
            if (labeled) {
                if (!same)
#pragma unroll
                    for (int q = 0; q < Q; ++q)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            e1[q][i] = exp2_fast(y[q][i] * kLog2e);
                            s[1] += e1[q][i];
                        }
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * (l + q * TPR) + i == lab) s[2] = y[q][i];
            }
            row_reduce<TPR>(s, AddOp(), sh, turn);
            if (en.taught) en.scatter(tile, 0, C, a.temp_a, &flag);
            if (same) s[1] = s[0];
            const float ct = en.taught ? a.soft : 0.f;
            // at T = 1 the label's share of the softmax joins the teacher's
            const float it = ct / s[0] + (same && labeled ? a.hard / s[0] : 0.f);
            float cross[1] = {0.f};
#pragma unroll
            for (int q = 0; q < Q; ++q) o[q] *= it;
            if (labeled) {
                const float i1 = a.hard / s[1];
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (!same) o[q] += e1[q] * i1;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * (l + q * TPR) + i == lab) o[q][i] -= a.hard;
                }
            }
            if (en.taught) {
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const row_f32x4 P = tiles[g][l + q * TPR];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // no 0 * infinity where the class has no P
                        cross[0] = fmaf(P[i], P[i] == 0.f ? 0.f : y[q][i], cross[0]);
                        o[q][i] = fmaf(-ct, P[i], o[q][i]);
                    }
                }
                row_reduce<TPR>(cross, AddOp(), sh, turn);
                if constexpr (TPR <= 64) row_sync<TPR>();    // P is read before it is cleared
                en.clear(tile, 0, C);
                row_sync<TPR>();
            }
            if (l == 0) {
                if (en.taught) soft += entropy - static_cast<double>(a.temp_a) * cross[0] + __builtin_amdgcn_logf(s[0]);
                if (labeled) hard += __builtin_amdgcn_logf(s[1]) - static_cast<double>(kLog2e) * s[2];
            }
        }
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
// A row that the registers do not hold is swept twice: a running maximum and sums, then the
// gradient, piece by piece of kPiece classes (their P in LDS).  A workgroup takes a row; where
// there are few rows, `splits` workgroups share each: a first launch leaves their maxima and sums
// in `stats`, the second joins them.
constexpr int kLong = 512;                           // threads
constexpr int kLongQ = 8;                            // quads a thread and piece
constexpr int kPiece = 4 * kLong * kLongQ;           // 16,384 classes, 64 KiB of P

struct RowStats {
    float m, st, s1;
};

// Quad q of this thread in the piece at class c, none from class c1 on (a whole number of quads, or
// the row's end).
__device__ __forceinline__ void place(QuadPlace &at, int c, int q, int c1, int C) {
    const int first = c + 4 * (static_cast<int>(threadIdx.x) + q * kLong);
    at.set(0, first < c1 ? first : C, C);
}

// Classes [c0, c1) of a row: maximum and sums at T and at 1, over the workgroup.
template <bool YBF>
__device__ __forceinline__ RowStats sweep_stats(const Args &a, int64_t row, int c0, int c1, bool one, float *sh,
                                                int &turn) {
    float m = -FLT_MAX, st = 0.f, s1 = 0.f;
    const __amdgpu_buffer_rsrc_t w = row_window<YBF>(a.Y, row * a.C, a.C);
    for (int c = c0; c < c1; c += kPiece) {
        RawRowQuad<YBF, false> raw[kLongQ];
        QuadPlace at[kLongQ];
#pragma unroll
        for (int q = 0; q < kLongQ; ++q) {
            place(at[q], c, q, c1, a.C);
            raw[q].load(w, at[q].at, at[q].count);
        }
        row_f32x4 y[kLongQ];
        float top = m;
#pragma unroll
        for (int q = 0; q < kLongQ; ++q) {
            y[q] = raw[q].get(at[q], a.C & 3);
            if (c + kPiece > c1)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= at[q].count) y[q][i] = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, y[q][i]);
        }
        st *= exp2_fast((m - top) * a.temp_a);
        s1 *= exp2_fast((m - top) * kLog2e);
        m = top;
#pragma unroll
        for (int q = 0; q < kLongQ; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) st += exp2_fast((y[q][i] - m) * a.temp_a);
        if (one)
#pragma unroll
            for (int q = 0; q < kLongQ; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) s1 += exp2_fast((y[q][i] - m) * kLog2e);
    }
    float all[1] = {m};
    row_reduce<kLong>(all, MaxOp(), sh, turn);
    float s[2] = {st * exp2_fast((m - all[0]) * a.temp_a), s1 * exp2_fast((m - all[0]) * kLog2e)};
    row_reduce<kLong>(s, AddOp(), sh, turn);
    return RowStats{all[0], s[0], s[1]};
}

__device__ __forceinline__ void put(const Args &a, int64_t row, const QuadPlace &at, row_f32x4 o) {
    const bool odd = a.C & 3;
    if (a.g_bf16) store_row_quad<true, false>(row_window<true>(a.G, row * a.C, a.C), at, o, odd, a.streaming);
    else store_row_quad<false, false>(row_window<false>(a.G, row * a.C, a.C), at, o, odd, a.streaming);
}

// The gradient of classes [c0, c1) and their part of the loss: sum of P (y - m), the
// label's y - m (both on every thread).
template <bool YBF, bool TBF>
__device__ __forceinline__ float2 sweep_grad(const Args &a, int64_t row, int c0, int c1, const RowStats &s,
                                             const Entries<kLong, TBF> &en, int lab, row_f32x4 *tile, int *flag, float *sh, int &turn) {
    const __amdgpu_buffer_rsrc_t wy = row_window<YBF>(a.Y, row * a.C, a.C);
    const bool odd = a.C & 3, labeled = lab >= 0 && lab < a.C, same = a.temp_a == kLog2e;
    const float ct = en.taught ? a.soft : 0.f, ch = labeled ? a.hard : 0.f;
    const float it = ct / s.st, i1 = ch / (same ? s.st : s.s1);
    float part[2] = {0.f, 0.f};
    for (int c = c0; c < c1; c += kPiece) {
        const int end = min(c1, c + kPiece);
        RawRowQuad<YBF, false> raw[kLongQ];
        QuadPlace at[kLongQ];
#pragma unroll
        for (int q = 0; q < kLongQ; ++q) {
            place(at[q], c, q, c1, a.C);
            raw[q].load(wy, at[q].at, at[q].count);
        }
        if (en.taught) en.scatter(reinterpret_cast<float *>(tile), c, end, a.temp_a, flag);
#pragma unroll
        for (int q = 0; q < kLongQ; ++q) {
            const int col = c + 4 * (static_cast<int>(threadIdx.x) + q * kLong);
            const row_f32x4 y = raw[q].get(at[q], odd);
            row_f32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = y[i] - s.m, e = exp2_fast(d * a.temp_a);
                o[i] = e * it;
                if (labeled) {
                    o[i] = fmaf(same ? e : exp2_fast(d * kLog2e), i1, o[i]);
                    if (col + i == lab && i < at[q].count) {   // places behind c1 are another split's
                        o[i] -= ch;
                        part[1] += d;
                    }
                }
            }
            if (en.taught) {
                const row_f32x4 P = tile[threadIdx.x + q * kLong];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    part[0] = fmaf(P[i], P[i] == 0.f ? 0.f : y[i] - s.m, part[0]);
                    o[i] = fmaf(-ct, P[i], o[i]);
                }
            }
            put(a, row, at[q], o);
        }
        if (en.taught) {
            __syncthreads();
            en.clear(reinterpret_cast<float *>(tile), c, end);
            __syncthreads();
        }
    }
    row_reduce<kLong>(part, AddOp(), sh, turn);
    return make_float2(part[0], part[1]);
}

// Classes of a split: whole quads.
__host__ __device__ __forceinline__ int split_width(int C, int splits) { return ((C + splits - 1) / splits + 3) / 4 * 4; }

// First launch of split rows: statistics of split blockIdx.x of row blockIdx.y (and rows 65,535 on).
template <bool YBF>
__global__ __launch_bounds__(kLong) void distill_stats_kernel(Args a) {
    __shared__ float sh[row_reduce_floats<kLong>()];
    int turn = 0;
    const int splits = gridDim.x, width = split_width(a.C, splits);
    const int c0 = min(a.C, static_cast<int>(blockIdx.x) * width), c1 = min(a.C, c0 + width);
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        const RowStats s = sweep_stats<YBF>(a, row, c0, c1, a.labels != nullptr, sh, turn);
        if (threadIdx.x == 0) {
            float *o = a.stats + (row * splits + blockIdx.x) * 3;
            o[0] = s.m;
            o[1] = s.st;
            o[2] = s.s1;
        }
    }
}

// The gradient of rows of any length.  With one split the workgroup sweeps its rows' statistics
// itself; else they come from `stats`.
template <bool YBF, bool TBF>
__global__ __launch_bounds__(kLong) void distill_long_kernel(Args a) {
    __shared__ float sh[row_reduce_floats<kLong>()];
    __shared__ row_f32x4 tile[kLong * kLongQ];
    __shared__ int flag;
    int turn = 0;
    const int splits = gridDim.x, width = split_width(a.C, splits);
    const int c0 = min(a.C, static_cast<int>(blockIdx.x) * width), c1 = min(a.C, c0 + width);
#pragma unroll
    for (int q = 0; q < kLongQ; ++q) tile[threadIdx.x + q * kLong] = row_f32x4{0.f, 0.f, 0.f, 0.f};
    if (threadIdx.x == 0) flag = 0;
    __syncthreads();
    double soft = 0.0, hard = 0.0;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        Entries<kLong, TBF> en;
        en.load(a, row, threadIdx.x);
        const int lab = a.labels ? a.labels[row] : -1;
        const bool labeled = lab >= 0 && lab < a.C;
        float entropy;
        en.prepare(a.temp_a, sh, turn, entropy);
        if (!en.taught && !labeled) {
            for (int c = c0; c < c1; c += 4 * kLong) {
                QuadPlace at;
                place(at, c, 0, c1, a.C);
                put(a, row, at, row_f32x4{0.f, 0.f, 0.f, 0.f});
            }
            continue;
        }
        RowStats s;
        if (splits == 1) {
            s = sweep_stats<YBF>(a, row, 0, a.C, labeled && a.temp_a != kLog2e, sh, turn);
        } else {
            s = RowStats{-FLT_MAX, 0.f, 0.f};
            const float *in = a.stats + row * splits * 3;
            for (int k = 0; k < splits; ++k) s.m = fmaxf(s.m, in[3 * k]);
            for (int k = 0; k < splits; ++k) {
                s.st = fmaf(in[3 * k + 1], exp2_fast((in[3 * k] - s.m) * a.temp_a), s.st);
                s.s1 = fmaf(in[3 * k + 2], exp2_fast((in[3 * k] - s.m) * kLog2e), s.s1);
            }
        }
        const float2 part = sweep_grad<YBF, TBF>(a, row, c0, c1, s, en, lab, tile, &flag, sh, turn);
        if (threadIdx.x == 0) {
            if (en.taught) {
                soft -= static_cast<double>(a.temp_a) * part.x;
                if (blockIdx.x == 0) soft += static_cast<double>(entropy) + __builtin_amdgcn_logf(s.st);
            }
            if (labeled) {
                hard -= static_cast<double>(kLog2e) * part.y;
                if (blockIdx.x == 0)
                    hard += __builtin_amdgcn_logf(a.temp_a == kLog2e ? s.st : s.s1);
            }
        }
    }
    write_partial<kLong>(soft, hard,
                         a.partial + 2 * (static_cast<int64_t>(blockIdx.y) * splits + blockIdx.x));
}

// loss = {soft + hard, soft, hard} from the workgroups' sums, by a fixed tree.
__global__ __launch_bounds__(kThreads) void distill_loss_kernel(const double *__restrict__ partial, int32_t count,
                                                                double soft, double hard, float *__restrict__ loss) {
    __shared__ double sh[2][kThreads];
    const int t = threadIdx.x;
    double a = 0.0, b = 0.0;
    for (int i = t; i < count; i += kThreads) {
        a += partial[2 * i];
        b += partial[2 * i + 1];
    }
    sh[0][t] = a;
    sh[1][t] = b;
    __syncthreads();
    for (int h = kThreads / 2; h > 0; h >>= 1) {
        if (t < h) {
            sh[0][t] += sh[0][t + h];
            sh[1][t] += sh[1][t + h];
        }
        __syncthreads();
    }
    if (t == 0) {
        const double s = soft * kLn2 * sh[0][0], r = hard * kLn2 * sh[1][0];
        loss[0] = static_cast<float>(s + r);
        loss[1] = static_cast<float>(s);
        loss[2] = static_cast<float>(r);
    }
}

// ------------------------------------------------------------------ dispatch

constexpr int kRegisterClasses = 8192;               // widest row in registers
constexpr int kMaxBlocks = 8192;
constexpr int kSplitBlocks = 512;                    // workgroups that fill the chip (two a CU)
constexpr int kMinSplit = 4096;                      // classes a split has at least

int splits_of(int32_t n, int32_t C) {
    if (n >= kSplitBlocks / 2) return 1;
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

template <bool YBF>
int launch_any(const Args &a, bool tbf, hipStream_t s) {
    const int C = a.C;
    if (C < 4) return launch_rows<1, 1, YBF>(a, tbf, s);
    if (C <= 32) return launch_rows<8, 1, YBF>(a, tbf, s);
    if (C <= 64) return launch_rows<16, 1, YBF>(a, tbf, s);
    if (C <= 128) return launch_rows<32, 1, YBF>(a, tbf, s);
    if (C <= 256) return launch_rows<64, 1, YBF>(a, tbf, s);
    if (C <= 512) return launch_rows<64, 2, YBF>(a, tbf, s);
    if (C <= 1024) return launch_rows<64, 4, YBF>(a, tbf, s);
    if (C <= 2048) return launch_rows<256, 2, YBF>(a, tbf, s);
    if (C <= 4096) return launch_rows<256, 4, YBF>(a, tbf, s);
    if (C <= kRegisterClasses) return launch_rows<512, 4, YBF>(a, tbf, s);
    const int splits = splits_of(a.n, C);
    const dim3 grid(splits, row_blocks(a.n, 1));
    if (splits > 1) hipLaunchKernelGGL(distill_stats_kernel<YBF>, grid, dim3(kLong), 0, s, a);
    if (tbf) hipLaunchKernelGGL((distill_long_kernel<YBF, true>), grid, dim3(kLong), 0, s, a);
    else hipLaunchKernelGGL((distill_long_kernel<YBF, false>), grid, dim3(kLong), 0, s, a);
    return static_cast<int>(grid.x * grid.y);
}

}  // namespace

size_t distill_workspace_bytes(int32_t n, int32_t C) {
    // partial sums of the loss, then the statistics of split rows (rows that are split are few)
    size_t bytes = 2 * sizeof(double) * kMaxBlocks;
    if (C > kRegisterClasses && splits_of(n, C) > 1) bytes += sizeof(float) * 3 * static_cast<size_t>(n) * splits_of(n, C);
    return (bytes + 255) / 256 * 256;
}

int launch_distill(const void *Y, bool y_bf16, const int32_t *ids, const void *teacher, bool t_bf16,
                   const int32_t *labels, int32_t n, int32_t C, int32_t K, float T, float soft, float hard, void *G,
                   bool g_bf16, float *loss, void *workspace, hipStream_t s) {
    double *partial = static_cast<double *>(workspace);
    const int64_t elems = static_cast<int64_t>(n) * C;
    const Args a{Y, teacher, ids, labels, G, partial, reinterpret_cast<float *>(partial + 2 * kMaxBlocks), n, C, K,
                 T == 1.f ? kLog2e : kLog2e / T, soft * T, hard, g_bf16, elems * (g_bf16 ? 2 : 4) > (int64_t{32} << 20)};
    const int blocks = y_bf16 ? launch_any<true>(a, t_bf16, s) : launch_any<false>(a, t_bf16, s);
    const int st = hip_status(hipGetLastError());
    if (st) return st;
    hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(kThreads), 0, s, partial, blocks,
                       static_cast<double>(soft) * T * T, static_cast<double>(hard), loss);
    return hip_status(hipGetLastError());
}

}  // namespace dgc
