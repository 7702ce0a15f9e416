// Device helpers of the row-wise operators (norm.hip, distill.hip, fp8.hip): four
// consecutive elements of a float32 or bfloat16 row at any alignment, and sums and maxima
// over the 2^k lanes that share a row.
#pragma once

#include "deep.h"

#include <type_traits>

namespace dgc {

typedef float row_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 row_bf16x4 __attribute__((ext_vector_type(4)));
typedef double row_f64x4 __attribute__((ext_vector_type(4)));
// rows may start at any element: the loads and stores below need no more than its alignment
typedef float row_f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short row_u16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short row_u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_to_float(unsigned short b) {
    return __uint_as_float(static_cast<uint32_t>(b) << 16);
}

// Consecutive rows as a buffer: accesses past its end read zeros and write nothing, so rows behind
// the last and lanes without a column need no branch and no clamped address, and lanes address
// it with 32 bits.
template <bool BF>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_window(const void *base, int64_t first, int64_t elems) {
    constexpr int kSize = BF ? 2 : 4;
    return __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(const_cast<void *>(base)) + first * kSize, 0,
                                             static_cast<int>(elems * kSize), 0x00020000);
}

constexpr uint32_t kNoQuad = 0x3FFFFF00u;            // an element offset past every window, also in bytes and with a quad's places
constexpr int kNonTemporal = 2;                      // a buffer access's hint

// A lane's four consecutive columns of a row of F that starts at element `row_at` of its window.
// A row that ends inside them is read from its last four on (so that every load is whole) and
// shifted; `part` is how many columns it then has, 0 elsewhere.
struct QuadPlace {
    uint32_t at, col;                // element offsets in the window and in the row, or kNoQuad
    int part, count;                 // count: columns of the row from the lane's first on (<= 0: none)
    __device__ __forceinline__ void set(uint32_t row_at, int first, int F) {
        count = F - first;
        part = count > 0 && count < 4 ? count : 0;
        const int c = part ? (F < 4 ? 0 : F - 4) : first;
        at = count > 0 ? row_at + c : kNoQuad;
        col = count > 0 ? c : kNoQuad;
    }
};

// Four elements as stored, and as float32.  TINY: rows of fewer than four elements.  odd: F is no
// multiple of four (the same for every lane).
template <bool BF, bool TINY>
struct RawRowQuad {
    typename std::conditional<BF, row_u16x4, row_f32x4>::type v;

    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t w, uint32_t at, int count) {
        if constexpr (TINY) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t e = i < count ? at + i : kNoQuad;
                if constexpr (BF) v[i] = __builtin_amdgcn_raw_buffer_load_b16(w, e * 2, 0, 0);
                else v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(w, e * 4, 0, 0));
            }
        } else if constexpr (BF) {
            v = __builtin_bit_cast(row_u16x4, __builtin_amdgcn_raw_buffer_load_b64(w, at * 2, 0, 0));
        } else {
            v = __builtin_bit_cast(row_f32x4, __builtin_amdgcn_raw_buffer_load_b128(w, at * 4, 0, 0));
        }
    }
    __device__ __forceinline__ row_f32x4 get(const QuadPlace &q, bool odd) const {
        row_f32x4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF) f[i] = bf16_to_float(v[i]);
            else f[i] = v[i];
        }
        if (!TINY && odd) {
            if (q.part == 3) f = row_f32x4{f[1], f[2], f[3], 0.f};
            if (q.part == 2) f = row_f32x4{f[2], f[3], 0.f, 0.f};
            if (q.part == 1) f = row_f32x4{f[3], 0.f, 0.f, 0.f};
        }
        return f;
    }
};

// A lane's four values to its place in the window, bfloat16 rounded to nearest even.  stream: with a
// non-temporal hint, for outputs that the caches would not keep.
template <bool BF, bool TINY>
__device__ __forceinline__ void store_row_quad(__amdgpu_buffer_rsrc_t w, const QuadPlace &q, row_f32x4 v, bool odd,
                                               bool stream) {
    const row_u16x4 h = __builtin_bit_cast(row_u16x4, __builtin_convertvector(v, row_bf16x4));
    if constexpr (!TINY) {
        const uint32_t at = odd && q.part ? kNoQuad : q.at;
        if constexpr (BF) {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            if (stream) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, h), w, at * 2, 0, kNonTemporal);
            else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, h), w, at * 2, 0, 0);
        } else {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            if (stream) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), w, at * 4, 0, kNonTemporal);
            else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), w, at * 4, 0, 0);
        }
    }
    if (TINY || (odd && q.part)) {
        const uint32_t at = TINY ? q.at : q.at + 4 - q.part;     // the lane's own first column
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (i < q.part) {
                if constexpr (BF) __builtin_amdgcn_raw_buffer_store_b16(h[i], w, (at + i) * 2, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[i]), w, (at + i) * 4, 0, 0);
            }
        }
    }
}

// Elements [at, at + count) of an array as float32, zeros from `count` on (count <= 0: nothing is
// read); for places with no row of at least four elements around them.
template <bool BF>
__device__ __forceinline__ row_f32x4 load_quad(const void *base, int64_t at, int count) {
    row_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (count >= 4) {
        if constexpr (BF) {
            const row_u16x4 u = *reinterpret_cast<const row_u16x4_any *>(static_cast<const unsigned short *>(base) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = bf16_to_float(u[i]);
        } else {
            v = *reinterpret_cast<const row_f32x4_any *>(static_cast<const float *>(base) + at);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < count) {
                if constexpr (BF) v[i] = bf16_to_float(static_cast<const unsigned short *>(base)[at + i]);
                else v[i] = static_cast<const float *>(base)[at + i];
            }
    }
    return v;
}

// The first `count` of four values to [at, at + count), bfloat16 rounded to nearest even.
template <bool BF>
__device__ __forceinline__ void store_quad(void *base, int64_t at, int count, row_f32x4 v) {
    if constexpr (BF) {
        unsigned short *p = static_cast<unsigned short *>(base) + at;
        const row_u16x4 u = __builtin_bit_cast(row_u16x4, __builtin_convertvector(v, row_bf16x4));
        if (count >= 4) {
            *reinterpret_cast<row_u16x4_any *>(p) = u;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < count) p[i] = u[i];
        }
    } else {
        float *p = static_cast<float *>(base) + at;
        if (count >= 4) {
            *reinterpret_cast<row_f32x4_any *>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < count) p[i] = v[i];
        }
    }
}

// The value of a float32 as it is when stored in bfloat16.
__device__ __forceinline__ float through_bf16(float f) { return static_cast<float>(static_cast<__bf16>(f)); }

// A value that the optimiser takes for a new one: what was computed from it before is not kept in
// registers for its next use.
template <class T>
__device__ __forceinline__ T anew(T v) {
    asm volatile("" : "+v"(v));
    return v;
}

struct AddOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct MaxOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// op over the LANES (a power of two up to 64) lanes of an aligned group, the same value in each
// of them.  Steps inside 16 lanes are DPP moves (quads swap, then mirrors: after each step the
// lanes of a half agree, so a mirror serves as the exchange); 16 and 32 lanes exchange by the
// row swaps of gfx950.  No step goes through LDS.  All lanes of a group must be active.
template <int LANES, class Op>
__device__ __forceinline__ float lanes_reduce(float v, Op op) {
    if constexpr (LANES >= 2) v = op(v, dpp<0xB1>(v));      // quad_perm [1, 0, 3, 2]
    if constexpr (LANES >= 4) v = op(v, dpp<0x4E>(v));      // quad_perm [2, 3, 0, 1]
    if constexpr (LANES >= 8) v = op(v, dpp<0x141>(v));     // row_half_mirror
    if constexpr (LANES >= 16) v = op(v, dpp<0x140>(v));    // row_mirror
    if constexpr (LANES >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (LANES >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}

// The same over THREADS threads of a row: lanes of one wavefront up to 64, the whole workgroup
// (of THREADS threads) above, through `sh` (two buffers of a quad for each wavefront, taken in turn:
// `turn` is the caller's counter).  Up to four values are reduced at once; every thread gets the results:
// it reads one wavefront's quad and joins them by lane exchanges (a read of every wavefront's
// values instead took most of a wide row's time: 16 wavefronts, 48 reads a thread).
template <int THREADS, int N, class Op>
__device__ __forceinline__ void row_reduce(float (&v)[N], Op op, row_f32x4 *sh, int &turn) {
    static_assert(N <= 4, "row_reduce: too many values");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_reduce<(THREADS < 64 ? THREADS : 64)>(v[i], op);
    if constexpr (THREADS > 64) {
        constexpr int kWaves = THREADS / 64;
        row_f32x4 *b = sh + (turn & 1) * kWaves;
        ++turn;
        if ((threadIdx.x & 63) == 0) {
            row_f32x4 mine = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < N; ++i) mine[i] = v[i];
            b[threadIdx.x >> 6] = mine;
        }
        __syncthreads();
        const row_f32x4 one = b[threadIdx.x & (kWaves - 1)];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_reduce<kWaves>(one[i], op);
    }
}

// The sum of a float64 over the same threads, likewise.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xF, 0xF, true),
                            __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xF, 0xF, true));
}
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v) {
    if constexpr (LANES >= 2) v += dpp<0xB1>(v);
    if constexpr (LANES >= 4) v += dpp<0x4E>(v);
    if constexpr (LANES >= 8) v += dpp<0x141>(v);
    if constexpr (LANES >= 16) v += dpp<0x140>(v);
    if constexpr (LANES >= 32) {
        const auto h = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
        const auto l = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
        v = __hiloint2double(h[0], l[0]) + __hiloint2double(h[1], l[1]);
    }
    if constexpr (LANES >= 64) {
        const auto h = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
        const auto l = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
        v = __hiloint2double(h[0], l[0]) + __hiloint2double(h[1], l[1]);
    }
    return v;
}
template <int THREADS>
__device__ __forceinline__ double row_sum(double v, row_f32x4 *sh, int &turn) {
    v = lanes_sum<(THREADS < 64 ? THREADS : 64)>(v);
    if constexpr (THREADS > 64) {
        constexpr int kWaves = THREADS / 64;
        row_f32x4 *b = sh + (turn & 1) * kWaves;
        ++turn;
        if ((threadIdx.x & 63) == 0)
            b[threadIdx.x >> 6] = row_f32x4{__int_as_float(__double2hiint(v)), __int_as_float(__double2loint(v)), 0.f, 0.f};
        __syncthreads();
        const row_f32x4 one = b[threadIdx.x & (kWaves - 1)];
        v = lanes_sum<kWaves>(__hiloint2double(__float_as_int(one[0]), __float_as_int(one[1])));
    }
    return v;
}

template <int THREADS>
constexpr int row_reduce_quads() {
    static_assert((THREADS & (THREADS - 1)) == 0 && THREADS <= 1024, "threads of a row");
    return THREADS > 64 ? 2 * (THREADS / 64) : 1;
}

}  // namespace dgc
