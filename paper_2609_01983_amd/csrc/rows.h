// Device helpers of the row-wise operators (norm.hip, distill.hip, fp8.hip): four
// consecutive elements of a float32 or bfloat16 row at any alignment, and sums and maxima
// over the 2^k lanes that share a row.
#pragma once

#include "internal.h"

#include <type_traits>

namespace dgc {

typedef float row_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 row_bf16x4 __attribute__((ext_vector_type(4)));
// rows may start at any element: the loads and stores below need no more than its alignment
typedef float row_f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short row_u16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short row_u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_to_float(unsigned short b) {
    return __uint_as_float(static_cast<uint32_t>(b) << 16);
}

// A lane's four consecutive columns of a row of F: `col` the first, `at` where they are read
// (the row's last four where the row ends inside them, so that every load is whole and none is
// under a condition: the compiler then keeps all loads of a row in flight), `shift` by how many
// columns that is early, `count` how many of the four the row has (<= 0: none).
struct QuadPlace {
    int at, shift, count;
    __device__ __forceinline__ void set(int col, int F) {
        at = F < 4 ? 0 : (col < F - 4 ? col : F - 4);
        shift = col - at;
        count = F - col;
    }
};

// Four elements as stored, and as float32.  TINY: rows of fewer than four elements.
template <bool BF, bool TINY>
struct RawRowQuad {
    typename std::conditional<BF, row_u16x4, row_f32x4>::type v;

    __device__ __forceinline__ void load(const void *base, int64_t row_at, const QuadPlace &q) {
        if constexpr (TINY) {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                v[i] = 0;
                if (i < q.count) {
                    if constexpr (BF) v[i] = static_cast<const unsigned short *>(base)[row_at + i];
                    else v[i] = static_cast<const float *>(base)[row_at + i];
                }
            }
            v[3] = 0;
        } else if constexpr (BF) {
            v = *reinterpret_cast<const row_u16x4_any *>(static_cast<const unsigned short *>(base) + row_at + q.at);
        } else {
            v = *reinterpret_cast<const row_f32x4_any *>(static_cast<const float *>(base) + row_at + q.at);
        }
    }
    // ragged: the row has fewer columns than its lanes have places (the same for every lane)
    __device__ __forceinline__ row_f32x4 get(const QuadPlace &q, bool ragged) const {
        row_f32x4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF) f[i] = bf16_to_float(v[i]);
            else f[i] = v[i];
        }
        if (!TINY && ragged) {
            if (q.shift & 1) f = row_f32x4{f[1], f[2], f[3], 0.f};
            if (q.shift & 2) f = row_f32x4{f[2], f[3], 0.f, 0.f};
            if (q.shift >= 4) f = row_f32x4{0.f, 0.f, 0.f, 0.f};
        }
        return f;
    }
};

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
// (of THREADS threads) above, through `sh` (two buffers of THREADS / 64 * N floats, taken in turn:
// `turn` is the caller's counter).  N values are reduced at once; every thread gets the results.
template <int THREADS, int N, class Op>
__device__ __forceinline__ void row_reduce(float (&v)[N], Op op, float *sh, int &turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_reduce<(THREADS < 64 ? THREADS : 64)>(v[i], op);
    if constexpr (THREADS > 64) {
        constexpr int kWaves = THREADS / 64;
        constexpr int kMost = 4;                      // values a buffer has room for
        static_assert(N <= kMost, "row_reduce: too many values");
        float *b = sh + (turn & 1) * kWaves * kMost;
        ++turn;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) b[(threadIdx.x >> 6) * kMost + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = b[i];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) s = op(s, b[w * kMost + i]);
            v[i] = s;
        }
    }
}

template <int THREADS>
constexpr int row_reduce_floats() {
    return THREADS > 64 ? 2 * (THREADS / 64) * 4 : 1;
}

}  // namespace dgc
