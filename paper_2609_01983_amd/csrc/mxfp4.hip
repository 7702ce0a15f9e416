// The update phase from 4 bits: e2m1 elements (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives), two a byte,
// with a scale for each 32 consecutive ones, a power of two held as its exponent + 127 in a byte (255: NaN).
//
//   T[v][j] = sum over blocks b of 32:  2^(sx[v][b] + sw[j][b] - 254) sum_{k in b} X4[v][k] W4[j][k]
//
// The matrix instructions of gfx950 take both operands and both scales as they are stored: a lane's 16
// bytes are one block of one row, and one scale goes with it.  Their sums are of float32 quality: of random
// elements with scales within 2^-10 .. 2^10 of each other, 4,096 products were off by 2^-22.5 of the sum of their
// magnitudes at most (by nothing where the scales are alike: the products are multiples of 1/4 up to 36), and
// scales of 2^123 beside 2^-123 make no difference.
//
// W stands as W4[j][k], its products' k along the rows, like X.  The matrix instruction gets W as its first
// operand and X as its second, so that a lane holds four consecutive columns of one row of T.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = DUALGCN_MX_BLOCK;             // 32 elements share a scale
constexpr int kBytes = kBlock / 2;                   // of a block
constexpr uint32_t kOne = 127, kNaN = 255;           // scales

// ------------------------------------------------------------------ quantisers

// The scale of a block whose largest magnitude has the bits `top` (the order of magnitudes is that of their
// bits, infinities and NaN last): the least power of two that brings it to 7 = 1.75 * 2^2 or below, 2^-127 at
// least, 1 for zeros.  What is then between 6 and 7 rounds to 6, so that no element is off by more than half a
// step of its binade; among the powers of two 7 has the least squared error too (normal numbers: 0.0125
// against 0.0133 for 6, which wastes a binade more often, and 0.0132 for 8, which cuts the largest off).
__device__ __forceinline__ uint32_t block_scale(uint32_t top) {
    if (top >= 0x7F800000u) return kNaN;
    if (top == 0) return kOne;
    const int k = static_cast<int>(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return k < 0 ? 0 : k;
}
__device__ __forceinline__ float scale_value(uint32_t s) {               // of any scale but NaN
    return __uint_as_float(s ? s << 23 : 0x400000u);
}

// Eight elements divided by the scale and rounded to nearest even, the first in the lowest bits.  A block that
// is not finite has elements of 0 beside its NaN.
__device__ __forceinline__ uint32_t to_e2m1(const float (&v)[8], uint32_t scale) {
    if (scale == kNaN) return 0;
    const float s = scale_value(scale);
    uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, v[0], v[1], s, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], s, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], s, 3);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
    return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), CTRL, 0xF, 0xF, true));
}

constexpr int kThreads = 256;
constexpr int kLanes = kBlock / 8;                   // lanes of a block: four, eight elements each
constexpr int kTurns = 4;                            // blocks a lane has in flight
constexpr int kGroup = kThreads / kLanes;            // blocks of a workgroup's turn

// A workgroup's blocks [first, first + kGroup kTurns) of the n * blocks of a matrix, row after row: a lane's
// block of turn t, and where it stands.  WHOLE: rows are whole blocks, so that the matrix is one row.
template <bool WHOLE>
struct BlockPlace {
    int64_t first, all;
    int32_t blocks, F;
    int64_t row0;
    uint32_t rem0;
    __device__ __forceinline__ BlockPlace(int64_t n, int32_t blocks_, int32_t F_)
        : first(static_cast<int64_t>(blockIdx.x) * (kGroup * kTurns)), all(n * blocks_), blocks(blocks_), F(F_) {
        row0 = WHOLE ? 0 : first / blocks;
        rem0 = WHOLE ? 0 : static_cast<uint32_t>(first - row0 * blocks);
    }
    // block number, the lane's first element in the matrix and how many of its eight are there
    __device__ __forceinline__ void at(int turn, int64_t &block, int64_t &elem, int &count) const {
        const uint32_t i = turn * kGroup + threadIdx.x / kLanes, sub = 8 * (threadIdx.x % kLanes);
        block = first + i;
        if (WHOLE) {
            elem = block * kBlock + sub;
            count = block < all ? 8 : 0;
            return;
        }
        const uint32_t place = rem0 + i, down = place / static_cast<uint32_t>(blocks);
        const int col = static_cast<int>(place - down * blocks) * kBlock + sub;
        elem = (row0 + down) * F + col;
        count = block < all ? min(8, F - col) : 0;
    }
};

template <bool BF, bool WHOLE>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const void *__restrict__ X, uint8_t *__restrict__ Q,
                                                            uint8_t *__restrict__ scales, int32_t n, int32_t F,
                                                            int32_t blocks) {
    const BlockPlace<WHOLE> place(n, blocks, F);
    row_f32x4 lo[kTurns], hi[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        int64_t block, elem;
        int count;
        place.at(t, block, elem, count);
        if (WHOLE) {
            lo[t] = load_quad<BF>(X, elem, count ? 4 : 0);
            hi[t] = load_quad<BF>(X, elem + 4, count ? 4 : 0);
        } else {
            lo[t] = load_quad<BF>(X, elem, count);
            hi[t] = load_quad<BF>(X, elem + 4, count - 4);
        }
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        int64_t block, elem;
        int count;
        place.at(t, block, elem, count);
        const float v[8] = {lo[t][0], lo[t][1], lo[t][2], lo[t][3], hi[t][0], hi[t][1], hi[t][2], hi[t][3]};
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[i]));
        top = max(top, dpp_u32<0xB1>(top));              // the four lanes of a block
        top = max(top, dpp_u32<0x4E>(top));
        const uint32_t s = block_scale(top), q = to_e2m1(v, s);
        if (block < place.all) {
            *reinterpret_cast<uint32_t *>(Q + block * kBytes + 4 * (threadIdx.x % kLanes)) = q;
            if (threadIdx.x % kLanes == 0) scales[block] = static_cast<uint8_t>(s);
        }
    }
}

// W (rows x cols, float32) transposed: a lane takes a block down a column, 32 loads of which each is a line
// or two for the wavefront.
__global__ __launch_bounds__(kThreads) void quantize_transposed_kernel(const float *__restrict__ W, int32_t rows,
                                                                       int32_t cols, uint8_t *__restrict__ Q,
                                                                       uint8_t *__restrict__ scales, int32_t blocks) {
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), b = blockIdx.y * (kThreads / 64) + (threadIdx.x >> 6);
    if (c >= cols || b >= blocks) return;
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kBlock; ++i) {
        const int r = b * kBlock + i;
        v[i / 8][i % 8] = r < rows ? W[static_cast<int64_t>(r) * cols + c] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kBlock; ++i) top = max(top, magnitude(v[i / 8][i % 8]));
    const uint32_t s = block_scale(top);
    const int64_t at = static_cast<int64_t>(c) * blocks + b;
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = to_e2m1(v[i], s);
    *reinterpret_cast<u32x4 *>(Q + at * kBytes) = q;
    scales[at] = static_cast<uint8_t>(s);
}

// Back to float32 or bfloat16 (exact but for what lies past float32's range).
template <bool BF, bool WHOLE>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const uint8_t *__restrict__ Q,
                                                              const uint8_t *__restrict__ scales, void *__restrict__ X,
                                                              int32_t n, int32_t F, int32_t blocks) {
    const BlockPlace<WHOLE> place(n, blocks, F);
    uint32_t q[kTurns], s[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        int64_t block, elem;
        int count;
        place.at(t, block, elem, count);
        q[t] = s[t] = 0;
        if (count > 0) {
            q[t] = *reinterpret_cast<const uint32_t *>(Q + block * kBytes + 4 * (threadIdx.x % kLanes));
            s[t] = scales[block];
        }
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        int64_t block, elem;
        int count;
        place.at(t, block, elem, count);
        const float f = s[t] == kNaN ? __uint_as_float(0x7FC00000u) : scale_value(s[t]);
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[t], 1.f, 0);
        const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[t], 1.f, 1);
        const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[t], 1.f, 2);
        const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[t], 1.f, 3);
        const row_f32x4 lo = {a[0] * f, a[1] * f, b[0] * f, b[1] * f}, hi = {c[0] * f, c[1] * f, d[0] * f, d[1] * f};
        store_quad<BF>(X, elem, count, lo);
        store_quad<BF>(X, elem + 4, count - 4, hi);
    }
}

// ------------------------------------------------------------------ product

struct ProductArgs {
    const uint8_t *X, *sx, *W, *sw;
    void *T;
    int32_t n, N, blocks;            // N = F_out, blocks of F_in
    bool out_bf16;
};

__device__ __forceinline__ i32x8 operand(u32x4 v) {
    return i32x8{static_cast<int>(v[0]), static_cast<int>(v[1]), static_cast<int>(v[2]), static_cast<int>(v[3]), 0, 0, 0, 0};
}
// 16 x 16 over four blocks of k: lane l has row l % 16 and block l / 16 of both operands; SX, SW: the bytes of the
// scale words that count.
template <int SW, int SX>
__device__ __forceinline__ f32x4 mfma16(u32x4 w, uint32_t sw, u32x4 x, uint32_t sx, f32x4 acc) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w), operand(x), acc, 4, 4, SW, static_cast<int>(sw), SX,
                                                            static_cast<int>(sx));
}

__device__ __forceinline__ void store_tile(const ProductArgs &a, int64_t row, int col, f32x4 v) {
    const int count = a.N - col;
    if (row >= a.n || count <= 0) return;
    if (a.out_bf16) store_quad<true>(a.T, row * a.N + col, count, v);
    else store_quad<false>(a.T, row * a.N + col, count, v);
}

// A workgroup makes 16 rows x 16 columns; its wavefronts take steps of four blocks in turn, operands straight
// from memory, and join their sums in order through LDS.
constexpr int kFewWaves = 8;
__global__ __launch_bounds__(kFewWaves * 64) void product_few_kernel(ProductArgs a) {
    __shared__ f32x4 part[kFewWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int cols = (a.N + 15) / 16, steps = (a.blocks + 3) / 4;
    const int64_t tiles = (static_cast<int64_t>(a.n) + 15) / 16 * cols;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int c0 = static_cast<int>(tile % cols) * 16;
        const int64_t row0 = tile / cols * 16;
        const int64_t xr = min(row0 + r, static_cast<int64_t>(a.n) - 1), wr = min(c0 + r, a.N - 1);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int s = wave; s < steps; s += kFewWaves) {
            const int b = 4 * s + g;
            u32x4 x = {0, 0, 0, 0}, w = {0, 0, 0, 0};
            uint32_t sx = kOne, sw = kOne;
            if (b < a.blocks) {
                const int64_t xb = xr * a.blocks + b, wb = wr * a.blocks + b;
                x = *reinterpret_cast<const u32x4 *>(a.X + xb * kBytes);
                w = *reinterpret_cast<const u32x4 *>(a.W + wb * kBytes);
                sx = a.sx[xb];
                sw = a.sw[wb];
            }
            acc = mfma16<0, 0>(w, sw, x, sx, acc);
        }
        part[wave][lane] = acc;
        __syncthreads();
        if (wave == 0) {
            for (int k = 1; k < min(kFewWaves, steps); ++k) acc += part[k][lane];
            store_tile(a, row0 + r, c0 + 4 * g, acc);
        }
        __syncthreads();
    }
}

}  // namespace

int launch_quantize_mxfp4(const void *X, bool bf16, int32_t n, int32_t F, void *Q, void *scales, hipStream_t s) {
    const int32_t blocks = (F + kBlock - 1) / kBlock;
    const int64_t all = static_cast<int64_t>(n) * blocks;
    uint8_t *q = static_cast<uint8_t *>(Q), *sc = static_cast<uint8_t *>(scales);
    const dim3 grid(static_cast<unsigned>((all + kGroup * kTurns - 1) / (kGroup * kTurns))), block(kThreads);
    if (F % kBlock == 0) {
        if (bf16) hipLaunchKernelGGL((quantize_kernel<true, true>), grid, block, 0, s, X, q, sc, n, F, blocks);
        else hipLaunchKernelGGL((quantize_kernel<false, true>), grid, block, 0, s, X, q, sc, n, F, blocks);
    } else {
        if (bf16) hipLaunchKernelGGL((quantize_kernel<true, false>), grid, block, 0, s, X, q, sc, n, F, blocks);
        else hipLaunchKernelGGL((quantize_kernel<false, false>), grid, block, 0, s, X, q, sc, n, F, blocks);
    }
    return hip_status(hipGetLastError());
}

int launch_quantize_weight_mxfp4(const float *W, int32_t rows, int32_t cols, void *Q, void *scales, hipStream_t s) {
    const int32_t blocks = (rows + kBlock - 1) / kBlock;
    hipLaunchKernelGGL(quantize_transposed_kernel, dim3((cols + 63) / 64, (blocks + kThreads / 64 - 1) / (kThreads / 64)),
                       dim3(kThreads), 0, s, W, rows, cols, static_cast<uint8_t *>(Q), static_cast<uint8_t *>(scales), blocks);
    return hip_status(hipGetLastError());
}

int launch_dequantize_mxfp4(const void *Q, const void *scales, int32_t n, int32_t F, void *X, bool bf16, hipStream_t s) {
    const int32_t blocks = (F + kBlock - 1) / kBlock;
    const int64_t all = static_cast<int64_t>(n) * blocks;
    const uint8_t *q = static_cast<const uint8_t *>(Q), *sc = static_cast<const uint8_t *>(scales);
    const dim3 grid(static_cast<unsigned>((all + kGroup * kTurns - 1) / (kGroup * kTurns))), block(kThreads);
    if (F % kBlock == 0) {
        if (bf16) hipLaunchKernelGGL((dequantize_kernel<true, true>), grid, block, 0, s, q, sc, X, n, F, blocks);
        else hipLaunchKernelGGL((dequantize_kernel<false, true>), grid, block, 0, s, q, sc, X, n, F, blocks);
    } else {
        if (bf16) hipLaunchKernelGGL((dequantize_kernel<true, false>), grid, block, 0, s, q, sc, X, n, F, blocks);
        else hipLaunchKernelGGL((dequantize_kernel<false, false>), grid, block, 0, s, q, sc, X, n, F, blocks);
    }
    return hip_status(hipGetLastError());
}

int launch_update_mxfp4(const void *X, const void *sx, const void *W, const void *sw, void *T, bool out_bf16, int32_t n,
                        int32_t F_in, int32_t F_out, hipStream_t s) {
    const ProductArgs a{static_cast<const uint8_t *>(X), static_cast<const uint8_t *>(sx), static_cast<const uint8_t *>(W),
                        static_cast<const uint8_t *>(sw), T, n, F_out, (F_in + kBlock - 1) / kBlock, out_bf16};
    const int64_t tiles = (static_cast<int64_t>(n) + 15) / 16 * ((F_out + 15) / 16);
    hipLaunchKernelGGL(product_few_kernel, dim3(static_cast<unsigned>(std::min<int64_t>(tiles, 1 << 20))), dim3(kFewWaves * 64), 0, s, a);
    return hip_status(hipGetLastError());
}

}  // namespace dgc
