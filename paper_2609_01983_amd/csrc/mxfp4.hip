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
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
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

// Bound by memory: 2^22 x 256 float32 970 us, 4.9 GB, 5.0 TB/s; 150,001 x 400 bfloat16 (a last block of 16) 28.4 us, 5.4 TB/s.
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
// or two for the wavefront.  Up to 1,024 x 1,024 5.8 us a call, 4,096 x 4,096 14.2 (5.3 TB/s; as it stands, by the kernel above, 12.3),
// 16,384 x 16,384 338 (3.6 TB/s; 229).
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

// Back to float32 or bfloat16 (exact but for what lies past float32's range).  2^22 x 256 to bfloat16 433 us, 2.7 GB, 6.3 TB/s.
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

// Few rows: a workgroup makes 16 rows x 16 columns; its wavefronts take steps of four blocks in turn, operands straight
// from memory (each of W is used once), and join their sums in order through LDS.  1 row 1,024 -> 256 4.7 us, the launch
// and two trips to memory.
constexpr int kFewWaves = 8;
constexpr int kFewAhead = 4;                         // steps whose operands are in flight
__global__ __launch_bounds__(kFewWaves * 64) void product_few_kernel(ProductArgs a) {
    __shared__ f32x4 part[kFewWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int cols = (a.N + 15) / 16, steps = (a.blocks + 3) / 4;
    const int c0 = static_cast<int>(blockIdx.x % cols) * 16;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x / cols) * 16;
    const int64_t xr = min(row0 + r, static_cast<int64_t>(a.n) - 1), wr = min(c0 + r, a.N - 1);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = wave; s0 < steps; s0 += kFewWaves * kFewAhead) {
        u32x4 x[kFewAhead], w[kFewAhead];
        uint32_t sx[kFewAhead], sw[kFewAhead];
#pragma unroll
        for (int k = 0; k < kFewAhead; ++k) {
            // (behind the last block its own once more, and 0 for one operand)
            const int b = min(4 * (s0 + k * kFewWaves) + g, a.blocks - 1);
            const int64_t xb = xr * a.blocks + b, wb = wr * a.blocks + b;
            x[k] = *reinterpret_cast<const u32x4 *>(a.X + xb * kBytes);
            w[k] = *reinterpret_cast<const u32x4 *>(a.W + wb * kBytes);
            sx[k] = a.sx[xb];
            sw[k] = a.sw[wb];
        }
#pragma unroll
        for (int k = 0; k < kFewAhead; ++k) {
            const bool there = 4 * (s0 + k * kFewWaves) + g < a.blocks;
            const u32x4 zero = {0, 0, 0, 0};
            acc = mfma16<0, 0>(w[k], there ? sw[k] : kOne, there ? x[k] : zero, there ? sx[k] : kOne, acc);
        }
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        for (int k = 1; k < min(kFewWaves, steps); ++k) acc += part[k][lane];
        store_tile(a, row0 + r, c0 + 4 * g, acc);
    }
}

constexpr int kXcds = 8;
constexpr uint32_t kFar = 0xFFFFFF00u;               // a byte offset past every window

// Many rows: a workgroup of WR x WC wavefronts makes a tile of T, each wavefront 32 R rows of 32 C columns of it.  X and W go
// through LDS, eight blocks (128 bytes a row) a stage, straight from memory, two stages in turn.  A row's eight blocks
// stand in an order that depends on the row, so that the lanes' reads of a block of 16 rows fall on all banks.  What a
// wavefront has made goes out by its own part of LDS, a row's piece of 64 C float32 or bfloat16 numbers in whole lines: stored as
// the lanes have them (16 bytes of each of 32 rows a store) 2^22 rows 256 -> 128 took 703 us, now 459, at 5.9 TB/s.
// 16,384 rows 4,096 -> 4,096 to bfloat16 take 167 us, 3.3 PFLOP/s (the instruction alone, from registers, 7.5): the matrix unit is busy
// 39% of the cycles, LDS 23%, and the wavefronts wait 31% of theirs, for the stage's operands (17 us of them where all came
// from the L2) and at its barrier; a tile's beginning and end, 19 us for a compute unit's four, stand by themselves.  A turn's operands read one
// turn ahead, and over the barrier, were 5%, scales of four stages at once 6%.  One wavefront a SIMD with 128 x 128 of its
// own was slower (195 us), a raised priority for the products made no difference.
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kStageBlocks = 8;
constexpr int kStageBytes = kStageBlocks * kBytes;   // of a row
constexpr int kWaitLds = 0xC07F;                     // s_waitcnt lgkmcnt(0), the other counters as they are
constexpr int kScaleStages = 4;                           // stages whose scales are read together

// Row i of a matrix instruction is column wide_column(i) of the 32, so that a lane's 16 results are consecutive columns.
__device__ __forceinline__ int wide_column(int i) { return (i >> 2 & 1) * 16 + (i >> 3) * 4 + (i & 3); }
__device__ __forceinline__ int wide_row_of(int column) { return (column >> 2 & 3) * 8 + (column >> 4 & 1) * 4 + (column & 3); }

template <int S>
__device__ __forceinline__ f32x16 mfma32(u32x4 w, uint32_t sw, u32x4 x, uint32_t sx, f32x16 acc) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(w), operand(x), acc, 4, 4, S, static_cast<int>(sw), S, static_cast<int>(sx));
}

template <int WR, int WC, int R, int C, bool BF>
struct Tile {
    static constexpr int kWaves = WR * WC, kBlockSize = 64 * kWaves, kRows = WR * R * 32, kCols = WC * C * 32;
    static constexpr int kStage = (kRows + kCols) * kStageBytes, kScales = (kRows + kCols) * kStageBlocks * kScaleStages;     // bytes
    static constexpr int kOut = 32 * (C * 32 * (BF ? 2 : 4) + 16);       // a wavefront's results on their way out
    static_assert(kRows % (8 * kWaves) == 0 && kCols % (8 * kWaves) == 0 && kWaves % 4 == 0, "pieces of a wavefront");
    static constexpr int kScaleRows = (kRows + kCols + kBlockSize - 1) / kBlockSize;       // of a thread
    static constexpr size_t lds(int blocks) {
        const size_t all = blocks <= kStageBlocks ? kStage + kScales / kScaleStages : 2 * kStage + (blocks > kScaleStages * kStageBlocks ? 2 : 1) * kScales;
        return std::max<size_t>(all, kWaves * kOut);
    }
};

template <int WR, int WC, int R, int C, bool BF>
__global__ __launch_bounds__(64 * WR * WC, R * C <= 2 ? 4 : R * C <= 4 ? 3 : 2) void product_tiles_kernel(ProductArgs a, int32_t row_tiles, int32_t col_tiles) {
    using K = Tile<WR, WC, R, C, BF>;
    extern __shared__ uint4 lds[];
    uint8_t *base = reinterpret_cast<uint8_t *>(lds);
    // Workgroup w is on XCD w % 8: each XCD takes consecutive tiles, eight of rows beside each other for each of columns, so that
    // those at work at a time share rows of X and columns of W.
    const int all = row_tiles * col_tiles, per = (all + kXcds - 1) / kXcds;
    const int tile = static_cast<int>(blockIdx.x % kXcds) * per + static_cast<int>(blockIdx.x / kXcds);
    if (static_cast<int>(blockIdx.x / kXcds) >= per || tile >= all) return;
    const int band = tile / (8 * col_tiles), high = min(8, row_tiles - 8 * band), in = tile - band * 8 * col_tiles;
    const int64_t row0 = static_cast<int64_t>(8 * band + in % high) * K::kRows;
    const int c0 = in / high * K::kCols;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, g = lane >> 5;
    const int row_bytes = a.blocks * kBytes;
    const int rows = static_cast<int>(min(static_cast<int64_t>(K::kRows), a.n - row0)), cols = min(K::kCols, a.N - c0);
    const __amdgpu_buffer_rsrc_t wx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.X) + row0 * row_bytes, 0, rows * row_bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t ww = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.W) + static_cast<int64_t>(c0) * row_bytes, 0, cols * row_bytes, 0x00020000);
    const uint8_t *sx = a.sx + row0 * a.blocks, *sw = a.sw + static_cast<int64_t>(c0) * a.blocks;

    // eight rows of 128 bytes an instruction: lane l has row l / 8's place l % 8.  What lies behind the last row or block is 0.
    const int line = wave * 8 + lane / 8;
    const int bx = lane % 8 ^ (line >> 1 & 7), bw = lane % 8 ^ (wide_row_of(line & 31) >> 1 & 7);
    const uint32_t from = static_cast<uint32_t>(line) * row_bytes;
    auto request = [&](int stage, int b0) {
        uint8_t *to = base + stage * K::kStage + wave * 8 * kStageBytes;
        const uint32_t x_at = b0 + bx < a.blocks ? from + (b0 + bx) * kBytes : kFar;
        const uint32_t w_at = b0 + bw < a.blocks ? from + (b0 + bw) * kBytes : kFar;
        typedef __attribute__((address_space(3))) void *lds_ptr;
#pragma unroll
        for (int i = 0; i < K::kRows / 8 / K::kWaves; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wx, (lds_ptr)(to + i * K::kWaves * 8 * kStageBytes), 16,
                                                     x_at == kFar ? kFar : x_at + static_cast<uint32_t>(i * K::kWaves * 8) * row_bytes, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < K::kCols / 8 / K::kWaves; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ww, (lds_ptr)(to + (K::kRows + i * K::kWaves * 8) * kStageBytes), 16,
                                                     w_at == kFar ? kFar : w_at + static_cast<uint32_t>(i * K::kWaves * 8) * row_bytes, 0, 0, 0);
    };
    // The scales of four stages' blocks of the thread's rows, eight bytes a stage; 1 behind the last block, where both operands are
    // 0.  (A stage's at a time cost as much as its operands: 64 rows are 64 lines, whatever is read of each.)
    uint64_t held[K::kScaleRows][kScaleStages];
    const uint32_t x_end = static_cast<uint32_t>(min((a.n - row0) * a.blocks, int64_t{1} << 31));      // of the operand
    const uint32_t w_end = static_cast<uint32_t>(min(static_cast<int64_t>(a.N - c0) * a.blocks, int64_t{1} << 31));
    uint8_t *const scales = base + (a.blocks > kStageBlocks ? 2 : 1) * K::kStage;
    auto request_scales = [&](int b0) {
        const int stages = min(kScaleStages, (a.blocks - b0 + kStageBlocks - 1) / kStageBlocks);
#pragma unroll
        for (int i = 0; i < K::kScaleRows; ++i) {
            const int row = i * K::kBlockSize + static_cast<int>(threadIdx.x);
            const bool of_x = row < K::kRows;
            const int own = of_x ? min(row, rows - 1) : min(row - K::kRows, cols - 1);
            const uint32_t at = own * static_cast<uint32_t>(a.blocks) + b0, end = of_x ? x_end : w_end;
            const uint8_t *from = (of_x ? sx : sw) + at;
#pragma unroll
            for (int q = 0; q < kScaleStages; ++q) {
                typedef uint64_t u64_at1 __attribute__((aligned(1)));
                held[i][q] = 0;
                if (q < stages) {                                        // uniform
                    if (at + (q + 1) * kStageBlocks <= end) {            // the next rows' scales are read along
                        held[i][q] = *reinterpret_cast<const u64_at1 *>(from + q * kStageBlocks);
                    } else {
#pragma unroll
                        for (int k = 0; k < kStageBlocks - 1; ++k)
                            if (at + q * kStageBlocks + k < end) held[i][q] |= static_cast<uint64_t>(from[q * kStageBlocks + k]) << 8 * k;
                    }
                }
            }
        }
    };
    auto keep_scales = [&](int b0) {
        uint8_t *to = scales + b0 / kStageBlocks / kScaleStages % 2 * K::kScales;
#pragma unroll
        for (int q = 0; q < kScaleStages; ++q) {
            const int left = a.blocks - b0 - q * kStageBlocks;
            if (left <= 0) break;                                        // uniform
            const uint64_t kept = left >= kStageBlocks ? ~uint64_t{0} : (uint64_t{1} << 8 * left) - 1;
#pragma unroll
            for (int i = 0; i < K::kScaleRows; ++i) {
                const int row = i * K::kBlockSize + static_cast<int>(threadIdx.x);
                if (row < K::kRows + K::kCols)
                    *reinterpret_cast<uint64_t *>(to + (q * (K::kRows + K::kCols) + row) * kStageBlocks) = (held[i][q] & kept) | (0x7F7F7F7F7F7F7F7Full & ~kept);
            }
        }
    };

    f32x16 acc[R][C];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < C; ++j) acc[i][j] = f32x16{};
    const int x0 = wave / WC * R * 32, w0 = wave % WC * C * 32;          // the wavefront's rows and columns of the tile
    // A turn multiplies two blocks of k; the next turn's operands are on their way from LDS meanwhile, also over the end of a
    // stage: the barrier that hands the stages over stands before its last turn's products.
    u32x4 x[2][R], w[2][C];
    u32x2 fx[R], fw[C];
    const int own_x = x0 + r, own_w = w0 + wide_column(r);
    auto fetch = [&](int stage, int k) {
        const uint8_t *xs = base + stage * K::kStage, *ws = xs + K::kRows * kStageBytes;
        const int place = (2 * k + g ^ (r >> 1 & 7)) * kBytes;
#pragma unroll
        for (int i = 0; i < R; ++i) x[k % 2][i] = *reinterpret_cast<const u32x4 *>(xs + (own_x + 32 * i) * kStageBytes + place);
#pragma unroll
        for (int j = 0; j < C; ++j) w[k % 2][j] = *reinterpret_cast<const u32x4 *>(ws + (own_w + 32 * j) * kStageBytes + place);
    };
    auto fetch_scales = [&](int b0) {
        const int q = b0 / kStageBlocks;
        const uint8_t *sc = scales + q / kScaleStages % 2 * K::kScales + q % kScaleStages * (K::kRows + K::kCols) * kStageBlocks;
#pragma unroll
        for (int i = 0; i < R; ++i) fx[i] = *reinterpret_cast<const u32x2 *>(sc + (own_x + 32 * i) * kStageBlocks);
#pragma unroll
        for (int j = 0; j < C; ++j) fw[j] = *reinterpret_cast<const u32x2 *>(sc + (K::kRows + own_w + 32 * j) * kStageBlocks);
    };
    // loads into LDS are waited for by hand: a barrier alone need not
    auto hand_over = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();
    };
    auto multiply = [&](int k, const uint32_t (&sx)[R], const uint32_t (&sw)[C]) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < C; ++j)
                acc[i][j] = k % 2 ? mfma32<2>(w[k % 2][j], sw[j], x[k % 2][i], sx[i], acc[i][j])
                                  : mfma32<0>(w[k % 2][j], sw[j], x[k % 2][i], sx[i], acc[i][j]);
        // the turns stay in order: without this the compiler reads several turns' operands first and spills
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < C; ++j) asm volatile("" : "+v"(acc[i][j])::"memory");
    };
    constexpr int kStageTurns = kStageBlocks / 2, kGroupBlocks = kScaleStages * kStageBlocks;
    request(0, 0);
    request_scales(0);
    keep_scales(0);
    hand_over();
    if (a.blocks > kStageBlocks) request(1, kStageBlocks);
    if (a.blocks > kGroupBlocks) request_scales(kGroupBlocks);
    fetch_scales(0);
    fetch(0, 0);
    uint32_t nx[R], nw[C];                           // a word of each for two turns
    auto scales_of = [&](int k) {
#pragma unroll
        for (int i = 0; i < R; ++i) nx[i] = fx[i][k / 2] >> 8 * g;
#pragma unroll
        for (int j = 0; j < C; ++j) nw[j] = fw[j][k / 2] >> 8 * g;
    };
    int stage = 0, b0 = 0;
    for (; b0 + kStageBlocks < a.blocks; b0 += kStageBlocks, stage ^= 1) {
#pragma unroll
        for (int k = 0; k < kStageTurns; ++k) {
            if (k % 2 == 0) scales_of(k);
            // a stage's first operands are waited for here: behind the next turn's reads the compiler waits for those too
            if (k == 0) __builtin_amdgcn_s_waitcnt(kWaitLds);
            if (k + 1 < kStageTurns) {
                fetch(stage, k + 1);
            } else {
                const int next = b0 + kStageBlocks;
                if (next % kGroupBlocks == 0) keep_scales(next);
                hand_over();                         // the next stage is there, this one has been read
                fetch_scales(next);
                fetch(stage ^ 1, 0);
                if (next + kStageBlocks < a.blocks) request(stage, next + kStageBlocks);
                if (next % kGroupBlocks == 0 && next + kGroupBlocks < a.blocks) request_scales(next + kGroupBlocks);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(k, nx, nw);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int k = 0; k < kStageTurns; ++k) {
        if (k % 2 == 0) scales_of(k);
        if (k == 0) __builtin_amdgcn_s_waitcnt(kWaitLds);
        if (k + 1 < kStageTurns) fetch(stage, k + 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(k, nx, nw);
        __builtin_amdgcn_sched_barrier(0);
    }
    // a lane's 16 results are columns 16 g .. 16 g + 15 of row r: 32 rows at a time go through the wavefront's own part of LDS,
    // so that a row is written in whole lines
    __syncthreads();
    constexpr int kSize = BF ? 2 : 4, kPer = 16 / kSize, kLine = C * 32 * kSize, kPitch = kLine + 16, kLanes = kLine / 16;
    uint8_t *own = base + wave * K::kOut;
    const int last = a.N - c0 - w0;                                      // columns there are of the wavefront's
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int q = 0; q < 16; q += kPer) {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (BF) {
                        typedef float f32x2 __attribute__((ext_vector_type(2)));
                        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                        v[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc[i][j][q + 2 * e], acc[i][j][q + 2 * e + 1]}), bf16x2));
                    } else {
                        v[e] = __float_as_uint(acc[i][j][q + e]);
                    }
                }
                *reinterpret_cast<u32x4 *>(own + r * kPitch + (32 * j + 16 * g + q) * kSize) = v;
            }
        __builtin_amdgcn_wave_barrier();
        const int64_t first = row0 + x0 + 32 * i;
#pragma unroll
        for (int k = 0; k < (32 * kLanes + 63) / 64; ++k) {
            const int piece = 64 * k + lane, row = piece / kLanes, col = piece % kLanes * kPer;
            if (row >= 32 || first + row >= a.n || col >= last) continue;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(own + row * kPitch + col * kSize);
            char *to = static_cast<char *>(a.T) + ((first + row) * a.N + c0 + w0 + col) * kSize;
            if (last - col >= kPer) {
                *reinterpret_cast<typename std::conditional<BF, u32x4_at2, u32x4_at4>::type *>(to) = v;
            } else {
#pragma unroll
                for (int e = 0; e < kPer - 1; ++e)
                    if (e < last - col) {
                        if constexpr (BF) reinterpret_cast<unsigned short *>(to)[e] = static_cast<unsigned short>(v[e / 2] >> 16 * (e % 2));
                        else reinterpret_cast<uint32_t *>(to)[e] = v[e];
                    }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

int allow_lds(const void *kernel, size_t bytes) {
    if (bytes <= 64 * 1024) return DUALGCN_OK;
    return hip_status(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
}

template <int WR, int WC, int R, int C, bool BF>
int launch_tiles(const ProductArgs &a, hipStream_t s) {
    using K = Tile<WR, WC, R, C, BF>;
    const size_t lds = K::lds(a.blocks);
    const int st = allow_lds(reinterpret_cast<const void *>(&product_tiles_kernel<WR, WC, R, C, BF>), lds);
    if (st) return st;
    const int64_t rows = (static_cast<int64_t>(a.n) + K::kRows - 1) / K::kRows, cols = (a.N + K::kCols - 1) / K::kCols;
    hipLaunchKernelGGL((product_tiles_kernel<WR, WC, R, C, BF>), dim3(static_cast<unsigned>((rows * cols + kXcds - 1) / kXcds * kXcds)),
                       dim3(K::kBlockSize), lds, s, a, static_cast<int32_t>(rows), static_cast<int32_t>(cols));
    return hip_status(hipGetLastError());
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

namespace {

int launch_product(const ProductArgs &a, hipStream_t s) {
    // Which kernel, us (f32 T; few, 256 x 256, 128 x 128, 128 x 64 tiles):
    //   few rows or tiles: 1 row 8,192 -> 1,024 7.9, -, -, 19.0; 64 rows 9.4, -, -, 19.6; 64 rows 4,096 -> 4,096 16.4, 29.8, 14.9, 11.3
    //   the largest, where they still fill the chip and several stages follow each other: 4,096^2 -> 4,096 -, 46.5, 54.3,
    //     68.9; 2^19 1,024 -> 1,024 -, 612, 673, 778; 200,000 512 -> 512 -, 103, 129, 126, but 512 -> 256 -, 52.6, 48.3, 48.1
    //   narrow tiles, where there are few columns or the others leave compute units idle: 10^6 rows 128 -> 16 -, 108, 50, 35;
    //     1,000 rows 4,096 -> 4,096 -, 35.4, 18.9, 18.8, but 2,000 rows -, 37.3, 28.1, 35.2
    auto tiles_of = [&](int64_t rows, int64_t cols) { return (a.n + rows - 1) / rows * ((a.N + cols - 1) / cols); };
    const int64_t cus = device_cus();
    if (a.n <= 32 || tiles_of(16, 16) <= cus) {
        hipLaunchKernelGGL(product_few_kernel, dim3(static_cast<unsigned>(tiles_of(16, 16))), dim3(kFewWaves * 64), 0, s, a);
        return hip_status(hipGetLastError());
    }
    if (a.blocks > kStageBlocks && (a.N > 256 || a.blocks > 2 * kStageBlocks) && 4 * tiles_of(256, 256) >= 3 * cus)
        return a.out_bf16 ? launch_tiles<2, 4, 4, 2, true>(a, s) : launch_tiles<2, 4, 4, 2, false>(a, s);
    if (a.N <= 64 || tiles_of(128, 128) < cus)
        return a.out_bf16 ? launch_tiles<4, 1, 1, 2, true>(a, s) : launch_tiles<4, 1, 1, 2, false>(a, s);
    return a.out_bf16 ? launch_tiles<2, 2, 2, 2, true>(a, s) : launch_tiles<2, 2, 2, 2, false>(a, s);
}

}  // namespace

int launch_update_mxfp4(const void *X, const void *sx, const void *W, const void *sw, void *T, bool out_bf16, int32_t n,
                        int32_t F_in, int32_t F_out, hipStream_t s) {
    ProductArgs a{static_cast<const uint8_t *>(X), static_cast<const uint8_t *>(sx), static_cast<const uint8_t *>(W),
                  static_cast<const uint8_t *>(sw), T, n, F_out, (F_in + kBlock - 1) / kBlock, out_bf16};
    // A launch has fewer than 2^32 threads: 2^22 of the smallest tiles at most, in rows of every size of tile.
    const int64_t most = std::max<int64_t>(1, (int64_t{1} << 21) / ((F_out + 63) / 64)) * 256;
    for (int64_t row = 0; row < n; row += most) {
        a.n = static_cast<int32_t>(std::min<int64_t>(most, n - row));
        const int st = launch_product(a, s);
        if (st) return st;
        a.X += most * a.blocks * kBytes;
        a.sx += most * a.blocks;
        a.T = static_cast<char *>(a.T) + most * F_out * (out_bf16 ? 2 : 4);
    }
    return DUALGCN_OK;
}

}  // namespace dgc
