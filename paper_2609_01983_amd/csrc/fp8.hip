// The update phase in 8 bits: T = X W from e4m3 operands (bias 7, largest 448, no infinity) with
// a float32 scale for each block of 128, and the quantisers that make them.
//
//   T[v][j] = sum over blocks b of F_in:  sx[v][b] sw[j / 128][b] sum_{k in b} X8[v][k] W8[j][k]
//
// The operands are widened to bfloat16, which holds every e4m3 number exactly, and a block is four
// v_mfma_f32_16x16x32_bf16 into fresh float32 accumulators, whose sums enter the running ones with one
// factor a row and block.  The 8-bit matrix instructions would halve the matrix unit's time, but
// their sums are not float32: measured on blocks of 128 random products, 1.5e-5 relative to the exact sums and
// up to 2^-12 of the largest product, against 8.5e-9 here, and the product is bound by memory
// for any F_out up to a few hundred (2 F_in F_out flops for F_in + 4 F_out bytes a row).
//
// W stands as W8[j][k], the products' k along the rows, like X: both operands are read as 16 bytes
// a lane.  The matrix instruction gets W as its first operand and X as its second, so that a lane
// holds four consecutive columns of one row of T: one scale a lane, and stores of 16 bytes.
//
// The kernel streams X: a workgroup keeps the W of its up to 128 columns in LDS, widened once, for
// its whole life, and its wavefronts request a tile's next block of X while the current one is
// multiplied.
#include "rows.h"

#include <algorithm>

namespace dgc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = kFp8Block;                    // 128 elements share a scale

// Eight e4m3 numbers as bfloat16 (exact).
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// ------------------------------------------------------------------ quantisers

// The least power of two that brings `amax` to 448 = 1.75 * 2^8 or below (2^-126 at least; 1 for a
// block of zeros), by its exponent: dividing by it is exact.
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    if (u == 0) return 0;
    const int k = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return k < -126 ? -126 : k;
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float(static_cast<uint32_t>(k + 127) << 23); }

// |x|, and 0 for infinities and NaN: they have no part in a block's scale (both become NaN)
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;
}

__device__ __forceinline__ uint32_t to_e4m3(row_f32x4 v) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], r, true);
    return static_cast<uint32_t>(r);
}

// A workgroup takes 16 rows, 16 lanes each, and up to eight blocks of them (blockIdx.y); a lane has
// the elements from 4 l and 64 + 4 l on of a block, and two blocks' loads are in flight.  Bound by
// memory: 2^21 x 256 464 us from float32, 280 from bfloat16 (5.8 TB/s); 200,003 x 528 bfloat16 69 to 73 us (4.3 to 4.6 TB/s: rows
// of 528 bytes end inside lines, which are written twice, 128 MB for 106).
constexpr int kQuantThreads = 256;
constexpr int kQuantLanes = 16;
constexpr int kQuantRows = kQuantThreads / kQuantLanes;
constexpr int kQuantBlocks = 8;
template <bool BF, bool TINY>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(const void *__restrict__ X, uint8_t *__restrict__ Q,
                                                                 float *__restrict__ scales, int32_t n, int32_t F,
                                                                 int32_t blocks) {
    const int l = threadIdx.x % kQuantLanes, g = threadIdx.x / kQuantLanes;
    const bool odd = F & 3;
    const int b0 = blockIdx.y * kQuantBlocks, b1 = min(blocks, b0 + kQuantBlocks);
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kQuantRows; row0 < n;
         row0 += static_cast<int64_t>(gridDim.x) * kQuantRows) {
        const int64_t rows = min(static_cast<int64_t>(kQuantRows), n - row0);
        const __amdgpu_buffer_rsrc_t wx = row_window<BF>(X, row0 * F, rows * F);
        const __amdgpu_buffer_rsrc_t wq = __builtin_amdgcn_make_buffer_rsrc(Q + row0 * F, 0, static_cast<int>(rows * F), 0x00020000);
        for (int b = b0; b < b1; b += 2) {
            QuadPlace at[2][2];
            RawRowQuad<BF, TINY> raw[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int first = (b + j) * kBlock + 64 * h + 4 * l;
                    at[j][h].set(static_cast<uint32_t>(g) * F, b + j < b1 ? first : F, F);
                    raw[j][h].load(wx, at[j][h].at, at[j][h].count);
                }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                row_f32x4 v[2];
                float amax = 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v[h] = raw[j][h].get(at[j][h], odd);
#pragma unroll
                    for (int i = 0; i < 4; ++i) amax = fmaxf(amax, finite_abs(v[h][i]));
                }
                amax = lanes_reduce<kQuantLanes>(amax, MaxOp());
                const int k = scale_exponent(amax);
                const float inv = power_of_two(-k);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t q = to_e4m3(v[h] * inv);
                    const QuadPlace &p = at[j][h];
                    const bool part = TINY || (odd && p.part);
                    if constexpr (!TINY) __builtin_amdgcn_raw_buffer_store_b32(q, wq, part ? kNoQuad : p.at, 0, 0);
                    if (part) {
                        const uint32_t to = TINY ? p.at : p.at + 4 - p.part;
#pragma unroll
                        for (int i = 0; i < 3; ++i)
                            if (i < p.part) __builtin_amdgcn_raw_buffer_store_b8(static_cast<uint8_t>(q >> 8 * i), wq, to + i, 0, 0);
                    }
                }
                if (l == 0 && g < rows && b + j < b1) scales[(row0 + g) * blocks + b + j] = power_of_two(k);
            }
        }
    }
}

// A block of 128 x 128 of W (rows x cols, float32), quantised into Q as it stands or transposed (through
// LDS, so that both sides' rows are whole lines).  1,024 x 1,024 11 us, 8,192 x 8,192 68 us (4.9 TB/s); done once a model.
constexpr int kTilePad = kBlock + 4;                 // bytes of a transposed row in LDS
__global__ __launch_bounds__(kQuantThreads) void quantize_weight_kernel(const float *__restrict__ W, int32_t rows,
                                                                        int32_t cols, int transpose,
                                                                        uint8_t *__restrict__ Q,
                                                                        float *__restrict__ scales) {
    __shared__ uint8_t tile[kBlock * kTilePad];
    __shared__ float top[kQuantThreads / 64];
    const int r0 = blockIdx.y * kBlock, c0 = blockIdx.x * kBlock;
    const int q = threadIdx.x % 32, rr = threadIdx.x / 32;        // a wavefront reads two rows
    constexpr int kRows = kBlock / (kQuantThreads / 32);          // rows a thread has: 16
    row_f32x4 v[kRows];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int r = r0 + rr + i * (kQuantThreads / 32), c = c0 + 4 * q;
        v[i] = load_quad<false>(W, static_cast<int64_t>(r) * cols + c, r < rows ? cols - c : 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) amax = fmaxf(amax, finite_abs(v[i][j]));
    }
    amax = lanes_reduce<64>(amax, MaxOp());
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / 64; ++w) amax = fmaxf(amax, top[w]);
    const int k = scale_exponent(amax);
    const float inv = power_of_two(-k);
    // the tile as it is written: [row of Q][k]
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t e = to_e4m3(v[i] * inv);
        const int r = rr + i * (kQuantThreads / 32);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = transpose ? (4 * q + j) * kTilePad + r : r * kTilePad + 4 * q + j;
            tile[at] = static_cast<uint8_t>(e >> 8 * j);
        }
    }
    __syncthreads();
    const int qrows = transpose ? cols : rows, qcols = transpose ? rows : cols;
    const int qr0 = transpose ? c0 : r0, qc0 = transpose ? r0 : c0;
    for (int i = threadIdx.x; i < kBlock * kBlock; i += kQuantThreads) {
        const int r = i / kBlock, c = i % kBlock;
        if (qr0 + r < qrows && qc0 + c < qcols) Q[static_cast<int64_t>(qr0 + r) * qcols + qc0 + c] = tile[r * kTilePad + c];
    }
    if (threadIdx.x == 0) {
        const int sb = (qcols + kBlock - 1) / kBlock;
        scales[static_cast<int64_t>(qr0 / kBlock) * sb + qc0 / kBlock] = power_of_two(k);
    }
}

// ------------------------------------------------------------------ product

struct ProductArgs {
    const uint8_t *X, *W;
    const float *sx, *sw;
    void *T;
    int32_t n, K, N, blocks;         // K = F_in, N = F_out, blocks of K
    bool out_bf16;
};

// A lane's 32 bytes of block b of row `row` (X8 or W8 with rows of K): chunks of 16 at 16 g and
// 64 + 16 g of the block, four steps of eight k each.  Both operands give a step the same k, so a
// block's sum is right whatever their order.  Chunks behind the row's end are zeroed by get().
constexpr int kSteps = kBlock / 32;
struct Fragment {
    u32x4 lo, hi;
    // from a window that starts at the block's first byte of the tile's first row; `at`: the row's offset + 16 g
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t w, uint32_t at) {
        lo = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(w, at, 0, 0));
        hi = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(w, at + 64, 0, 0));
    }
    __device__ __forceinline__ void load(const uint8_t *base, int64_t row, int K, int b, int g) {
        const uint8_t *r = base + row * K;
        const int k = b * kBlock + 16 * g;
        lo = *reinterpret_cast<const u32x4 *>(r + (k < K ? k : 0));
        hi = *reinterpret_cast<const u32x4 *>(r + (k + 64 < K ? k + 64 : 0));
    }
    __device__ __forceinline__ void get(int K, int b, int g, bf16x8 (&out)[kSteps]) const {
        u32x4 x = lo, y = hi;
        if (K % kBlock) {                                // uniform
            const int k = b * kBlock + 16 * g;
            const u32x4 zero = {0, 0, 0, 0};
            x = k < K ? lo : zero;
            y = k + 64 < K ? hi : zero;
        }
        out[0] = widen(x[0], x[1]);
        out[1] = widen(x[2], x[3]);
        out[2] = widen(y[0], y[1]);
        out[3] = widen(y[2], y[3]);
    }
};

// The product x w of two scales as f g, g a power of two and f a normal number.  x w itself may be no float32 (it
// overflows, or falls among the subnormal numbers and loses bits) though its product with a block's sum, 0 or between
// 2^-18 and 2^25, is one: the sum is multiplied by g first, which is exact.  Where x w is between 2^-100 and 2^100, g is 1.
struct Scales {
    float f, g;
    __device__ __forceinline__ Scales(float x, float w) {
        f = x * w;
        g = 1.f;
        const float a = fabsf(f);
        if (!(a >= 0x1p-100f && a <= 0x1p100f) && x != 0.f && w != 0.f) {
            const int e = __builtin_amdgcn_frexp_expf(x) + __builtin_amdgcn_frexp_expf(w);      // 0 of infinity and NaN
            const int eg = e - min(max(e, -100), 100);
            f = __builtin_amdgcn_ldexpf(__builtin_amdgcn_frexp_mantf(x) * __builtin_amdgcn_frexp_mantf(w), e - eg);
            g = __builtin_amdgcn_ldexpf(1.f, min(max(eg, -126), 127));           // past these the result is 0 or infinite
        }
    }
};
// Is a scale of X outside [2^-85, 2^85], one of W outside [2^-40, 2^40]?  Two inside have a product that may be used as it is:
// a normal number.  (Zeros, infinities and NaN may too.)  X has the wider range: gradients are small, weights are not.
constexpr int kFarX = 85, kFarW = 40;
template <int E>
__device__ __forceinline__ bool far_scale(float x) {
    return static_cast<uint32_t>(__builtin_amdgcn_frexp_expf(x) + E - 1) > 2u * E - 1u;
}

__device__ __forceinline__ void store_tile(const ProductArgs &a, int64_t row, int col, int last, f32x4 v) {
    const int count = last - col;
    if (row >= a.n || count <= 0) return;
    if (a.out_bf16) store_quad<true>(a.T, row * a.N + col, count, v);
    else store_quad<false>(a.T, row * a.N + col, count, v);
}

// Workgroups of eight wavefronts, 32 rows each, with W of CT tiles of 16 columns in LDS.  Measured:
// 2^22 rows 256 -> 128 float32 652 us a call, 3.25 GB, 5.0 TB/s, bound by memory; 2^19 rows 1,024 -> 1,024 1.55 ms, 710 TFLOP/s,
// and 200,003 rows 528 -> 200 84 us, 500 TFLOP/s: there the matrix unit is busy 31 and 33% of the time, the vector unit
// 34 and 43% (widening X, scaling sums), LDS 16 and 18%, by their counters, and the wavefronts wait for each
// other's turns.  Taking all registers where W leaves room for one workgroup a CU, for W's fragments ahead of their products,
// was 1 to 3% faster for 528 -> 200, 512 -> 200 and 400 -> 400 and 1 to 2% slower for 512 -> 512, 672 -> 128 and 1,024 -> 256.
// Requests of X two to four blocks ahead, or W's reads ordered a tile ahead of its products, made wide products 2%
// faster and narrow ones 3 to 15% slower.
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kRowTiles = 2;
constexpr int kRows = 16 * kRowTiles;                // of a wavefront
constexpr int kRowsPerBlock = kWaves * kRows;
// bfloat16 elements of a tile of 16 columns in LDS: [block][step][g][column][8], so that a wavefront's
// read of an operand is 1,024 consecutive bytes (rows of W side by side, padded by 16 bytes, had half
// of their reads' cycles in bank conflicts).
__host__ __device__ __forceinline__ int lds_tile(int blocks) { return blocks * kBlock * 16; }

// The slices of a row tile run at one time on one XCD and read its X from that L2: workgroups go to
// the XCDs in turn, so number w has XCD w % 8, slice w / 8 % slices, and the tiles w / (8 slices) 8 + w % 8, ...
// (with the slices of a tile on different XCDs, X came from beyond the L2 once a slice: 2^20 rows
// 512 -> 512 933 us against 822, 1,024 -> 256 1,120 against 842).  `side` is that 8, or 1 where the
// tiles are too few to give each XCD its share.
constexpr int kXcds = 8;
constexpr int kMostBlocks = 8;                       // F_in up to 1,024
// The 32 rows of a wavefront from row0 on once more, a tile of 16 x 16 at a time, with scales of any size; `w`: W in
// LDS.  Apart from the main loop, so that it takes few of its registers: tests for such scales alone cost
// (us with and without) 2^22 rows 32 -> 16 100, 93, 2^20 128 -> 64 64, 60, 200,003 528 -> 200 82, 80, nothing where rows are wider.
// Rows that need it take 1.3 to 4.4 times as long (all of 2^22 256 -> 128 1,530, 645; of 2^19 1,024 -> 1,024 6,800, 1,545).
// With a second way beside the main loop's products, whose registers then bound the kernel, 528 -> 200 took 91.
template <int CT>
__device__ __forceinline__ void product_of_far_scales(const ProductArgs &a, const __bf16 *w, int64_t row0, int c0, int turn,
                                                      const float (&column_scales)[2][kMostBlocks]) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, last = min(a.N, c0 + 16 * CT);
#pragma unroll 1
    for (int tile = 0; tile < kRowTiles * CT; ++tile) {
        const int c = tile % CT;
        const int64_t row = row0 + tile / CT * 16 + r, xr = min(row, static_cast<int64_t>(a.n) - 1);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int b = 0; b < a.blocks; ++b) {
            Fragment x;
            x.load(a.X, xr, a.K, b, g);
            bf16x8 xs[kSteps];
            x.get(a.K, b, g, xs);
            const __bf16 *p = w + c * lds_tile(a.blocks) + b * kSteps * 512 + lane * 8;
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8 *>(p + 512 * k), xs[k], s, 0, 0, 0);
            const Scales f(a.sx[xr * a.blocks + b], column_scales[c < turn ? 0 : 1][b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = fmaf(f.f, s[i] * f.g, acc[i]);
        }
        store_tile(a, row, c0 + 16 * c + 4 * g, last, acc);
    }
}

// (the second bound: two workgroups a CU, three for one tile)
template <int CT>
__global__ __launch_bounds__(kThreads, CT == 1 ? 6 : CT <= 4 ? 4 : 2) void product_kernel(ProductArgs a, int32_t slices, int32_t side) {
    extern __shared__ uint4 lds[];
    __bf16 *w = reinterpret_cast<__bf16 *>(lds);
    const int tile_elems = lds_tile(a.blocks);
    const int c0 = static_cast<int>(blockIdx.x) / side % slices * 16 * CT;
    const int64_t stride = gridDim.x / slices;
    const int64_t tiles = (static_cast<int64_t>(a.n) + kRowsPerBlock - 1) / kRowsPerBlock;
    int64_t tile = static_cast<int64_t>(blockIdx.x) / (side * slices) * side + blockIdx.x % side;
    if (tile >= tiles) return;                       // the grid has a whole number of tiles for each XCD
    // W of the columns [c0, c0 + 16 CT), zeros past F_out and past F_in: 16 bytes of W8 are two
    // steps of a lane group
    const int per_row = a.blocks * kBlock / 16;
    for (int i = threadIdx.x; i < 16 * CT * per_row; i += kThreads) {
        const int c = i / (16 * per_row) * 16 + i % 16, chunk = i / 16 % per_row, k = chunk * 16;
        u32x4 v = {0, 0, 0, 0};
        if (c0 + c < a.N && k < a.K) v = *reinterpret_cast<const u32x4 *>(a.W + static_cast<int64_t>(c0 + c) * a.K + k);
        const int b = chunk / 8, half = chunk % 8 / 4, g = chunk % 4;
        __bf16 *to = w + c / 16 * tile_elems + (((b * kSteps + 2 * half) * 4 + g) * 16 + c % 16) * 8;
        *reinterpret_cast<bf16x8 *>(to) = widen(v[0], v[1]);
        *reinterpret_cast<bf16x8 *>(to + 4 * 16 * 8) = widen(v[2], v[3]);
    }
    // the columns' scales by LDS too: a load of them among those of X would wait for the next block's X,
    // the loads being answered in order
    __shared__ float column_scales[2][kMostBlocks];
    if (static_cast<int>(threadIdx.x) < 2 * a.blocks) {
        const int next = threadIdx.x / a.blocks, b = threadIdx.x % a.blocks;
        const int row = min(c0 / kBlock + next, (a.N + kBlock - 1) / kBlock - 1);
        column_scales[next][b] = a.sw[static_cast<int64_t>(row) * a.blocks + b];
    }
    __syncthreads();

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    // the columns' scales: tiles of 16 columns from `turn` on are in the next block of 128
    const int turn = (kBlock - c0 % kBlock) / 16;
    const int last = min(a.N, c0 + 16 * CT);

    // A tile's rows as windows, from block b on: rows behind the last are zeros, and lanes address
    // them with 32 bits (256 rows of at most 1,024 bytes).
    Fragment in[kRowTiles];
    float sc[kRowTiles], sn[kRowTiles];
    uint32_t at[kRowTiles];
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t) at[t] = wave * kRows + t * 16 + r;
    auto request = [&](int64_t tile, int b) {
        const int64_t row0 = tile * kRowsPerBlock;
        const int64_t rows = max(int64_t{0}, min(static_cast<int64_t>(kRowsPerBlock), a.n - row0));
        const __amdgpu_buffer_rsrc_t wx = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t *>(a.X) + row0 * a.K + b * kBlock, 0,
            rows ? static_cast<int>(rows * a.K - b * kBlock) : 0, 0x00020000);
        const __amdgpu_buffer_rsrc_t ws = row_window<false>(a.sx, row0 * a.blocks + b, rows ? rows * a.blocks - b : 0);
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) {
            in[t].load(wx, at[t] * a.K + 16 * g);
            sn[t] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ws, at[t] * a.blocks * 4, 0, 0));
        }
    };
    request(tile, 0);
    for (; tile < tiles; tile += stride) {
        f32x4 acc[kRowTiles][CT];
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        bool far = false;
        for (int b = 0; b < a.blocks; ++b) {
            bf16x8 x[kRowTiles][kSteps];
#pragma unroll
            for (int t = 0; t < kRowTiles; ++t) {
                in[t].get(a.K, b, g, x[t]);
                sc[t] = sn[t];
                far |= far_scale<kFarX>(sc[t]);
            }
            // the next block of this tile, or the first of the next tile (past the last: zeros), into the
            // registers that the widened ones have left
            const bool more = b + 1 < a.blocks;
            request(more ? tile : tile + stride, more ? b + 1 : 0);
            const float sw0 = column_scales[0][b], sw1 = column_scales[1][b];
            far |= far_scale<kFarW>(sw0);
            far |= far_scale<kFarW>(sw1);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const __bf16 *p = w + c * tile_elems + b * kSteps * 512 + lane * 8;
                f32x4 s[kRowTiles];
#pragma unroll
                for (int t = 0; t < kRowTiles; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    const bf16x8 wf = *reinterpret_cast<const bf16x8 *>(p + 512 * k);
#pragma unroll
                    for (int t = 0; t < kRowTiles; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, x[t][k], s[t], 0, 0, 0);
                }
                const float swc = c < turn ? sw0 : sw1;
#pragma unroll
                for (int t = 0; t < kRowTiles; ++t) {
                    const float f = sc[t] * swc;
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][c][i] = fmaf(f, s[t][i], acc[t][c][i]);
                }
            }
        }
        const int64_t row0 = tile * kRowsPerBlock;
        if (__ballot(far)) {                         // scales whose products may not be used as they are: not from acc
            product_of_far_scales<CT>(a, w, row0 + wave * kRows, c0, turn, column_scales);
            continue;
        }
        const int64_t elems = min(static_cast<int64_t>(kRowsPerBlock), a.n - row0) * a.N;
        const int own = anew(4 * g);                 // the places are worked out here, not kept over the tiles
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const int col = c0 + 16 * c + own;
                QuadPlace to;
                to.count = last - col;
                to.part = to.count > 0 && to.count < 4 ? to.count : 0;
                to.at = to.count > 0 ? at[t] * a.N + col - (to.part ? 4 - to.part : 0) : kNoQuad;
                to.col = 0;
                if (a.out_bf16) store_row_quad<true, false>(row_window<true>(a.T, row0 * a.N, elems), to, acc[t][c], a.N & 3, false);
                else store_row_quad<false, false>(row_window<false>(a.T, row0 * a.N, elems), to, acc[t][c], a.N & 3, false);
            }
    }
}

// Few rows: a workgroup makes 16 rows x 16 columns, its wavefronts take the blocks of K in turn
// (W8 straight from memory: each of it is used once) and join their sums in order through LDS.
// 1 row 1,024 -> 256: 3.2 us, the launch and two trips to memory.
__global__ __launch_bounds__(kThreads) void product_few_kernel(ProductArgs a) {
    __shared__ f32x4 part[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int c0 = blockIdx.x * 16;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * 16;
    const int64_t xr = min(row0 + r, static_cast<int64_t>(a.n) - 1), wr = min(c0 + r, a.N - 1);
    const float *sw = a.sw + static_cast<int64_t>(c0 / kBlock) * a.blocks;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int b = wave; b < a.blocks; b += kWaves) {
        Fragment x, w;
        x.load(a.X, xr, a.K, b, g);
        w.load(a.W, wr, a.K, b, g);
        const Scales f(a.sx[xr * a.blocks + b], sw[b]);
        bf16x8 xs[kSteps], ws[kSteps];
        x.get(a.K, b, g, xs);
        w.get(a.K, b, g, ws);
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ws[k], xs[k], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(f.f, s[i] * f.g, acc[i]);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        for (int k = 1; k < min(kWaves, a.blocks); ++k) acc += part[k][lane];
        store_tile(a, row0 + r, c0 + 4 * g, min(a.N, c0 + 16), acc);
    }
}

int allow_lds(const void *kernel, size_t bytes) {
    if (bytes <= 64 * 1024) return DUALGCN_OK;
    return hip_status(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
}

// At most kMostCols tiles of 16 columns a slice: what the accumulators and (by F_in) a CU's LDS hold.
constexpr int kMostCols = 8;
constexpr size_t kLds = 160 * 1024 - 2 * kMostBlocks * sizeof(float);   // beside the scales
// Workgroups for each place on the chip, at most.  Where W takes up to 64 KB of LDS it is laid out quickly and
// many short-lived workgroups keep the memory busier; a larger one has to serve many rows.  us with 2 and 16:
// 2^22 rows 256 -> 128 676, 650; 2^22 256 -> 64 460, 429; 2^20 256 -> 256 334, 294; and past 64 KB
// 2^21 384 -> 128 406, 414; 2^21 512 -> 128 451, 481; 2^20 1,024 -> 256 839, 903.
inline int64_t over(size_t lds) { return lds <= 64 * 1024 ? 16 : 2; }

// Row tiles from which the slices of one share an XCD.  Fewer leave XCDs idle or with an uneven share (us side
// by side and over the XCDs in turn, 1,024 -> 1,024: 1,000 rows 27.8 and 15.8, 16,000 rows 63.6 and 62.2;
// past that the shared L2 wins).
constexpr int64_t kSideTiles = 64;

template <int CT>
int launch_product(const ProductArgs &a, int slices, hipStream_t s) {
    const size_t lds = static_cast<size_t>(CT) * lds_tile(a.blocks) * sizeof(uint16_t);
    const int st = allow_lds(reinterpret_cast<const void *>(&product_kernel<CT>), lds);
    if (st) return st;
    const int64_t tiles = (static_cast<int64_t>(a.n) + kRowsPerBlock - 1) / kRowsPerBlock;
    // registers: up to 128 a thread for four tiles of columns, hence two workgroups a CU
    const int64_t resident = static_cast<int64_t>(device_cus()) * (CT <= 4 && 2 * lds <= kLds ? 2 : 1);
    // row tiles at a time, a whole number for each XCD
    const int side = tiles >= kSideTiles ? kXcds : 1;
    const int64_t per = std::max<int64_t>(1, (std::min<int64_t>(tiles, over(lds) * resident / slices) + side - 1) / side) * side;
    hipLaunchKernelGGL((product_kernel<CT>), dim3(static_cast<unsigned>(per * slices)), dim3(kThreads), lds, s, a, slices, side);
    return hip_status(hipGetLastError());
}

// Slices of equal width: as few as fit, then as narrow as those need.
int launch_slices(const ProductArgs &a, int most, hipStream_t s) {
    const int cols = (a.N + 15) / 16;
    while (most > 1 && static_cast<size_t>(most) * lds_tile(a.blocks) * sizeof(uint16_t) > kLds) --most;
    const int slices = (cols + most - 1) / most;
    switch ((cols + slices - 1) / slices) {
        case 1: return launch_product<1>(a, slices, s);
        case 2: return launch_product<2>(a, slices, s);
        case 3: return launch_product<3>(a, slices, s);
        case 4: return launch_product<4>(a, slices, s);
        case 5: return launch_product<5>(a, slices, s);
        case 6: return launch_product<6>(a, slices, s);
        case 7: return launch_product<7>(a, slices, s);
        default: return launch_product<8>(a, slices, s);
    }
}

}  // namespace

int launch_quantize(const void *X, bool bf16, int32_t n, int32_t F, void *Q, float *scales, hipStream_t s) {
    const int32_t blocks = (F + kBlock - 1) / kBlock;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((static_cast<int64_t>(n) + kQuantRows - 1) / kQuantRows, 1 << 20)),
                    (blocks + kQuantBlocks - 1) / kQuantBlocks);
    uint8_t *q = static_cast<uint8_t *>(Q);
    const dim3 block(kQuantThreads);
    if (F < 4) {
        if (bf16) hipLaunchKernelGGL((quantize_kernel<true, true>), grid, block, 0, s, X, q, scales, n, F, blocks);
        else hipLaunchKernelGGL((quantize_kernel<false, true>), grid, block, 0, s, X, q, scales, n, F, blocks);
    } else {
        if (bf16) hipLaunchKernelGGL((quantize_kernel<true, false>), grid, block, 0, s, X, q, scales, n, F, blocks);
        else hipLaunchKernelGGL((quantize_kernel<false, false>), grid, block, 0, s, X, q, scales, n, F, blocks);
    }
    return hip_status(hipGetLastError());
}

int launch_quantize_weight(const float *W, int32_t rows, int32_t cols, bool transpose, void *Q, float *scales,
                           hipStream_t s) {
    hipLaunchKernelGGL(quantize_weight_kernel, dim3((cols + kBlock - 1) / kBlock, (rows + kBlock - 1) / kBlock),
                       dim3(kQuantThreads), 0, s, W, rows, cols, transpose ? 1 : 0, static_cast<uint8_t *>(Q), scales);
    return hip_status(hipGetLastError());
}

int launch_update_fp8(const void *X, const float *sx, const void *W, const float *sw, void *T, bool out_bf16,
                      int32_t n, int32_t F_in, int32_t F_out, hipStream_t s) {
    const ProductArgs a{static_cast<const uint8_t *>(X), static_cast<const uint8_t *>(W), sx, sw, T, n, F_in, F_out,
                        (F_in + kBlock - 1) / kBlock, out_bf16};
    // us few and many rows' kernel: 256 -> 128 at 256, 512 rows 9.7, 10.2 and 9.4, 10.7; 1,024 -> 1,024 at 256, 512, 1,024
    // rows 9.8, 15.1 and 12.3, 15.4 and 21.9, 15.9
    if (n <= 512) {
        hipLaunchKernelGGL(product_few_kernel, dim3((F_out + 15) / 16, (n + 15) / 16), dim3(kThreads), 0, s, a);
        return hip_status(hipGetLastError());
    }
    // few tiles: narrower slices until they are about as many as the CUs (us so and with the widest slices, 256 -> 128:
    // 1,000 rows 9.3, 10.6, 20,000 rows 9.4, 12.3; 1,024 -> 1,024, 1,000 rows 15.9, 18.1)
    const int64_t tiles = (static_cast<int64_t>(n) + kRowsPerBlock - 1) / kRowsPerBlock;
    const int64_t share = device_cus() / tiles;                          // slices there may be
    const int cols = (F_out + 15) / 16;
    const int most = share <= 1 ? kMostCols : std::max<int>(1, static_cast<int>(std::min<int64_t>(kMostCols, (cols + share - 1) / share)));
    return launch_slices(a, most, s);
}

}  // namespace dgc
