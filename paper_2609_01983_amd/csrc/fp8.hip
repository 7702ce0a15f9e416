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

typedef uint32_t u32_any __attribute__((aligned(1)));

// 16 lanes a block of 128, two quads a lane (a lane's elements 4 l and 64 + 4 l on).
constexpr int kQuantThreads = 256;
constexpr int kQuantLanes = 16;
template <bool BF>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(const void *__restrict__ X, uint8_t *__restrict__ Q,
                                                                 float *__restrict__ scales, int64_t items,
                                                                 int32_t F, int32_t blocks) {
    const int l = threadIdx.x % kQuantLanes;
    constexpr int kPer = kQuantThreads / kQuantLanes;
    for (int64_t it = static_cast<int64_t>(blockIdx.x) * kPer + threadIdx.x / kQuantLanes; it < items;
         it += static_cast<int64_t>(gridDim.x) * kPer) {
        const int64_t row = it / blocks;
        const int b = static_cast<int>(it - row * blocks);
        const int64_t r0 = row * F;
        row_f32x4 v[2];
        float amax = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = b * kBlock + 64 * h + 4 * l;
            v[h] = load_quad<BF>(X, r0 + col, F - col);
#pragma unroll
            for (int i = 0; i < 4; ++i) amax = fmaxf(amax, finite_abs(v[h][i]));
        }
        amax = lanes_reduce<kQuantLanes>(amax, MaxOp());
        const int k = scale_exponent(amax);
        const float inv = power_of_two(-k);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = b * kBlock + 64 * h + 4 * l, count = F - col;
            const uint32_t q = to_e4m3(v[h] * inv);
            uint8_t *p = Q + r0 + col;
            if (count >= 4) {
                *reinterpret_cast<u32_any *>(p) = q;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < count) p[i] = static_cast<uint8_t>(q >> 8 * i);
            }
        }
        if (l == 0) scales[it] = power_of_two(k);
    }
}

// A block of 128 x 128 of W (rows x cols, float32), quantised into Q as it stands or transposed.
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
// block's sum is right whatever their order.  Chunks behind the row's end are read at its start
// and zeroed by get().
constexpr int kSteps = kBlock / 32;
struct Fragment {
    u32x4 lo, hi;
    __device__ __forceinline__ void load(const uint8_t *base, int64_t row, int K, int b, int g) {
        const uint8_t *r = base + row * K;
        const int k = b * kBlock + 16 * g;
        lo = *reinterpret_cast<const u32x4 *>(r + (k < K ? k : 0));
        hi = *reinterpret_cast<const u32x4 *>(r + (k + 64 < K ? k + 64 : 0));
    }
    __device__ __forceinline__ void get(int K, int b, int g, bf16x8 (&out)[kSteps]) const {
        const int k = b * kBlock + 16 * g;
        const u32x4 zero = {0, 0, 0, 0};
        const u32x4 x = k < K ? lo : zero, y = k + 64 < K ? hi : zero;
        out[0] = widen(x[0], x[1]);
        out[1] = widen(x[2], x[3]);
        out[2] = widen(y[0], y[1]);
        out[3] = widen(y[2], y[3]);
    }
};

__device__ __forceinline__ void store_tile(const ProductArgs &a, int64_t row, int col, int last, f32x4 v) {
    const int count = last - col;
    if (row >= a.n || count <= 0) return;
    if (a.out_bf16) store_quad<true>(a.T, row * a.N + col, count, v);
    else store_quad<false>(a.T, row * a.N + col, count, v);
}

// Workgroups of eight wavefronts, 32 rows each, with W of CT tiles of 16 columns in LDS.
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kRowTiles = 2;
constexpr int kRows = 16 * kRowTiles;                // of a wavefront
constexpr int kRowsPerBlock = kWaves * kRows;
// bfloat16 elements of a W row in LDS: whole blocks, in the order the lanes read them, and 8 more
// so that the 16 rows a read touches start in 16 different groups of four banks
__host__ __device__ __forceinline__ int lds_row(int blocks) { return blocks * kBlock + 8; }

template <int CT>
__global__ __launch_bounds__(kThreads) void product_kernel(ProductArgs a) {
    extern __shared__ uint4 lds[];
    __bf16 *w = reinterpret_cast<__bf16 *>(lds);
    const int ld = lds_row(a.blocks);
    const int c0 = blockIdx.y * 16 * CT;
    // W of the columns [c0, c0 + 16 CT), zeros past F_out and past F_in: 16 bytes of W8 are two
    // steps of a lane group, [block][step][g][8]
    const int per_row = a.blocks * kBlock / 16;
    for (int i = threadIdx.x; i < 16 * CT * per_row; i += kThreads) {
        const int c = i / per_row, chunk = i % per_row, k = chunk * 16;
        u32x4 v = {0, 0, 0, 0};
        if (c0 + c < a.N && k < a.K) v = *reinterpret_cast<const u32x4 *>(a.W + static_cast<int64_t>(c0 + c) * a.K + k);
        const int b = chunk / 8, half = chunk % 8 / 4, g = chunk % 4;
        __bf16 *to = w + c * ld + b * kBlock + half * 64 + g * 8;
        *reinterpret_cast<bf16x8 *>(to) = widen(v[0], v[1]);
        *reinterpret_cast<bf16x8 *>(to + 32) = widen(v[2], v[3]);
    }
    __syncthreads();

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const float *sw = a.sw + static_cast<int64_t>(c0 / kBlock) * a.blocks;
    const int64_t tiles = (static_cast<int64_t>(a.n) + kRowsPerBlock - 1) / kRowsPerBlock;
    const int last = min(a.N, c0 + 16 * CT);

    auto row_of = [&](int64_t tile, int t) {
        const int64_t row = tile * kRowsPerBlock + wave * kRows + t * 16 + r;
        return row < a.n ? row : static_cast<int64_t>(a.n) - 1;
    };
    Fragment cur[kRowTiles], nxt[kRowTiles];
    float sc[kRowTiles], sn[kRowTiles];
    int64_t tile = blockIdx.x;                       // the grid has at most one workgroup a tile and slice
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t) {
        const int64_t row = row_of(tile, t);
        cur[t].load(a.X, row, a.K, 0, g);
        sc[t] = a.sx[row * a.blocks];
    }
    for (; tile < tiles; tile += gridDim.x) {
        f32x4 acc[kRowTiles][CT];
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int b = 0; b < a.blocks; ++b) {
            // the next block of this tile, or the first of the next tile (past the last: rows n - 1)
            const bool more = b + 1 < a.blocks;
            const int nb = more ? b + 1 : 0;
            const int64_t nt = more ? tile : tile + gridDim.x;
#pragma unroll
            for (int t = 0; t < kRowTiles; ++t) {
                const int64_t row = row_of(nt, t);
                nxt[t].load(a.X, row, a.K, nb, g);
                sn[t] = a.sx[row * a.blocks + nb];
            }
            bf16x8 x[kRowTiles][kSteps];
            float f[kRowTiles];
#pragma unroll
            for (int t = 0; t < kRowTiles; ++t) {
                cur[t].get(a.K, b, g, x[t]);
                f[t] = sc[t] * sw[b];
            }
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const __bf16 *p = w + (16 * c + r) * ld + b * kBlock + 8 * g;
                f32x4 s[kRowTiles];
#pragma unroll
                for (int t = 0; t < kRowTiles; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    const bf16x8 wf = *reinterpret_cast<const bf16x8 *>(p + 32 * k);
#pragma unroll
                    for (int t = 0; t < kRowTiles; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, x[t][k], s[t], 0, 0, 0);
                }
#pragma unroll
                for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][c][i] = fmaf(f[t], s[t][i], acc[t][c][i]);
            }
#pragma unroll
            for (int t = 0; t < kRowTiles; ++t) {
                cur[t] = nxt[t];
                sc[t] = sn[t];
            }
        }
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) {
            const int64_t row = tile * kRowsPerBlock + wave * kRows + t * 16 + r;
#pragma unroll
            for (int c = 0; c < CT; ++c) store_tile(a, row, c0 + 16 * c + 4 * g, last, acc[t][c]);
        }
    }
}

// Few rows: a workgroup makes 16 rows x 16 columns, its wavefronts take the blocks of K in turn
// (W8 straight from memory: each of it is used once) and join their sums in order through LDS.
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
        const float f = a.sx[xr * a.blocks + b] * sw[b];
        bf16x8 xs[kSteps], ws[kSteps];
        x.get(a.K, b, g, xs);
        w.get(a.K, b, g, ws);
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ws[k], xs[k], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(f, s[i], acc[i]);
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

template <int CT>
int launch_product(const ProductArgs &a, hipStream_t s) {
    const size_t lds = static_cast<size_t>(16 * CT) * lds_row(a.blocks) * sizeof(uint16_t);
    const int st = allow_lds(reinterpret_cast<const void *>(&product_kernel<CT>), lds);
    if (st) return st;
    const int per_cu = std::max<int>(1, std::min<int>(2, static_cast<int>((160 * 1024) / lds)));
    const int64_t tiles = (static_cast<int64_t>(a.n) + kRowsPerBlock - 1) / kRowsPerBlock;
    const int slices = (a.N + 16 * CT - 1) / (16 * CT);
    const int64_t grid = std::max<int64_t>(1, std::min<int64_t>(tiles, static_cast<int64_t>(device_cus()) * per_cu / slices));
    hipLaunchKernelGGL(product_kernel<CT>, dim3(static_cast<unsigned>(grid), slices), dim3(kThreads), lds, s, a);
    return hip_status(hipGetLastError());
}

}  // namespace

int launch_quantize(const void *X, bool bf16, int32_t n, int32_t F, void *Q, float *scales, hipStream_t s) {
    const int32_t blocks = (F + kBlock - 1) / kBlock;
    const int64_t items = static_cast<int64_t>(n) * blocks;
    constexpr int kPer = kQuantThreads / kQuantLanes;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((items + kPer - 1) / kPer, static_cast<int64_t>(device_cus()) * 8)));
    if (bf16) hipLaunchKernelGGL(quantize_kernel<true>, grid, dim3(kQuantThreads), 0, s, X, static_cast<uint8_t *>(Q), scales, items, F, blocks);
    else hipLaunchKernelGGL(quantize_kernel<false>, grid, dim3(kQuantThreads), 0, s, X, static_cast<uint8_t *>(Q), scales, items, F, blocks);
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
    if (n <= 256) {
        hipLaunchKernelGGL(product_few_kernel, dim3((F_out + 15) / 16, (n + 15) / 16), dim3(kThreads), 0, s, a);
        return hip_status(hipGetLastError());
    }
    if (F_out <= 32 || static_cast<int64_t>(n) * ((F_out + 127) / 128) <= int64_t{kRowsPerBlock} * 256)
        return launch_product<2>(a, s);
    // W of 128 columns fits a workgroup's LDS up to F_in = 512
    return a.blocks <= 4 ? launch_product<8>(a, s) : launch_product<4>(a, s);
}

}  // namespace dgc
