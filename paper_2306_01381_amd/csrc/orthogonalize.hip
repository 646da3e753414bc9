// Newton-Schulz steps on the matrix cores (adaqp_dense.h).
//
// With n <= m a step is three products: A = X X^T (n x n over m), Q = a I + b A + c A A (n x n over n) and X <- Q X (n x m over n).  A and Q are symmetric,
// so only the tiles on and below the diagonal are computed and each is stored twice.
//
// fp32 products run at a tenth of the fp16 rate on this machine (8192^3: 0.15 and 1.47 PFLOP/s), and fp16 has 11 bits.  Every matrix is therefore held as hi + lo, two
// fp16 numbers with 22 bits together, in units of a power of two that keeps the entries below 2^14 (the host knows a bound on the singular values after
// every step), and a product is hi hi + hi lo + lo hi, summed in fp32: what is left out is below 2^-22 of a term.  Memory holds lines of 128 bytes: 32 hi,
// then the 32 lo of the same columns, which is what a step of the products' loop takes of a row.  Both X and its transpose are kept, since the loop
// runs along rows of both operands.
//
// What bounds it: matrices of some hundred rows the chain of launches, each about 4 us from its start over one or two waits for memory to its end (3 of 256 x 256:
// 17 launches, 70 us; one of 602 x 256 the same); large ones the matrix cores: one of 2048 x 4096 1020 to 1070 us with the clock that a run finds, 0.86 PFLOP/s counting three fp16 products
// each (a large fp16 product reaches 1.47).  Its step's products run at 1.1 PFLOP/s (103 GFLOP in 96 us), X X^T in 61 us and 10 to join, A A in 34 and 11, whose 136 tiles in three cuts are
// 408 workgroups for 512 places; of zeros, which draw less, it takes 814.
#include <math.h>

#include "lines.hpp"
#include "orthogonalize.hpp"

namespace adaqp {
namespace {

constexpr int kPad = 64;                            // rows and columns of the held matrices are multiples
constexpr int kNormBlocks = 512;                    // of a matrix, at most
constexpr int kNormRun = 8 * kBlock;                // columns
constexpr int kMostPower = 14;
constexpr int64_t kMostSize = (int64_t)1 << 20;

// Where (row, col) of a held matrix lies: hi there, lo 64 bytes on.
__device__ __forceinline__ int64_t held_at(int64_t row, int64_t col, int64_t pitch) { return row * pitch + col / 32 * kLine + col % 32 * 2; }

// Sums of squares of a share of each matrix: blocks [x] of matrix [y], runs of eight columns a thread.
template <typename T>
__global__ __launch_bounds__(kBlock) void update_norm_kernel(const T *g, int64_t ldg, int64_t stride, int64_t n_rows, int64_t n_cols, double *partial)
{
    __shared__ double lds[kWavesPerBlock];
    g += blockIdx.y * stride;
    const uint32_t runs = (uint32_t)((n_cols + kNormRun - 1) / kNormRun);
    const int64_t total = n_rows * runs;
    double sum = 0.0;
    for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
        const int64_t row = at / runs, col = (at - row * runs) * kNormRun + threadIdx.x;
        float v[kNormRun / kBlock];
#pragma unroll
        for (int k = 0; k < kNormRun / kBlock; ++k) v[k] = (float)g[row * ldg + min(col + k * kBlock, n_cols - 1)];
#pragma unroll
        for (int k = 0; k < kNormRun / kBlock; ++k)
            if (col + k * kBlock < n_cols) sum = fma((double)v[k], (double)v[k], sum);
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// A matrix's sum of squares, by all threads of a workgroup.
__device__ __forceinline__ double norm_square(const double *partial, int n_partial, double *lds)
{
    static_assert(kNormBlocks <= 2 * kBlock, "two partial sums a thread");
    const int t = threadIdx.x;
    return block_sum((t < n_partial ? partial[t] : 0.0) + (t + kBlock < n_partial ? partial[t + kBlock] : 0.0), lds);
}

// G / (norm + eps) in units of 2^-power as held matrices: as it lies (`same`) and transposed (`other`), zeros up to the padded sizes.  Tiles of 32 x 32, a line of each row
// of either form: blocks [x] of matrix [y] take turns, a thread four neighbours of a row, then of a column.
template <typename T>
__global__ __launch_bounds__(kBlock) void update_split_kernel(const T *g, int64_t ldg, int64_t stride, int64_t n_rows, int64_t n_cols, const double *partial,
                                                              int n_partial, double eps, int power, uint8_t *same, uint8_t *other, int64_t pitch_same,
                                                              int64_t pitch_other, int64_t held_bytes, uint32_t tiles_r, uint32_t tiles_c)
{
    constexpr int kTile = 32, kEach = kTile * kTile / kBlock;
    __shared__ double lds[kWavesPerBlock];
    __shared__ float tile[2][kTile][kTile + 1];
    g += blockIdx.y * stride;
    same += blockIdx.y * held_bytes;
    other += blockIdx.y * held_bytes;
    const int major = threadIdx.x / (kTile / kEach), minor = threadIdx.x % (kTile / kEach) * kEach;
    auto store = [](uint8_t *to, const float (&v)[kEach]) {
        half4 hi, lo;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            _Float16 a, b;
            split(v[k], a, b);
            hi[k] = a;
            lo[k] = b;
        }
        *reinterpret_cast<half4 *>(to) = hi;
        *reinterpret_cast<half4 *>(to + 64) = lo;
    };
    double scale = 0.0;
    int turn = 0;
    for (uint32_t at = blockIdx.x; at < tiles_r * tiles_c; at += gridDim.x, turn ^= 1) {
        const int64_t row0 = (int64_t)(at / tiles_c) * kTile, col0 = (int64_t)(at % tiles_c) * kTile;
        const int64_t row = row0 + major, col = col0 + minor;
        float v[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) v[k] = (float)g[min(row, n_rows - 1) * ldg + min(col + k, n_cols - 1)];
        if (at == blockIdx.x) scale = ldexp(one_over_norm(norm_square(partial + blockIdx.y * n_partial, n_partial, lds), eps), power);
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            v[k] = row < n_rows && col + k < n_cols ? (float)((double)v[k] * scale) : 0.0f;      // behind the edge also where the scale is not finite
            tile[turn][major][minor + k] = v[k];
        }
        store(same + held_at(row, col, pitch_same), v);
        __syncthreads();                            // the other tile of the LDS is written next
#pragma unroll
        for (int k = 0; k < kEach; ++k) v[k] = tile[turn][minor + k][major];
        store(other + held_at(col0 + major, row0 + minor, pitch_other), v);
    }
}

enum Product { GRAM, POLY, STEP, LAST };

struct ProductArgs {
    const uint8_t *p, *q;                           // D = p q^T
    int64_t rows, cols;                             // of D, padded
    int64_t lines;                                  // of a row of p and q that hold columns
    int64_t pitch;                                  // of p and q
    uint8_t *same, *other;                          // D and its transpose, held
    int64_t pitch_same, pitch_other;
    int64_t bytes_p, bytes_q, bytes_d;              // from matrix to matrix
    float scale;                                    // of the sums in the units of what is stored
    float diagonal, linear;                         // POLY: what is added, of I and of p, in those units
    void *out;                                      // LAST: D itself
    int64_t ldo, stride_o, out_rows, out_cols, written;
    int64_t tiles_r, tiles_c;
    int parts;                                      // cuts of the lines
    float *sums;                                    // of parts, more than one: [matrix][part][tile][a workgroup's registers]
};

// Tiles below and on the diagonal, row by row.
__device__ __forceinline__ void triangle_tile(uint32_t block, int64_t &row, int64_t &col)
{
    row = (int64_t)((sqrtf(8.0f * block + 1.0f) - 1.0f) * 0.5f);
    while (row * (row + 1) / 2 > block) --row;
    while ((row + 1) * (row + 2) / 2 <= block) ++row;
    col = block - row * (row + 1) / 2;
}

// The same in squares of 4 x 4 tiles: `block` of a square's 16, squares below and on the diagonal row by row.  Workgroups of tiles that are not there (beyond the
// diagonal, or the edge) have nothing to do.
constexpr int kSquare = 4;

__host__ __device__ inline int64_t squares_of(int64_t tiles)
{
    const int64_t n = (tiles + kSquare - 1) / kSquare;
    return n * (n + 1) / 2;
}

// v in the units of POLY's sums: b A + c A A + a I, of which `p` holds A.
__device__ __forceinline__ float polynomial(const ProductArgs &g, const uint8_t *p, int64_t row, int64_t col, float v)
{
    const uint8_t *from = p + held_at(row, col, g.pitch);
    const float a = (float)*reinterpret_cast<const _Float16 *>(from) + (float)*reinterpret_cast<const _Float16 *>(from + 64);
    return fmaf(g.linear, a, v) + (row == col ? g.diagonal : 0.0f);
}

constexpr int kSmallTile = 32, kSmallWaves = 8;

// Few tiles: 32 x 32 each, whose eight waves share the lines (w, w + 8, ...), each with a part of the LDS of its own and two lines under way: no wave waits for
// another before the sums are added, and a product of 256 x 256 x 256 waits for memory once.
template <Product KIND, typename T>
__global__ __launch_bounds__(kSmallWaves * kWave) void update_small_product_kernel(ProductArgs g)
{
    constexpr bool kSymmetric = KIND == GRAM || KIND == POLY;
    constexpr int kStages = 2, kOperand = kSmallTile * kLine, kLoads = 2 * kOperand / (kWave * 16);
    __shared__ __align__(16) uint8_t lds[kSmallWaves][kStages][2][kOperand];
    __shared__ float tile[kSmallTile][kSmallTile + 1];
    int64_t tr, tc;
    if (kSymmetric) triangle_tile(blockIdx.x, tr, tc);
    else {
        tr = blockIdx.x / g.tiles_c;
        tc = blockIdx.x % g.tiles_c;
    }
    const uint8_t *p = g.p + blockIdx.y * g.bytes_p, *q = g.q + blockIdx.y * g.bytes_q;
    const int64_t row0 = tr * kSmallTile, col0 = tc * kSmallTile;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    sums16 sums;
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[e] = 0.0f;
    const uint8_t *from[2] = {p + row0 * g.pitch, q + col0 * g.pitch};
    uint32_t offset[kLoads / 2];
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) offset[i] = (uint32_t)(i * 8 + lane / 8) * (uint32_t)g.pitch + part_of_lane(i) * 16;
    auto load = [&](int line, int stage) {
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds_offset(lds[wave][stage][o]));
#pragma unroll
            for (int i = 0; i < kLoads / 2; ++i) load_to_lds_16(from[o] + (int64_t)line * kLine, offset[i], to + i * 8 * kLine);
        }
    };
    const int lines = (int)g.lines;
    auto one = [&](int stage) {
        const uint8_t *left = lds[wave][stage][0], *right = lds[wave][stage][1];
        half8 x[4], y[4];                           // hi of the two halves of a line, lo of them
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] = *reinterpret_cast<const half8 *>(line_part(left, r, k * 2 + h));
            y[k] = *reinterpret_cast<const half8 *>(line_part(right, r, k * 2 + h));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            sums = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[2 + k], y[k], sums, 0, 0, 0);
            sums = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[k], y[2 + k], sums, 0, 0, 0);
            sums = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[k], y[k], sums, 0, 0, 0);
        }
    };
    if (wave < lines) load(wave, 0);
    if (wave + kSmallWaves < lines) load(wave + kSmallWaves, 1);
    int stage = 0;
    for (int line = wave; line < lines; line += kSmallWaves, stage ^= 1) {
        if (line + kSmallWaves < lines) own_arrived<kLoads>();
        else                            own_arrived<0>();
        one(stage);
        if (line + 2 * kSmallWaves < lines) {
            own_read();
            load(line + 2 * kSmallWaves, stage);
        }
    }
    own_read();
    float (*parts)[sizeof(lds[0]) / 4] = reinterpret_cast<float (*)[sizeof(lds[0]) / 4]>(lds);  // a wave's sums lie where its lines were
#pragma unroll
    for (int e = 0; e < 16; ++e) parts[wave][(e / 4 * 8 + h * 4 + e % 4) * kSmallTile + r] = sums[e];
    __syncthreads();
    // two neighbouring columns a thread, then two rows
    const int major = threadIdx.x / 16, minor = threadIdx.x % 16 * 2;
    float v[2] = {0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) {
        v[0] += parts[w][major * kSmallTile + minor];
        v[1] += parts[w][major * kSmallTile + minor + 1];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v[k] *= g.scale;
        if (KIND == POLY) v[k] = polynomial(g, p, row0 + major, col0 + minor + k, v[k]);
    }
    if constexpr (KIND == LAST) {
        T *out = (T *)g.out + blockIdx.y * g.stride_o;
        const int64_t row = row0 + major;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int64_t col = col0 + minor + k;
            if (row < g.out_rows && col < g.written) out[row * g.ldo + col] = col < g.out_cols ? (T)v[k] : (T)0.0f;
        }
    } else {
        auto store = [](uint8_t *to, float first, float second) {
            half2 hi, lo;
            _Float16 a, b;
            split(first, a, b);
            hi[0] = a;
            lo[0] = b;
            split(second, a, b);
            hi[1] = a;
            lo[1] = b;
            *reinterpret_cast<half2 *>(to) = hi;
            *reinterpret_cast<half2 *>(to + 64) = lo;
        };
        store(g.same + blockIdx.y * g.bytes_d + held_at(row0 + major, col0 + minor, g.pitch_same), v[0], v[1]);
        if (kSymmetric && tr == tc) return;
        tile[major][minor] = v[0];
        tile[major][minor + 1] = v[1];
        __syncthreads();
        store(g.other + blockIdx.y * g.bytes_d + held_at(col0 + major, row0 + minor, g.pitch_other), tile[minor][major], tile[minor + 1][major]);
    }
}

// Which tile, and which cut of the lines; false: none.  XCDs get neighbouring tiles.
template <bool SYMMETRIC>
__device__ __forceinline__ bool product_tile(const ProductArgs &g, int64_t &tr, int64_t &tc, int &part)
{
    if (SYMMETRIC) {
        const uint32_t at = xcd_neighbour(blockIdx.x, gridDim.x), in_square = at % (kSquare * kSquare), square = at / (kSquare * kSquare);
        int64_t row, col;
        triangle_tile(square / g.parts, row, col);
        part = (int)(square % g.parts);
        tr = row * kSquare + in_square / kSquare;
        tc = col * kSquare + in_square % kSquare;
        return tr < g.tiles_r && tc <= tr;
    }
    const TilePlace place = tile_place(blockIdx.x, gridDim.x, (uint32_t)g.tiles_r, (uint32_t)g.tiles_c, 1);
    tr = place.row;
    tc = place.col;
    part = 0;
    return place.part >= 0;
}

// A wave's 32 x 32 sums on their way out, in the LDS.
constexpr int kSheetPitch = 36;
struct alignas(16) Sheet { float v[32 * kSheetPitch]; };
static_assert(alignof(Sheet) % alignof(float4) == 0, "read in vectors");

// 16 neighbouring columns of a held row, from a multiple of 16 on.
__device__ __forceinline__ void store_held(uint8_t *to, const float (&v)[16])
{
    half8 hi[2], lo[2];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        _Float16 a, b;
        split(v[k], a, b);
        hi[k / 8][k % 8] = a;
        lo[k / 8][k % 8] = b;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        *reinterpret_cast<half8 *>(to + k * 16) = hi[k];
        *reinterpret_cast<half8 *>(to + 64 + k * 16) = lo[k];
    }
}

// Stores what a wave's 32 x 32 sums at (row0, col0) of D say.  Held matrices through the sheet, so that a lane has 16 neighbours of a row, then 16 of a column: stored
// from the sums' own places, two bytes and four rows a lane, a product of 4096 x 2048 x 2048 took 31 of its 104 us for it.
template <Product KIND, typename T>
__device__ __forceinline__ void store_sums(const ProductArgs &g, const uint8_t *p, int64_t row0, int64_t col0, bool on_diagonal, const sums16 &sums, Sheet &sheet)
{
    constexpr bool kSymmetric = KIND == GRAM || KIND == POLY;
    const int lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    if (row0 >= g.rows || col0 >= g.cols) return;   // the sizes are multiples of 64
    if constexpr (KIND == LAST) {
        T *out = (T *)g.out + blockIdx.y * g.stride_o + row0 * g.ldo + col0 + r;
        const int rows = (int)min(g.out_rows - row0, (int64_t)32), cols = (int)min(g.out_cols - col0, (int64_t)32), written = (int)min(g.written - col0, (int64_t)32);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int row = e / 4 * 8 + h * 4 + e % 4;
            if (row < rows && r < written) out[row * g.ldo] = r < cols ? (T)(sums[e] * g.scale) : (T)0.0f;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) sheet.v[(e / 4 * 8 + h * 4 + e % 4) * kSheetPitch + r] = sums[e] * g.scale;
        const int line = lane / 2, part = lane % 2 * 16;
        float v[16];
#pragma unroll
        for (int k = 0; k < 16; k += 4) {
            const float4 w = *reinterpret_cast<const float4 *>(&sheet.v[line * kSheetPitch + part + k]);
            v[k] = w.x;
            v[k + 1] = w.y;
            v[k + 2] = w.z;
            v[k + 3] = w.w;
        }
        if (KIND == POLY) {
            const uint8_t *from = p + held_at(row0 + line, col0 + part, g.pitch);
            half8 hi[2], lo[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                hi[k] = *reinterpret_cast<const half8 *>(from + k * 16);
                lo[k] = *reinterpret_cast<const half8 *>(from + 64 + k * 16);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                v[k] = fmaf(g.linear, (float)hi[k / 8][k % 8] + (float)lo[k / 8][k % 8], v[k]) + (row0 + line == col0 + part + k ? g.diagonal : 0.0f);
                sheet.v[line * kSheetPitch + part + k] = v[k];
            }
        }
        store_held(g.same + blockIdx.y * g.bytes_d + held_at(row0 + line, col0 + part, g.pitch_same), v);
        if (kSymmetric && on_diagonal) return;      // of a tile on the diagonal both halves are there
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = sheet.v[(part + k) * kSheetPitch + line];
        store_held(g.other + blockIdx.y * g.bytes_d + held_at(col0 + line, row0 + part, g.pitch_other), v);
    }
}

// Tiles of TR x TC, a quarter each wave of four.  With GROUPS = 2 eight waves share a tile, every second line each four of them: where there is a tile for each
// CU at most, half as many lines and barriers come one after the other.
template <Product KIND, typename T, int TR, int TC, int STAGES, int GROUPS>
__global__ __launch_bounds__(kBlock * GROUPS) void update_product_kernel(ProductArgs g)
{
    constexpr bool kSymmetric = KIND == GRAM || KIND == POLY;
    constexpr int FR = TR / 64, FC = TC / 64;       // 32 x 32 parts of a wave
    struct Stage { uint8_t p[TR * kLine], q[TC * kLine]; };
    __shared__ __align__(16) uint8_t lds[sizeof(Stage) * STAGES * GROUPS];
    static_assert(sizeof(Stage) * STAGES >= kWavesPerBlock * sizeof(Sheet), "the sheets lie where the operands were");
    static_assert(GROUPS == 1 || sizeof(Stage) * STAGES >= TR * TC * 4, "the other groups' sums, too");
    const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kBlock);
    Stage *stage = reinterpret_cast<Stage *>(lds) + group * STAGES;
    int64_t tr, tc;
    int part;
    if (!product_tile<kSymmetric>(g, tr, tc, part)) return;
    const uint8_t *p = g.p + blockIdx.y * g.bytes_p, *q = g.q + blockIdx.y * g.bytes_q;
    const int64_t row0 = tr * TR, col0 = tc * TC, pitch = g.pitch;
    const int wave = threadIdx.x % kBlock / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int wr = wave / 2 * (TR / 2), wc = wave % 2 * (TC / 2);

    sums16 sums[FR][FC];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[i][j][e] = 0.0f;

    const TileLoads<TR> of_p(row0, g.rows, pitch);
    const TileLoads<TC> of_q(col0, g.cols, pitch);
    constexpr int kLoadsP = TileLoads<TR>::kLoads, kLoads = kLoadsP + TileLoads<TC>::kLoads;
    // of the tile, or of the group: sizes are multiples of 64, so there is an even number
    const int per_part = (int)((g.lines + g.parts - 1) / g.parts), begin = part * per_part, lines = min(per_part, (int)g.lines - begin) / GROUPS;
    const uint8_t *from_p = p + row0 * pitch + (int64_t)(begin + group) * kLine, *from_q = q + col0 * pitch + (int64_t)(begin + group) * kLine;
    // Load i of a line of both operands.
    auto load = [&](int i, int line, const auto &s) {
        if (i < kLoadsP) of_p.template load<false>(i, from_p + (int64_t)line * (kLine * GROUPS), TileLoads<TR>::place(s.p));
        else             of_q.template load<false>(i - kLoadsP, from_q + (int64_t)line * (kLine * GROUPS), TileLoads<TC>::place(s.q));
    };
    // The operands of half a line, 16 columns: read from the LDS while the half before is multiplied, one by one between its products, in the order in which they
    // are needed (2048 x 4096 1080 us with them in a row before the products).
    struct Half { half8 ph[FR], pl[FR], qh[FC], ql[FC]; } half[2];
    constexpr int kReads = 2 * (FR + FC);
    auto read = [&](const auto &s, int k, int i, Half &to) {
        const bool second = i >= FR + FC;           // hi of p and lo of q
        i -= second ? FR + FC : 0;
        if (i == 0 || i > FC) {
            const int row = i == 0 ? 0 : i - FC;
            (second ? to.ph : to.pl)[row] = *reinterpret_cast<const half8 *>(line_part(s.p, wr + row * 32 + r, (second ? 0 : 4) + k * 2 + h));
        } else
            (second ? to.ql : to.qh)[i - 1] = *reinterpret_cast<const half8 *>(line_part(s.q, wc + (i - 1) * 32 + r, (second ? 4 : 0) + k * 2 + h));
    };
    // `between(i)` is done behind product i of the half's 3 FR FC.
    auto multiply = [&](const Half &f, auto between) {
#pragma unroll
        for (int w = 0; w < 3; ++w)                 // the small ones first
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FC; ++j) {
                    sums[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w == 0 ? f.pl[i] : f.ph[i], w == 1 ? f.ql[j] : f.qh[j], sums[i][j], 0, 0, 0);
                    between((w * FR + i) * FC + j);
                }
        __builtin_amdgcn_sched_barrier(0);
    };

    // Up to STAGES lines are under way.  A line's second half is multiplied behind the barrier after which the next line is in the LDS and its own buffer
    // free; the loads into that buffer are spread over that half's products and those of the next line's first half.  No branches: across one the compiler
    // would take products to the other side of the barrier.
    constexpr int kProducts = 3 * FR * FC, kReadsAtOnce = (kReads + kProducts - 1) / kProducts, kFirst = kLoads / 2;   // loads behind the products of a second half
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < lines)
#pragma unroll
            for (int l = 0; l < (s < STAGES - 1 ? kLoads : kFirst); ++l) load(l, s, stage[s]);
    if (lines >= STAGES) arrived<kLoads * (STAGES - 2) + kFirst>();
    else                 arrived<0>();
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(stage[0], 0, i, half[0]);
    int now = 0, before = STAGES - 1;
    auto one = [&](int line, auto pending, auto more) {
        constexpr bool kPending = decltype(pending)::value, kMore = decltype(more)::value;
        const Stage &s = stage[now], &last = stage[before];
        before = now;
        now = now + 1 == STAGES ? 0 : now + 1;
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[0], [&](int i) {
#pragma unroll
            for (int at = i * kReadsAtOnce; at < (i + 1) * kReadsAtOnce && at < kReads; ++at) read(s, 1, at, half[1]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kPending) {
#pragma unroll
                for (int l = kFirst + i * (kLoads - kFirst) / kProducts; l < kFirst + (i + 1) * (kLoads - kFirst) / kProducts; ++l) load(l, line - 1 + STAGES, last);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        arrived<kPending ? kLoads * (STAGES - 2) : 0>();
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[1], [&](int i) {
#pragma unroll
            for (int at = i * kReadsAtOnce; at < (i + 1) * kReadsAtOnce && at < kReads; ++at) read(stage[now], 0, at, half[0]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kMore) {
#pragma unroll
                for (int l = i * kFirst / kProducts; l < (i + 1) * kFirst / kProducts; ++l) load(l, line + STAGES, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    };
    int line = 0;
    for (; line + STAGES < lines; ++line) one(line, std::true_type(), std::true_type());
    if (lines >= STAGES) one(line++, std::true_type(), std::false_type());
    for (; line < lines; ++line) one(line, std::false_type(), std::false_type());

    if (kSymmetric && g.parts > 1) {
        float4 *to = reinterpret_cast<float4 *>(g.sums + ((blockIdx.y * g.parts + part) * (g.tiles_r * (g.tiles_r + 1) / 2) + tr * (tr + 1) / 2 + tc) * (TR * TC));
#pragma unroll
        for (int i = 0; i < FR; ++i)
#pragma unroll
            for (int j = 0; j < FC; ++j)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    to[((i * FC + j) * 4 + e / 4) * kBlock + threadIdx.x] = make_float4(sums[i][j][e], sums[i][j][e + 1], sums[i][j][e + 2], sums[i][j][e + 3]);
        return;
    }
    arrived<0>();                                   // nobody reads the operands any more
    if constexpr (GROUPS > 1) {
        float4 *others = reinterpret_cast<float4 *>(lds + sizeof(Stage) * STAGES);
        static_assert(GROUPS == 2 && FR == 1 && FC == 1, "one other group's 32 x 32 sums a wave");
        if (group > 0)
#pragma unroll
            for (int e = 0; e < 16; e += 4) others[e / 4 * kBlock + threadIdx.x % kBlock] = make_float4(sums[0][0][e], sums[0][0][e + 1], sums[0][0][e + 2], sums[0][0][e + 3]);
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const float4 v = others[e / 4 * kBlock + threadIdx.x];
            sums[0][0][e] += v.x;
            sums[0][0][e + 1] += v.y;
            sums[0][0][e + 2] += v.z;
            sums[0][0][e + 3] += v.w;
        }
    }
    Sheet &sheet = reinterpret_cast<Sheet *>(lds)[wave];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) store_sums<KIND, T>(g, p, row0 + wr + i * 32, col0 + wc + j * 32, tr == tc, sums[i][j], sheet);
}

// A symmetric product whose lines were cut: the parts' sums, in order, and what is made of them.  A workgroup takes a part (i, j) = blockIdx.z of each wave's.
template <Product KIND, int TILE>
__global__ __launch_bounds__(kBlock) void update_join_kernel(ProductArgs g)
{
    constexpr int F = TILE / 64;
    __shared__ Sheet sheets[kWavesPerBlock];
    int64_t tr, tc;
    triangle_tile(blockIdx.x, tr, tc);
    const int wave = threadIdx.x / kWave, i = blockIdx.z / F, j = blockIdx.z % F;
    const int64_t tiles = g.tiles_r * (g.tiles_r + 1) / 2;
    const float4 *from = reinterpret_cast<const float4 *>(g.sums + (blockIdx.y * g.parts * tiles + blockIdx.x) * (TILE * TILE)) + blockIdx.z * 4 * kBlock + threadIdx.x;
    sums16 sums;
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[e] = 0.0f;
    for (int part = 0; part < g.parts; ++part, from += tiles * (TILE * TILE) / 4) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const float4 v = from[e / 4 * kBlock];
            sums[e] += v.x;
            sums[e + 1] += v.y;
            sums[e + 2] += v.z;
            sums[e + 3] += v.w;
        }
    }
    store_sums<KIND, float>(g, g.p + blockIdx.y * g.bytes_p, tr * TILE + wave / 2 * (TILE / 2) + i * 32, tc * TILE + wave % 2 * (TILE / 2) + j * 32, tr == tc, sums,
                              sheets[wave]);
}

template <typename T>
__global__ __launch_bounds__(kBlock) void update_scale_kernel(const T *g, int64_t ldg, int64_t stride, int64_t n_rows, int64_t n_cols, const double *partial,
                                                              int n_partial, double eps, T *out, int64_t ldo, int64_t stride_o, int64_t written)
{
    __shared__ double lds[kWavesPerBlock];
    const double scale = one_over_norm(norm_square(partial + blockIdx.y * n_partial, n_partial, lds), eps);
    g += blockIdx.y * stride;
    out += blockIdx.y * stride_o;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < n_rows * written; at += (int64_t)gridDim.x * kBlock) {
        const int64_t row = at / written, col = at % written;
        out[row * ldo + col] = col < n_cols ? (T)(float)((double)(float)g[row * ldg + col] * scale) : (T)0.0f;
    }
}

int64_t padded(int64_t v) { return (v + kPad - 1) / kPad * kPad; }

// Bytes from row to row of a held matrix: an odd number of lines, so that the same line of all rows is spread over the L2's channels.
int64_t held_pitch(int64_t cols) { return (cols / 32 | 1) * kLine; }

struct UpdateLayout {
    bool flip;                                      // more rows than columns: X is the transpose
    int64_t n, m;                                   // padded, n of the smaller
    int64_t big, small;                             // bytes of X and of A
    int64_t norm_blocks;
    int parts_m, parts_n;                           // cuts of the lines of symmetric products over m and over n, tiles of 128 x 128
    int64_t partial_at, x_at, a_at, q_at, sums_at, bytes;       // X, its transpose, both again for the next step
};

// Cuts of the lines of a symmetric product of n x n: two tiles of 128 x 128 share a CU, and with at least kCutTiles of them there are enough for tiles of that size to
// pay, but fewer than there is room for.  us uncut and cut: 2048 x 4096, 136 tiles, X X^T 109 and 75, A A 50 and 47; 1300 x 1300, 66 tiles, 23.5 and 25.5.
constexpr int kCutTiles = 128, kRoom = 512, kLeastLines = 16;

int update_parts(int64_t n, int64_t lines, int64_t n_matrices)
{
    const int64_t t = (n + 127) / 128, tiles = t * (t + 1) / 2 * n_matrices;
    if (tiles < kCutTiles || 2 * tiles > kRoom) return 1;
    const int64_t parts = kRoom / tiles < lines / kLeastLines ? kRoom / tiles : lines / kLeastLines;
    return parts < 1 ? 1 : (int)((lines + (lines + parts - 1) / parts - 1) / ((lines + parts - 1) / parts));
}

UpdateLayout update_layout(int32_t n_matrices, int64_t n_rows, int64_t n_cols)
{
    UpdateLayout u{};
    u.flip = n_rows > n_cols;
    u.n = padded(u.flip ? n_cols : n_rows);
    u.m = padded(u.flip ? n_rows : n_cols);
    const int64_t of_x = u.n * held_pitch(u.m), of_xt = u.m * held_pitch(u.n);
    u.big = of_x > of_xt ? of_x : of_xt;
    u.small = u.n * held_pitch(u.n);
    u.norm_blocks = n_rows * ((n_cols + kNormRun - 1) / kNormRun);
    if (u.norm_blocks > kNormBlocks) u.norm_blocks = kNormBlocks;
    u.partial_at = 0;
    if (small_update_fits(n_rows, n_cols)) {        // its steps are in the LDS; without steps only the norms' sums are needed
        u.bytes = (int64_t)n_matrices * kNormBlocks * 8;
        return u;
    }
    u.x_at = (n_matrices * u.norm_blocks * 8 + 255) / 256 * 256;
    u.a_at = u.x_at + 4 * n_matrices * u.big;
    u.q_at = u.a_at + n_matrices * u.small;
    u.sums_at = u.q_at + n_matrices * u.small;
    u.parts_m = update_parts(u.n, u.m / 32, n_matrices);
    u.parts_n = update_parts(u.n, u.n / 32, n_matrices);
    const int64_t parts = u.parts_m > u.parts_n ? u.parts_m : u.parts_n, t = (u.n + 127) / 128;
    u.bytes = u.sums_at + (parts > 1 ? parts * n_matrices * (t * (t + 1) / 2) * 128 * 128 * 4 : 0);
    return u;
}

// The largest |x q(x^2)| and |q(x^2)| over 0 <= x <= most, q(y) = a + b y + c y^2: at the ends or where a derivative is zero.
void bounds(double a, double b, double c, double most, double *of_step, double *of_q)
{
    const double end = most * most;
    auto q = [&](double y) { return fabs(a + b * y + c * y * y); };
    double step = most * q(end), quadratic = fmax(q(0.0), q(end));
    auto at = [&](double y, bool both) {
        if (!(y > 0.0 && y < end)) return;
        step = fmax(step, sqrt(y) * q(y));
        if (both) quadratic = fmax(quadratic, q(y));
    };
    if (c != 0.0) {
        at(-b / (2.0 * c), true);
        const double root = 9.0 * b * b - 20.0 * a * c;             // a + 3 b y + 5 c y^2 = 0
        if (root >= 0.0) {
            at((-3.0 * b + sqrt(root)) / (10.0 * c), false);
            at((-3.0 * b - sqrt(root)) / (10.0 * c), false);
        }
    } else if (b != 0.0) at(-a / (3.0 * b), false);
    *of_step = step;
    *of_q = quadratic;
}

// The power of two whose units keep numbers up to `most` (with what rounding adds) below 2^14 and a bit.
int power_for(double most)
{
    int e;
    frexp(fmax(most, 1e-6) * 1.001, &e);            // most <= 2^e
    return kMostPower - e;
}

// Of 32 x 32, one for each CU: up to there they wait less than they read more.  us of 32 x 32 and of 64 x 64: X X^T of 700 x 3000, 253 tiles, 12.9 and 19.2; of
// 768 x 768, 300 tiles, 9.1 and 8.8; of 1024 x 1024, 528 tiles, 14.9 and 10.4; a step of 640 x 640, 400 tiles, 8.6 and 8.4.
constexpr int64_t kFewTiles = 256;

template <Product KIND, typename T>
hipError_t launch_product(ProductArgs g, int32_t n_matrices, hipStream_t st)
{
    constexpr bool kSymmetric = KIND == GRAM || KIND == POLY;
    auto tiles = [&](int64_t r, int64_t c) {
        g.tiles_r = (g.rows + r - 1) / r;
        g.tiles_c = (g.cols + c - 1) / c;
        return (kSymmetric ? g.tiles_r * (g.tiles_r + 1) / 2 : g.tiles_r * g.tiles_c) * n_matrices;
    };
    auto grid = [&] {
        return dim3((uint32_t)(kSymmetric ? (squares_of(g.tiles_r) * kSquare * kSquare * g.parts + 7) / 8 * 8 : tile_blocks(g.tiles_r * g.tiles_c, 1)),
                    (uint32_t)n_matrices);
    };
    if (tiles(kSmallTile, kSmallTile) <= kFewTiles) {
        const int64_t blocks = kSymmetric ? g.tiles_r * (g.tiles_r + 1) / 2 : g.tiles_r * g.tiles_c;
        update_small_product_kernel<KIND, T><<<dim3((uint32_t)blocks, (uint32_t)n_matrices), kSmallWaves * kWave, 0, st>>>(g);
        return hipGetLastError();
    }
    // The largest tiles that there are enough of for all CUs.  us: a step of 2048 x 4096, 256 x 128 and 128 x 128, 104 and 116; two of 1024 x 2048, 128 x 128 and
    // 64 x 64, 38.0 and 39.7.  One matrix of 1024 x 1024, 64 x 64 with eight and with four waves, 193 and 206 in all.
    if constexpr (kSymmetric) {
        if (g.parts > 1 || tiles(128, 128) >= 256) {
            tiles(128, 128);
            update_product_kernel<KIND, T, 128, 128, 2, 1><<<grid(), kBlock, 0, st>>>(g);
            if (g.parts > 1) {
                if (hipError_t e = hipGetLastError()) return e;
                update_join_kernel<KIND, 128><<<dim3((uint32_t)(g.tiles_r * (g.tiles_r + 1) / 2), (uint32_t)n_matrices, 4), kBlock, 0, st>>>(g);
            }
            return hipGetLastError();
        }
    } else {
        if (tiles(256, 128) >= 256) {
            update_product_kernel<KIND, T, 256, 128, 3, 1><<<grid(), kBlock, 0, st>>>(g);
            return hipGetLastError();
        }
        if (tiles(128, 128) >= 200) {
            update_product_kernel<KIND, T, 128, 128, 2, 1><<<grid(), kBlock, 0, st>>>(g);
            return hipGetLastError();
        }
    }
    if (tiles(64, 64) <= 256) update_product_kernel<KIND, T, 64, 64, 4, 2><<<grid(), kBlock * 2, 0, st>>>(g);
    else                      update_product_kernel<KIND, T, 64, 64, 4, 1><<<grid(), kBlock, 0, st>>>(g);
    return hipGetLastError();
}

template <typename T>
hipError_t orthogonalize(const T *g, int64_t ldg, int64_t stride_g, T *out, int64_t ldo, int64_t stride_o, int32_t n_matrices, int64_t n_rows, int64_t n_cols,
                         int32_t n_steps, const float *coef, const int *x_power, const int *a_power, const int *q_power, float eps, uint8_t *work, hipStream_t st)
{
    const UpdateLayout u = update_layout(n_matrices, n_rows, n_cols);
    double *partial = (double *)(work + u.partial_at);
    const int64_t line = 128 / sizeof(T);
    const int64_t written = whole_lines(out, ldo, sizeof(T)) && stride_o * (int64_t)sizeof(T) % 128 == 0 ? (n_cols + line - 1) / line * line : n_cols;
    if (n_steps > 0 && small_update_fits(n_rows, n_cols)) {
        SmallUpdate small{g, out, ldg, stride_g, ldo, stride_o, (int32_t)n_rows, (int32_t)n_cols, (int32_t)written, n_steps, eps, x_power[0]};
        for (int32_t s = 0; s < n_steps; ++s) {
            small.of_gram[s] = ldexpf(1.0f, a_power[s] - 2 * x_power[s]);
            small.of_poly[s] = ldexpf(coef[3 * s + 2], q_power[s] - 2 * a_power[s]);
            small.linear[s] = ldexpf(coef[3 * s + 1], q_power[s] - a_power[s]);
            small.diagonal[s] = ldexpf(coef[3 * s], q_power[s]);
            small.of_step[s] = ldexpf(1.0f, (s + 1 < n_steps ? x_power[s + 1] : 0) - x_power[s] - q_power[s]);
        }
        return launch_small_update(small, n_matrices, sizeof(T) == 4 ? ADAQP_F32 : ADAQP_BF16, st);
    }
    update_norm_kernel<T><<<dim3((uint32_t)u.norm_blocks, (uint32_t)n_matrices), kBlock, 0, st>>>(g, ldg, stride_g, n_rows, n_cols, partial);
    if (hipError_t e = hipGetLastError()) return e;
    if (n_steps == 0) {
        const int64_t blocks = (n_rows * written + kBlock - 1) / kBlock;
        update_scale_kernel<T><<<dim3((uint32_t)(blocks < 2048 ? blocks : 2048), (uint32_t)n_matrices), kBlock, 0, st>>>(
            g, ldg, stride_g, n_rows, n_cols, partial, (int)u.norm_blocks, eps, out, ldo, stride_o, written);
        return hipGetLastError();
    }
    const int64_t lines_n = u.n / 32, lines_m = u.m / 32, pitch_n = held_pitch(u.n), pitch_m = held_pitch(u.m);
    uint8_t *x[2], *xt[2], *a = work + u.a_at, *q = work + u.q_at;
    for (int i = 0; i < 2; ++i) {
        x[i] = work + u.x_at + 2 * i * n_matrices * u.big;
        xt[i] = x[i] + n_matrices * u.big;
    }
    const int64_t tiles_r = padded(n_rows) / 32, tiles_c = padded(n_cols) / 32, tiles = tiles_r * tiles_c;
    update_split_kernel<T><<<dim3((uint32_t)(tiles < 2048 ? tiles : 2048), (uint32_t)n_matrices), kBlock, 0, st>>>(
        g, ldg, stride_g, n_rows, n_cols, partial, (int)u.norm_blocks, eps, x_power[0], u.flip ? xt[0] : x[0], u.flip ? x[0] : xt[0],
        u.flip ? pitch_n : pitch_m, u.flip ? pitch_m : pitch_n, u.big, (uint32_t)tiles_r, (uint32_t)tiles_c);
    if (hipError_t e = hipGetLastError()) return e;
    for (int32_t s = 0; s < n_steps; ++s) {
        const int now = s % 2;
        const float *abc = coef + 3 * s;
        ProductArgs gram{};
        gram.p = gram.q = x[now];
        gram.rows = gram.cols = u.n;
        gram.lines = lines_m;
        gram.pitch = pitch_m;
        gram.same = gram.other = a;
        gram.pitch_same = gram.pitch_other = pitch_n;
        gram.bytes_p = gram.bytes_q = u.big;
        gram.bytes_d = u.small;
        gram.parts = u.parts_m;
        gram.sums = (float *)(work + u.sums_at);
        gram.scale = ldexpf(1.0f, a_power[s] - 2 * x_power[s]);
        if (hipError_t e = launch_product<GRAM, float>(gram, n_matrices, st)) return e;
        ProductArgs poly = gram;
        poly.p = poly.q = a;
        poly.lines = lines_n;
        poly.pitch = pitch_n;
        poly.parts = u.parts_n;
        poly.same = poly.other = q;
        poly.bytes_p = poly.bytes_q = u.small;
        poly.scale = ldexpf(abc[2], q_power[s] - 2 * a_power[s]);
        poly.linear = ldexpf(abc[1], q_power[s] - a_power[s]);
        poly.diagonal = ldexpf(abc[0], q_power[s]);
        if (hipError_t e = launch_product<POLY, float>(poly, n_matrices, st)) return e;
        ProductArgs step{};
        step.parts = 1;
        step.lines = lines_n;
        step.pitch = pitch_n;
        if (s + 1 < n_steps) {                      // X^T Q, stored both ways
            step.p = xt[now];
            step.q = q;
            step.rows = u.m;
            step.cols = u.n;
            step.same = xt[1 - now];
            step.other = x[1 - now];
            step.pitch_same = pitch_n;
            step.pitch_other = pitch_m;
            step.bytes_p = step.bytes_d = u.big;
            step.bytes_q = u.small;
            step.scale = ldexpf(1.0f, x_power[s + 1] - x_power[s] - q_power[s]);
            if (hipError_t e = launch_product<STEP, float>(step, n_matrices, st)) return e;
        } else {                                    // as it lies in out
            step.p = u.flip ? xt[now] : q;
            step.q = u.flip ? q : xt[now];
            step.rows = u.flip ? u.m : u.n;
            step.cols = u.flip ? u.n : u.m;
            step.bytes_p = u.flip ? u.big : u.small;
            step.bytes_q = u.flip ? u.small : u.big;
            step.out = out;
            step.ldo = ldo;
            step.stride_o = stride_o;
            step.out_rows = n_rows;
            step.out_cols = n_cols;
            step.written = written;
            step.scale = ldexpf(1.0f, -x_power[s] - q_power[s]);
            if (hipError_t e = launch_product<LAST, T>(step, n_matrices, st)) return e;
        }
    }
    return hipSuccess;
}

int check_sizes(int32_t n_matrices, int64_t n_rows, int64_t n_cols)
{
    if (n_matrices < 0 || n_rows < 0 || n_cols < 0) return ADAQP_EINVAL;
    return n_matrices > 65535 || n_rows >= kMostSize || n_cols >= kMostSize ? ADAQP_ESIZE : ADAQP_OK;
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_orthogonalize_workspace_bytes(int32_t n_matrices, int64_t n_rows, int64_t n_cols, int64_t *bytes_out)
{
    if (!bytes_out) return ADAQP_EINVAL;
    ADAQP_TRY(check_sizes(n_matrices, n_rows, n_cols));
    *bytes_out = n_matrices && n_rows && n_cols ? update_layout(n_matrices, n_rows, n_cols).bytes : 0;
    return ADAQP_OK;
}

extern "C" int adaqp_orthogonalize(const void *g_dev, int64_t ldg, int64_t stride_g, void *out_dev, int64_t ldo, int64_t stride_o,
                                   int32_t n_matrices, int64_t n_rows, int64_t n_cols, int32_t type, int32_t n_steps, const float *coef_host, float eps,
                                   void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    ADAQP_TRY(check_sizes(n_matrices, n_rows, n_cols));
    if (!valid_type(type) || n_steps < 0 || (n_steps > 0 && !coef_host) || !(eps >= 0.0f && eps <= 3.402823466e+38f)) return ADAQP_EINVAL;
    if (n_steps > kMostSteps) return ADAQP_ESIZE;
    int x_power[kMostSteps + 1], a_power[kMostSteps], q_power[kMostSteps];
    double most = 1.0;
    for (int32_t s = 0; s < n_steps; ++s) {
        double step, quadratic;
        bounds(coef_host[3 * s], coef_host[3 * s + 1], coef_host[3 * s + 2], most, &step, &quadratic);
        if (!(step <= ADAQP_ORTHOGONALIZE_MOST)) return ADAQP_EINVAL;
        x_power[s] = power_for(most);
        a_power[s] = power_for(most * most);
        q_power[s] = power_for(quadratic);
        x_power[s + 1] = power_for(step);
        most = fmax(step, 1e-6);
    }
    if (n_matrices == 0 || n_rows == 0 || n_cols == 0) return ADAQP_OK;
    const int64_t bytes = element_bytes(type);
    if (!g_dev || !out_dev || ldg < n_cols || ldo < n_cols || !aligned_to(g_dev, bytes) || !aligned_to(out_dev, bytes)) return ADAQP_EINVAL;
    if (n_matrices > 1 && (stride_g < n_rows * ldg || stride_o < n_rows * ldo)) return ADAQP_EINVAL;
    if (g_dev == out_dev && (ldg != ldo || (n_matrices > 1 && stride_g != stride_o))) return ADAQP_EINVAL;
    const UpdateLayout u = update_layout(n_matrices, n_rows, n_cols);
    if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
    if (workspace_bytes < u.bytes) return ADAQP_ESIZE;
    if (type == ADAQP_F32)
        ADAQP_HIP_TRY((orthogonalize<float>((const float *)g_dev, ldg, stride_g, (float *)out_dev, ldo, stride_o, n_matrices, n_rows, n_cols, n_steps, coef_host,
                                            x_power, a_power, q_power, eps, (uint8_t *)workspace_dev, (hipStream_t)stream)));
    else
        ADAQP_HIP_TRY((orthogonalize<__bf16>((const __bf16 *)g_dev, ldg, stride_g, (__bf16 *)out_dev, ldo, stride_o, n_matrices, n_rows, n_cols, n_steps,
                                             coef_host, x_power, a_power, q_power, eps, (uint8_t *)workspace_dev, (hipStream_t)stream)));
    return ADAQP_OK;
}
