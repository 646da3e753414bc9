// Products of MX matrices on the matrix cores (adaqp_dense.h): out = a b^T, both operands rows of k columns.
//
// gfx950's scaled products take 4-bit codes and a power of two for 32 of them as they lie in memory: nothing is unpacked.  A workgroup of four waves
// takes a tile of BM x BN outputs, a quarter each wave, and walks k in steps of 256 columns, a line of 128 bytes of a row.  The next step's codes and
// scales go from memory straight into the LDS while the current one is multiplied.
//
// Where the tiles are few, k is split over workgroups; the parts' sums, fp32, are added in order by a second kernel.
#include "lines.hpp"
#include "mx4.hpp"

namespace adaqp {
namespace {

constexpr int kStepChunks = 2;                      // scale words

typedef int mx_codes __attribute__((ext_vector_type(8)));       // of which 4-bit codes fill the first half
typedef float mx_sums __attribute__((ext_vector_type(16)));

struct MulArgs {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    void *out;
    int64_t m, n, ldo;
    int64_t written;                                // columns of out: n, or its whole lines
    int64_t pitch;                                  // of a row of codes, both operands
    int64_t chunks;                                 // scale words of a row
    int64_t steps, steps_per_split;
    int64_t tiles_m, tiles_n;
};

// A step's scales of ROWS rows into the LDS, [2][ROWS] words.
template <int ROWS>
__device__ __forceinline__ void load_scales(const uint8_t *scales, int64_t row0, int64_t n_rows, int64_t chunks, int64_t step, uint8_t *lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
#pragma unroll
    for (int i = 0; i < (ROWS * kStepChunks + kBlock - 1) / kBlock; ++i) {
        const int first = (i * kWavesPerBlock + wave) * kWave;  // words
        if (ROWS * kStepChunks < kBlock && first >= ROWS * kStepChunks) break;
        const int64_t row = row0 + first % ROWS + lane, chunk = step * kStepChunks + first / ROWS;
        load_to_lds_4(row < n_rows && chunk < chunks ? (const void *)(scales + (chunk * n_rows + row) * 4) : zeros(), lds + first * 4);
    }
}

template <int BM, int BN>
struct Stage {
    uint8_t a[BM * kLine], b[BN * kLine];
    uint8_t sa[BM * kStepChunks * 4], sb[BN * kStepChunks * 4];
};

template <typename T, int BM, int BN>
__global__ __launch_bounds__(kBlock) void mx4_matmul_kernel(MulArgs g)
{
    constexpr int FM = BM / 64, FN = BN / 64;       // 32 x 32 parts of a wave
    __shared__ Stage<BM, BN> stage[2];
    const int64_t tiles = g.tiles_m * g.tiles_n;
    const int64_t split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int64_t row0 = tile / g.tiles_n * BM, col0 = tile % g.tiles_n * BN;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int wm = wave / 2 * (BM / 2), wn = wave % 2 * (BN / 2);
    const int64_t begin = split * g.steps_per_split, end = min(begin + g.steps_per_split, g.steps);

    auto load = [&](int64_t step, Stage<BM, BN> &s) {
        load_lines<BM>(g.a_codes, row0, g.m, g.pitch, step, s.a);
        load_lines<BN>(g.b_codes, col0, g.n, g.pitch, step, s.b);
        load_scales<BM>(g.a_scales, row0, g.m, g.chunks, step, s.sa);
        load_scales<BN>(g.b_scales, col0, g.n, g.chunks, step, s.sb);
    };
    mx_sums sums[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) sums[i][j][q] = 0.0f;

    if (begin < end) load(begin, stage[0]);
    landed();
    for (int64_t step = begin; step < end; ++step) {
        const Stage<BM, BN> &s = stage[(step - begin) % 2];
        if (step + 1 < end) load(step + 1, stage[(step - begin + 1) % 2]);
#pragma unroll
        for (int c = 0; c < kStepChunks; ++c) {
            uint32_t sa[FM], sb[FN];                // of this lane's rows; the upper half of a wave has the odd blocks
#pragma unroll
            for (int i = 0; i < FM; ++i) sa[i] = *reinterpret_cast<const uint32_t *>(s.sa + (c * BM + wm + i * 32 + r) * 4) >> (8 * h);
#pragma unroll
            for (int j = 0; j < FN; ++j) sb[j] = *reinterpret_cast<const uint32_t *>(s.sb + (c * BN + wn + j * 32 + r) * 4) >> (8 * h);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int part = c * 4 + q * 2 + h;
                mx_codes a[FM], b[FN];
                auto codes = [&](const uint8_t *lines, int row) {
                    const int4 v = *reinterpret_cast<const int4 *>(line_part(lines, row, part));
                    return mx_codes{v.x, v.y, v.z, v.w, 0, 0, 0, 0};
                };
#pragma unroll
                for (int i = 0; i < FM; ++i) a[i] = codes(s.a, wm + i * 32 + r);
#pragma unroll
                for (int j = 0; j < FN; ++j) b[j] = codes(s.b, wn + j * 32 + r);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        sums[i][j] = q == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i], b[j], sums[i][j], 4, 4, 0, (int)sa[i], 0, (int)sb[j])
                                            : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i], b[j], sums[i][j], 4, 4, 2, (int)sa[i], 2, (int)sb[j]);
            }
        }
        landed();
    }

    T *out = (T *)g.out + (split ? split * g.m * g.n : 0);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int64_t row = row0 + wm + i * 32 + q / 4 * 8 + h * 4 + q % 4, col = col0 + wn + j * 32 + r;
                if (row < g.m && col < g.written) out[row * g.ldo + col] = col < g.n ? (T)sums[i][j][q] : (T)0.0f;
            }
}

// The splits' sums, in order; columns from n to `written` are zeros.
template <typename T>
__global__ __launch_bounds__(kBlock) void mx4_join_kernel(const float *parts, int64_t n_parts, int64_t m, int64_t n, int64_t written, T *out, int64_t ldo)
{
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < m * written; at += (int64_t)gridDim.x * kBlock) {
        const int64_t row = at / written, col = at % written;
        float sum = 0.0f;
        if (col < n)
            for (int64_t s = 0; s < n_parts; ++s) sum += parts[(s * m + row) * n + col];
        out[row * ldo + col] = (T)sum;
    }
}

struct MulShape {
    int tile;
    int64_t tiles_m, tiles_n, steps, splits, steps_per_split, bytes;
};

MulShape mul_shape(int64_t m, int64_t n, int64_t k)
{
    MulShape s{};
    auto tiles = [&](int t) {
        s.tile = t;
        s.tiles_m = (m + t - 1) / t;
        s.tiles_n = (n + t - 1) / t;
        return s.tiles_m * s.tiles_n;
    };
    if (tiles(128) < 256) tiles(64);
    const int64_t blocks = s.tiles_m * s.tiles_n;
    s.steps = (mx_chunks(k) + kStepChunks - 1) / kStepChunks;
    int64_t splits = blocks >= 256 || blocks == 0 ? 1 : 512 / blocks;
    if (splits > s.steps / 2) splits = s.steps / 2;
    if (splits < 1) splits = 1;
    s.steps_per_split = (s.steps + splits - 1) / splits;
    s.splits = s.steps ? (s.steps + s.steps_per_split - 1) / s.steps_per_split : 1;
    s.bytes = s.splits > 1 ? (s.splits * m * n * 4 + 255) / 256 * 256 : 0;
    return s;
}

template <typename T>
void launch_tiles(const MulArgs &g, const MulShape &s, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)(s.tiles_m * s.tiles_n * s.splits);
    if (s.tile == 128) mx4_matmul_kernel<T, 128, 128><<<blocks, kBlock, 0, st>>>(g);
    else               mx4_matmul_kernel<T, 64, 64><<<blocks, kBlock, 0, st>>>(g);
}

int check_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return ADAQP_EINVAL;
    return m >= kMxMost || n >= kMxMost || k >= kMxMost || (m + 63) / 64 * ((n + 63) / 64) >= 0x7FFFFFFF ? ADAQP_ESIZE : ADAQP_OK;
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_mx4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t *bytes_out)
{
    if (!bytes_out) return ADAQP_EINVAL;
    ADAQP_TRY(check_sizes(m, n, k));
    *bytes_out = mul_shape(m, n, k).bytes;
    return ADAQP_OK;
}

extern "C" int adaqp_mx4_matmul(const uint8_t *a_codes_dev, const uint8_t *a_scales_dev, int64_t m,
                                const uint8_t *b_codes_dev, const uint8_t *b_scales_dev, int64_t n, int64_t k,
                                void *out_dev, int64_t ldo, int32_t type, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    ADAQP_TRY(check_sizes(m, n, k));
    if (!valid_type(type)) return ADAQP_EINVAL;
    if (m == 0 || n == 0) return ADAQP_OK;
    if (!out_dev || ldo < n || !aligned_to(out_dev, element_bytes(type))) return ADAQP_EINVAL;
    if (k > 0 && (!valid_mx(a_codes_dev, a_scales_dev) || !valid_mx(b_codes_dev, b_scales_dev))) return ADAQP_EINVAL;
    const MulShape s = mul_shape(m, n, k);
    if (s.splits > 1) {
        if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
        if (workspace_bytes < s.bytes) return ADAQP_ESIZE;
    }
    MulArgs g{a_codes_dev, a_scales_dev, b_codes_dev, b_scales_dev, out_dev, m, n, ldo, 0, mx_pitch(k), mx_chunks(k), s.steps, s.steps_per_split,
              s.tiles_m, s.tiles_n};
    const hipStream_t st = (hipStream_t)stream;
    const int64_t line = 128 / element_bytes(type);
    const int64_t written = whole_lines(out_dev, ldo, element_bytes(type)) ? (n + line - 1) / line * line : n;
    g.written = s.splits > 1 ? n : written;
    if (s.splits > 1) {
        g.out = workspace_dev;
        g.ldo = n;
        launch_tiles<float>(g, s, st);
        ADAQP_HIP_TRY(hipGetLastError());
        const int64_t blocks = (m * written + kBlock - 1) / kBlock;
        const uint32_t grid = (uint32_t)(blocks < 4096 ? blocks : 4096);
        if (type == ADAQP_F32) mx4_join_kernel<float><<<grid, kBlock, 0, st>>>((const float *)workspace_dev, s.splits, m, n, written, (float *)out_dev, ldo);
        else                   mx4_join_kernel<__bf16><<<grid, kBlock, 0, st>>>((const float *)workspace_dev, s.splits, m, n, written, (__bf16 *)out_dev, ldo);
    } else if (type == ADAQP_F32) launch_tiles<float>(g, s, st);
    else                          launch_tiles<__bf16>(g, s, st);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}
