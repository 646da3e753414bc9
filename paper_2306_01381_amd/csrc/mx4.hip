// MX matrices: writing them from rows, columns or both, and reading them back (adaqp_dense.h).
//
// 4 lanes hold a block of 32 columns, 8 neighbouring ones each (a granule: one Philox call, one 32-bit word of codes).  Where only the rows' form is wanted
// the blocks of all rows are dealt out in a row, so that no lane stands for columns that do not exist.  For the columns' form a workgroup takes a tile of 128
// columns and 64 rows through the LDS once, and a lane takes 32 rows of one column.  x is read once whichever of the two forms is wanted.  To nearest, the
// conversions are gfx950's own, two values an instruction, and all is bound by memory: 4 bytes read per element of fp32 and 0.53 written per form.
// Stochastically the vector instructions are as long at work as the memory: of each element and form 17 where both forms are made, 8 of them Philox, and 26 where only
// the rows' are, whose 8 values at a time look for their row and its end.
// Measured: 58 000 x 602 fp32 to nearest, rows' form, 35 us (159 MB, 4.5 TB/s), both forms, as a layer's forward pass in training makes them, 38 us (177 MB, 4.7 TB/s);
// 196 000 x 256 fp32, both forms, stochastic, 67 us of unpadded rows (254 MB, 3.8 TB/s), 55 of padded ones; half of the LDS's cycles are conflicts of the lanes that write the tile.
// 179 000 x 300 bf16, rows' form, stochastic, 43 us (143 MB, 3.3 TB/s), and read back 29 us (143 MB, 5.0 TB/s).
#include "mx4.hpp"
#include "philox.hpp"

namespace adaqp {
namespace {

constexpr uint32_t kMxTag = 0x4d583443u;
constexpr uint32_t kLargestByte = 126 + 127;        // of magnitudes beyond 1.5 * 2^127, to be rounded stochastically
constexpr int kLanes = kMxChunk / 8;                // of a row
constexpr int kPassRows = kBlock / kLanes;          // a lane has one row of each pass

struct MxArgs {
    const void *x;
    int64_t ld, n_rows, n_cols;
    uint32_t tiles_r, tiles_c;
    uint32_t row_blocks;                            // blocks of a row that have columns
    uint32_t row_factor, row_shift;                 // n / row_blocks = n * row_factor >> row_shift for the n below 2^31 that there are; 0: there are more
    int ragged;                                     // 0: all blocks are full; else the last may end inside a vector (1) or not (2)
    uint64_t seed;
    uint8_t *codes, *scales, *codes_t, *scales_t;
    int64_t pitch, pitch_t;
};

// The scale byte of a block whose largest magnitude has these bits (sign cleared).
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    const int field = (int)(most >> 23);
    if (field == 255) return 255;                               // an infinity or NaN
    const int byte = field - 2 + (STOCHASTIC && (most & 0x7FFFFFu) > 0x400000u ? 1 : 0);       // beyond 1.5 * 2^floor: 6 * 2^e would be passed
    return byte < 0 ? 0 : byte;
}

// The codes of 8 values, low nibble first.
__device__ __forceinline__ uint32_t nearest_codes(const float (&x)[8], uint32_t byte)
{
    const float scale = __builtin_bit_cast(float, byte << 23);  // the conversion goes by its exponent
    uint32_t word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], scale, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], scale, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], scale, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], scale, 3);
    return byte == 255 ? 0 : word;
}

// Scaled so that 1 is the smallest normal fp32 number, a block's values have the code's own form: below 1 subnormal numbers, from there on exponent and first
// fraction bit.  Bits 22..24 are the code below the value, the 22 bits behind them the share of the way to the next, and adding the random number to
// the upper 16 of those carries into the code as often as it should.  What is shifted out of a subnormal number has to be cut off: round_toward_zero().
__device__ __forceinline__ uint32_t stochastic_codes(const float (&x)[8], uint32_t byte, const Rand128 &rnd)
{
    const uint32_t w[4] = {rnd.w0, rnd.w1, rnd.w2, rnd.w3};
    const int power = 127 - 126 - (int)byte;
    uint32_t codes = 0, signs = 0;
#pragma unroll
    for (int j = 7; j >= 0; --j) signs = __builtin_amdgcn_alignbit(signs, __builtin_bit_cast(uint32_t, x[j]), 28);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t r = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
        codes |= ((__builtin_bit_cast(uint32_t, __builtin_amdgcn_ldexpf(fabsf(x[j]), power)) + (r << 6)) >> 22) << (4 * j);
    }
    if (byte == kLargestByte) {                     // no fp32 number is 4 * 2^126: of magnitudes there (up to 4 units) code 6 becomes 5
        const uint32_t six = codes >> 2 & codes >> 1 & 0x11111111u;
        codes -= six;
    }
    return byte == 255 ? 0 : (codes & 0x77777777u) | (signs & 0x88888888u);
}

// For the wave that calls it and all its fp32 arithmetic from there on: bits 0 and 1 of the mode register.
__device__ __forceinline__ void round_toward_zero() { __builtin_amdgcn_s_setreg(1 | 0 << 6 | (2 - 1) << 11, 3); }

__device__ __forceinline__ Rand128 random_words(uint64_t seed, int64_t row, int64_t granule)
{
    return philox4x32_10((uint32_t)granule, (uint32_t)row, 0u, kMxTag, (uint32_t)seed, (uint32_t)(seed >> 32));
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

// The largest magnitude, NaN where there is one.
template <int N>
__device__ __forceinline__ float largest(const float (&x)[N])
{
    float most = __builtin_elementwise_maximum(fabsf(x[0]), fabsf(x[1]));
#pragma unroll
    for (int k = 2; k < N; k += 2) most = __builtin_elementwise_maximum(most, __builtin_elementwise_maximum(fabsf(x[k]), fabsf(x[k + 1])));
    return most;
}

template <int PATTERN>
__device__ __forceinline__ uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, PATTERN, 0xF, 0xF, false);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;       // partners of a butterfly over 16 lanes

// 8 columns of a row from col on.  No branches, so that many such loads are under way together: what lies behind the last vector is loaded from there and set to
// zero afterwards (keep_granule).
template <typename T, int VW>
__device__ __forceinline__ void load_granule(const MxArgs &a, int64_t row, int64_t col, float (&x)[8])
{
    const T *from = (const T *)a.x + min(row, a.n_rows - 1) * a.ld;
    const int64_t last = (a.n_cols - 1) / VW * VW;
#pragma unroll
    for (int v = 0; v < 8; v += VW) {
        float part[VW];
        load_elements<T, VW>(from + min(col + v, last), part);
#pragma unroll
        for (int k = 0; k < VW; ++k) x[v + k] = part[k];
    }
}

// STEP: columns that are there or not together.
template <int STEP>
__device__ __forceinline__ void keep_granule(const MxArgs &a, int64_t row, int64_t col, float (&x)[8])
{
    const int left = row < a.n_rows ? (int)min(a.n_cols - col, (int64_t)8) : 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = k / STEP * STEP < left ? x[k] : 0.0f;
}

// The rows' form alone: blocks of 32 columns, kEach for a lane, row by row.
template <typename T, int VW, bool STOCHASTIC>
__global__ __launch_bounds__(kBlock) void mx4_quantize_rows_kernel(MxArgs a)
{
    constexpr int kEach = 2, kBlocks = kBlock / 4;
    if (STOCHASTIC) round_toward_zero();            // nothing but the scaling rounds here
    const uint64_t first = (uint64_t)xcd_neighbour(workgroup(), workgroups()) * (kBlocks * kEach) + threadIdx.x / 4;
    const int l = threadIdx.x % 4;
    int64_t row[kEach];
    uint32_t block[kEach];
    float x[kEach][8];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint64_t at = first + e * kBlocks;    // may lie behind the last block: so does its row then
        row[e] = a.row_factor ? (uint64_t)(uint32_t)at * a.row_factor >> a.row_shift : at / a.row_blocks;
        block[e] = (uint32_t)at - (uint32_t)row[e] * a.row_blocks;
        load_granule<T, VW>(a, row[e], block[e] * kMxBlock + l * 8, x[e]);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (a.ragged == 1) keep_granule<1>(a, row[e], block[e] * kMxBlock + l * 8, x[e]);
        if (a.ragged > 1) keep_granule<VW>(a, row[e], block[e] * kMxBlock + l * 8, x[e]);
        uint32_t most = magnitude(largest<8>(x[e]));
        most = max(most, moved<kSwap1>(most));
        most = max(most, moved<kSwap2>(most));
        const uint32_t byte = scale_byte<STOCHASTIC>(most);
        const uint32_t word = STOCHASTIC ? stochastic_codes(x[e], byte, random_words(a.seed, row[e], block[e] * 4 + l)) : nearest_codes(x[e], byte);
        if (row[e] >= a.n_rows) continue;
        uint8_t *codes = a.codes + row[e] * a.pitch, *scales = a.scales + row[e] * 4;
        *reinterpret_cast<uint32_t *>(codes + block[e] * 16 + l * 4) = word;
        if (l == 0) scales[block[e] / 4 * a.n_rows * 4 + block[e] % 4] = (uint8_t)byte;
        if (block[e] + 1 == a.row_blocks)           // the rest of the chunk
            for (uint32_t b = block[e] + 1; b % 4 != 0; ++b) {
                *reinterpret_cast<uint32_t *>(codes + b * 16 + l * 4) = 0;
                if (l == 0) scales[b / 4 * a.n_rows * 4 + b % 4] = 0;
            }
    }
}

constexpr int kTileRows = 64;
struct alignas(16) Tile { float v[kTileRows * kMxChunk]; };

// The columns' form, and the rows'.
template <typename T, int VW, bool ROWS, bool STOCHASTIC>
__global__ __launch_bounds__(kBlock) void mx4_quantize_kernel(MxArgs a)
{
    constexpr int kRows = kTileRows, kPasses = kRows / kPassRows;
    __shared__ Tile tile_of;
    static_assert(alignof(Tile) % alignof(float4) == 0, "written in vectors");
    float *tile = tile_of.v;
    if (STOCHASTIC) round_toward_zero();
    // an XCD gets neighbouring tiles, four tile rows together: their parts of the columns' lines meet in its L2
    constexpr uint32_t kGroup = 4;
    const uint32_t at = xcd_neighbour(workgroup(), workgroups());
    const uint32_t group = at / (kGroup * a.tiles_c), in_group = at % (kGroup * a.tiles_c);
    if (group * kGroup >= a.tiles_r) return;
    const uint32_t rows = min(kGroup, a.tiles_r - group * kGroup);
    const int64_t tile_r = group * kGroup + in_group % rows, chunk_c = in_group / rows;
    if (chunk_c >= a.tiles_c) return;
    const int l = threadIdx.x % kLanes, r = threadIdx.x / kLanes;
    float x[kPasses][8];
    const int64_t col = chunk_c * kMxChunk + l * 8;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        load_granule<T, VW>(a, tile_r * kRows + p * kPassRows + r, col, x[p]);
    }
    if ((tile_r + 1) * kRows > a.n_rows || (chunk_c + 1) * kMxChunk > a.n_cols)
#pragma unroll
        for (int p = 0; p < kPasses; ++p) keep_granule<1>(a, tile_r * kRows + p * kPassRows + r, col, x[p]);
    {
        // rows 32 .. 63 are turned by 32 columns: then the lanes of a wave, 32 columns of both blocks, read 64 banks
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int row = p * kPassRows + r;
            float *to = tile + row * kMxChunk + (l * 8 + row / kMxBlock * 32) % kMxChunk;
#pragma unroll
            for (int k = 0; k < 8; k += 4) *reinterpret_cast<float4 *>(to + k) = make_float4(x[p][k], x[p][k + 1], x[p][k + 2], x[p][k + 3]);
        }
    }
    if (ROWS) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int64_t row = tile_r * kRows + p * kPassRows + r;
            uint32_t most = magnitude(largest<8>(x[p]));
            most = max(most, moved<kSwap1>(most));
            most = max(most, moved<kSwap2>(most));
            const uint32_t byte = scale_byte<STOCHASTIC>(most);
            const uint32_t word = STOCHASTIC ? stochastic_codes(x[p], byte, random_words(a.seed, row, col / 8)) : nearest_codes(x[p], byte);
            uint32_t scales = byte << (8 * (l / 4));
            scales |= moved<kMirror8>(scales);
            scales |= moved<kMirror16>(scales);
            if (row < a.n_rows) {
                *reinterpret_cast<uint32_t *>(a.codes + row * a.pitch + chunk_c * kMxChunkBytes + l * 4) = word;
                if (l == 0) *reinterpret_cast<uint32_t *>(a.scales + (chunk_c * a.n_rows + row) * 4) = scales;
            }
        }
    }
    __syncthreads();
    {
        const int b = threadIdx.x % 2, c = threadIdx.x / 2;     // block of 32 rows, column
        const int64_t row = chunk_c * kMxChunk + c;             // of the transpose
        if (row >= a.n_cols) return;
        const float *from = tile + b * kMxBlock * kMxChunk + (c + 32 * b) % kMxChunk;
        float v[4][8];
#pragma unroll
        for (int k = 0; k < kMxBlock; ++k) v[k / 8][k % 8] = from[k * kMxChunk];
        uint32_t most = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) most = max(most, magnitude(largest<8>(v[g])));
        const uint32_t byte = scale_byte<STOCHASTIC>(most);
        uint32_t word[4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
            word[g] = STOCHASTIC ? stochastic_codes(v[g], byte, random_words(a.seed + 1, row, tile_r * (kRows / 8) + b * 4 + g)) : nearest_codes(v[g], byte);
        const uint32_t scales = byte << (8 * b) | moved<kSwap1>(byte << (8 * b));
        const int64_t chunk_r = tile_r / 2, part = tile_r % 2;  // of the transpose's columns
        *reinterpret_cast<uint4 *>(a.codes_t + row * a.pitch_t + chunk_r * kMxChunkBytes + (part * 2 + b) * 16) = make_uint4(word[0], word[1], word[2], word[3]);
        if (b == 0) *reinterpret_cast<uint16_t *>(a.scales_t + (chunk_r * a.n_cols + row) * 4 + part * 2) = (uint16_t)scales;
    }
}

// 8 values of one word of codes.
__device__ __forceinline__ void values_of(uint32_t word, uint32_t byte, float (&v)[8])
{
    // the conversion goes by the scale's exponent; 255 is NaN
    const float scale = __builtin_bit_cast(float, byte << 23), nan = __builtin_nanf("");
    const auto put = [&](int j, auto pair) {
        v[j] = byte == 255 ? nan : pair[0];
        v[j + 1] = byte == 255 ? nan : pair[1];
    };
    put(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 0));
    put(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 1));
    put(4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 2));
    put(6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 3));
}

template <typename T, int VW, bool WHOLE>
__global__ __launch_bounds__(kBlock) void mx4_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, int64_t n_rows, int64_t n_cols, int64_t written,
                                                                int64_t pitch, T *x, int64_t ld, int64_t granules)
{
    const uint64_t at = (uint64_t)workgroup() * kBlock + threadIdx.x;
    const int64_t row = at >> 32 ? at / (uint64_t)granules : (uint32_t)at / (uint32_t)granules, g = at - row * granules;
    if (row >= n_rows) return;
    float v[8];
    if (g * 8 < n_cols) values_of(*reinterpret_cast<const uint32_t *>(codes + row * pitch + g * 4), scales[(g / 16 * n_rows + row) * 4 + g / 4 % 4], v);
    else for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    T *to = x + row * ld + g * 8;
#pragma unroll
    for (int k = 0; k < 8; k += VW) {
        float part[VW];
#pragma unroll
        for (int j = 0; j < VW; ++j) part[j] = g * 8 + k + j < n_cols ? v[k + j] : 0.0f;
        if (g * 8 + k + VW <= written) store_elements<T, VW, WHOLE>(to + k, part);
        else for (int j = 0; j < VW; ++j) if (g * 8 + k + j < written) to[k + j] = (T)part[j];
    }
}

template <typename T, int VW>
void launch_quantize(const MxArgs &a, int32_t rounding, int64_t blocks, hipStream_t st)
{
    auto go = [&](auto stochastic) {
        constexpr bool S = decltype(stochastic)::value;
        if (!a.codes_t)   mx4_quantize_rows_kernel<T, VW, S><<<grid_of(blocks, kBlock), kBlock, 0, st>>>(a);
        else if (a.codes) mx4_quantize_kernel<T, VW, true, S><<<grid_of(blocks, kBlock), kBlock, 0, st>>>(a);
        else              mx4_quantize_kernel<T, VW, false, S><<<grid_of(blocks, kBlock), kBlock, 0, st>>>(a);
    };
    if (rounding == ADAQP_MX4_STOCHASTIC) go(std::true_type());
    else                                  go(std::false_type());
}

template <typename T>
hipError_t launch_quantize(const MxArgs &a, int vw, int32_t rounding, int64_t blocks, hipStream_t st)
{
    if (vw * (int)sizeof(T) == 16)     launch_quantize<T, 16 / sizeof(T)>(a, rounding, blocks, st);
    else if (vw * (int)sizeof(T) == 8) launch_quantize<T, 8 / sizeof(T)>(a, rounding, blocks, st);
    else                               launch_quantize<T, 1>(a, rounding, blocks, st);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t n_rows, int64_t n_cols, void *x, int64_t ld, hipStream_t st)
{
    const bool whole = whole_lines(x, ld, sizeof(T));
    const int64_t line = 128 / sizeof(T), written = whole ? (n_cols + line - 1) / line * line : n_cols;
    const int64_t granules = (written + 7) / 8, blocks = (n_rows * granules + kBlock - 1) / kBlock;
    constexpr int VW = 16 / sizeof(T);
    int vw = VW;
    while (vw > 1 && (!aligned_to(x, vw * sizeof(T)) || ld % vw != 0)) vw /= 2;
    auto go = [&](auto vw, auto lines) {
        mx4_dequantize_kernel<T, decltype(vw)::value, decltype(lines)::value>
            <<<grid_of(blocks, kBlock), kBlock, 0, st>>>(codes, scales, n_rows, n_cols, written, mx_pitch(n_cols), (T *)x, ld, granules);
    };
    if (whole)              go(std::integral_constant<int, VW>(), std::true_type());
    else if (vw == VW)      go(std::integral_constant<int, VW>(), std::false_type());
    else if (vw == VW / 2)  go(std::integral_constant<int, VW / 2>(), std::false_type());
    else                    go(std::integral_constant<int, 1>(), std::false_type());
    return hipGetLastError();
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int64_t adaqp_mx4_code_bytes(int64_t n_rows, int64_t n_cols)
{
    if (n_rows < 0 || n_cols < 0 || n_rows >= kMxMost || n_cols >= kMxMost) return -1;
    return n_rows * mx_pitch(n_cols);
}

extern "C" int64_t adaqp_mx4_scale_bytes(int64_t n_rows, int64_t n_cols)
{
    if (n_rows < 0 || n_cols < 0 || n_rows >= kMxMost || n_cols >= kMxMost) return -1;
    return n_rows * mx_chunks(n_cols) * 4;
}

extern "C" int adaqp_mx4_quantize(const void *x_dev, int64_t ld, int64_t n_rows, int64_t n_cols, int32_t type, int32_t rounding, uint64_t seed,
                                  uint8_t *codes_dev, uint8_t *scales_dev, uint8_t *codes_t_dev, uint8_t *scales_t_dev, void *stream)
{
    if (n_rows < 0 || n_cols < 0 || !valid_type(type) || (rounding != ADAQP_MX4_NEAREST && rounding != ADAQP_MX4_STOCHASTIC)) return ADAQP_EINVAL;
    if (!codes_dev != !scales_dev || !codes_t_dev != !scales_t_dev) return ADAQP_EINVAL;
    if (n_rows >= kMxMost || n_cols >= kMxMost) return ADAQP_ESIZE;
    if (n_rows == 0 || n_cols == 0 || (!codes_dev && !codes_t_dev)) return ADAQP_OK;
    if (!x_dev || ld < n_cols || !aligned_to(x_dev, element_bytes(type))) return ADAQP_EINVAL;
    if ((codes_dev && !valid_mx(codes_dev, scales_dev)) || (codes_t_dev && !valid_mx(codes_t_dev, scales_t_dev))) return ADAQP_EINVAL;
    // the columns' form writes whole chunks of 128 rows: two tiles of 64
    const int64_t tiles_r = mx_chunks(n_rows) * 2, tiles_c = mx_chunks(n_cols), row_blocks = (n_cols + kMxBlock - 1) / kMxBlock;
    const int64_t blocks = ((codes_t_dev ? tiles_r * tiles_c : (n_rows * row_blocks + kBlock / 2 - 1) / (kBlock / 2)) + 7) / 8 * 8;
    if (blocks > kMostWorkgroups) return ADAQP_ESIZE;
    const int64_t bytes = element_bytes(type);
    const int vw = whole_lines(x_dev, ld, bytes) ? (int)(16 / bytes) : vector_elements(x_dev, ld, n_cols, bytes);       // in its own lines a vector may pass the last column
    int bits = 0;
    while (((int64_t)1 << bits) < row_blocks) ++bits;
    const bool below = n_rows * row_blocks + kBlock < ((int64_t)1 << 31);
    const uint64_t factor = (((uint64_t)1 << (31 + bits)) + row_blocks - 1) / row_blocks;      // below 2^32: row_blocks is above 2^(bits - 1)
    MxArgs a{x_dev, ld, n_rows, n_cols, (uint32_t)tiles_r, (uint32_t)tiles_c, (uint32_t)row_blocks, below ? (uint32_t)factor : 0, (uint32_t)(31 + bits),
             n_cols % kMxBlock == 0 ? 0 : n_cols % vw ? 1 : 2, seed, codes_dev, scales_dev, codes_t_dev, scales_t_dev, mx_pitch(n_cols),
             mx_pitch(n_rows)};
    if (type == ADAQP_F32) ADAQP_HIP_TRY((launch_quantize<float>(a, vw, rounding, blocks, (hipStream_t)stream)));
    else                   ADAQP_HIP_TRY((launch_quantize<__bf16>(a, vw, rounding, blocks, (hipStream_t)stream)));
    return ADAQP_OK;
}

extern "C" int adaqp_mx4_dequantize(const uint8_t *codes_dev, const uint8_t *scales_dev, int64_t n_rows, int64_t n_cols, void *x_dev, int64_t ld,
                                    int32_t type, void *stream)
{
    if (n_rows < 0 || n_cols < 0 || !valid_type(type)) return ADAQP_EINVAL;
    if (n_rows >= kMxMost || n_cols >= kMxMost) return ADAQP_ESIZE;
    if (n_rows == 0 || n_cols == 0) return ADAQP_OK;
    if (!valid_mx(codes_dev, scales_dev) || !x_dev || ld < n_cols || !aligned_to(x_dev, element_bytes(type))) return ADAQP_EINVAL;
    if ((n_cols + 127) / 8 * n_rows / kBlock >= kMostWorkgroups) return ADAQP_ESIZE;
    if (type == ADAQP_F32) ADAQP_HIP_TRY((launch_dequantize<float>(codes_dev, scales_dev, n_rows, n_cols, x_dev, ld, (hipStream_t)stream)));
    else                   ADAQP_HIP_TRY((launch_dequantize<__bf16>(codes_dev, scales_dev, n_rows, n_cols, x_dev, ld, (hipStream_t)stream)));
    return ADAQP_OK;
}
