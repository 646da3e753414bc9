// Matrices in 8 bits: writing them from rows, columns or both, and reading them back (adaqp_train.h).
//
// 16 lanes hold the 128 columns of a block, 8 neighbouring ones each.  Where only the rows' form with a scale for each row is wanted the blocks of all rows are dealt out in a row; else a
// workgroup takes a tile of 128 columns and 128 rows in registers.  x is read once.  Bound by memory.  Measured: 58 000 x 602 fp32 rows 27 us (176 MB, 6.5 TB/s, in part from the last cache), both forms 40 us (5.2 TB/s; 68 with fp32 values
// turned in the LDS, of which two workgroups fit a CU), on operands that no cache holds 33 and 45; with a scale for a tile 36 and 44; 179 000 x 300 bf16 rows 30 us, read back 28 us (5.7 TB/s).
#include "f8.hpp"
#include "rows.hpp"

namespace adaqp {
namespace {

constexpr uint32_t kLargestByte = 120 + 127;        // of magnitudes beyond 1.75 * 2^127

struct F8Args {
    const void *x;
    int64_t ld, n_rows, n_cols, span;
    int64_t chunks;                                 // of a row
    uint64_t blocks;                                // of all rows
    Divider chunks_of_row;
    uint32_t tiles_r, tiles_c;
    uint8_t *codes, *scales, *codes_t, *scales_t;
    int64_t scale_pitch, pitch_t, scale_pitch_t;
};

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

// The scale byte of a block whose largest magnitude has these bits: 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    const int field = (int)(most >> 23);
    if (field == 255) return 255;                               // an infinity or NaN
    const int byte = field - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return byte < 0 ? 0 : byte;
}

// The scale as the conversions take it: they go by its exponent, and 0 is 2^-127.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

typedef short two_codes __attribute__((ext_vector_type(2)));     // in its lower or upper half

// The codes of 4 values.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, uint32_t byte)
{
    two_codes v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a, b, scale_of(byte), false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c, d, scale_of(byte), true);
    return __builtin_bit_cast(uint32_t, v);
}

// What conversions do not know: blocks that are NaN have codes 0, and 256 becomes 240 where it would be 2^128.
__device__ __forceinline__ uint32_t kept_codes(uint32_t word, uint32_t byte)
{
    if (byte == kLargestByte) word -= word >> 3 & word >> 4 & word >> 5 & word >> 6 & 0x01010101;
    return byte == 255 ? 0 : word;
}

__device__ __forceinline__ float largest(const float (&x)[8])
{
    float most = fabsf(x[0]);
#pragma unroll
    for (int k = 1; k < 8; ++k) most = __builtin_elementwise_maximum(most, fabsf(x[k]));       // NaN where there is one
    return most;
}

// Over the 16 lanes of a block.
__device__ __forceinline__ uint32_t most_of_block(uint32_t most)
{
    auto moved = [](uint32_t v, auto pattern) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(pattern)::value, 0xF, 0xF, false); };
    most = max(most, moved(most, std::integral_constant<int, 0xB1>()));        // quad_perm [1, 0, 3, 2]
    most = max(most, moved(most, std::integral_constant<int, 0x4E>()));        // quad_perm [2, 3, 0, 1]
    most = max(most, moved(most, std::integral_constant<int, 0x141>()));       // row_half_mirror
    most = max(most, moved(most, std::integral_constant<int, 0x140>()));       // row_mirror
    return most;
}

// The rows' form alone, a scale for each row.
template <typename T>
__global__ __launch_bounds__(kBlock) void f8_quantize_rows_kernel(F8Args a)
{
    constexpr int kEach = 2, kBlocks = kBlock / 16;
    const uint64_t first = (uint64_t)workgroup() * (kBlocks * kEach) + threadIdx.x / 16;
    const int l = threadIdx.x % 16;
    int64_t row[kEach], chunk[kEach];
    float x[kEach][8];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint64_t at = min(first + e * kBlocks, a.blocks - 1);
        row[e] = a.chunks_of_row.quotient(at);
        chunk[e] = at - row[e] * a.chunks;
        const int64_t col = chunk[e] * kF8Block + l * 8;
        const int left = (int)min(a.n_cols - col, (int64_t)8);
        if (left > 0) load_piece<T, 8>((const T *)a.x, row[e] * a.ld + col, left, a.span, x[e]);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[e][k] = k < left ? x[e][k] : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint32_t byte = scale_byte(most_of_block(magnitude(largest(x[e]))));
        if (first + e * kBlocks >= a.blocks) continue;
        *reinterpret_cast<uint2 *>(a.codes + (row[e] * a.chunks + chunk[e]) * kF8Block + l * 8) =
            make_uint2(kept_codes(codes_of(x[e][0], x[e][1], x[e][2], x[e][3], byte), byte), kept_codes(codes_of(x[e][4], x[e][5], x[e][6], x[e][7], byte), byte));
        uint8_t *scales = a.scales + chunk[e] * a.scale_pitch;
        if (l == 0) scales[row[e]] = (uint8_t)byte;
        if (row[e] == a.n_rows - 1 && a.n_rows + l < a.scale_pitch) scales[a.n_rows + l] = 0;
    }
}

constexpr int kTile = kF8Block, kTilePieces = kTile / 8;

// Over the four groups of 16 lanes.
__device__ __forceinline__ uint32_t most_of_groups(uint32_t most)
{
    const auto a = __builtin_amdgcn_permlane16_swap(most, most, false, false);
    most = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(most, most, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// A tile of 128 rows and 128 columns, of which a thread has 8 x 8: the columns' form, the rows' form or both, a scale for each row (column) or for the tile.  A column's largest is found over
// the threads that have it, its codes are made where the values are, and only they, a quarter of the bytes, pass the LDS.
template <typename T, bool TILES>
__global__ __launch_bounds__(kBlock) void f8_quantize_kernel(F8Args a)
{
    __shared__ uint2 turned[kTile * kTilePieces];   // codes of the transpose: of each column 16 pieces of 8 rows
    __shared__ uint4 most_of_cols[kWavesPerBlock][kTile / 4];
    __shared__ uint32_t most_of_tile[kWavesPerBlock];
    const uint64_t at = workgroup();
    const int64_t tile_r = at / a.tiles_c, tile_c = at % a.tiles_c;
    if (tile_r >= a.tiles_r) return;
    const int l = threadIdx.x % kTilePieces, r = threadIdx.x / kTilePieces, wave = threadIdx.x / kWave;    // columns 8 l .., rows 8 r ..
    const int64_t col = tile_c * kTile + l * 8, row0 = tile_r * kTile + r * 8;
    const int left = (int)min(max(a.n_cols - col, (int64_t)0), (int64_t)8);
    float x[8][8];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const bool there = row0 + p < a.n_rows && left > 0;
        if (there) load_piece<T, 8>((const T *)a.x, (row0 + p) * a.ld + col, left, a.span, x[p]);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[p][k] = there && k < left ? x[p][k] : 0.0f;
    }
    uint32_t tile_byte = 0;
    if (TILES) {
        uint32_t most = 0;
#pragma unroll
        for (int p = 0; p < 8; ++p) most = max(most, magnitude(largest(x[p])));
        most = most_of_groups(most_of_block(most));
        if (threadIdx.x % kWave == 0) most_of_tile[wave] = most;
        __syncthreads();
        tile_byte = scale_byte(max(max(most_of_tile[0], most_of_tile[1]), max(most_of_tile[2], most_of_tile[3])));
    }
    if (a.codes) {
        uint32_t bytes[2] = {0, 0};
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const uint32_t byte = TILES ? tile_byte : scale_byte(most_of_block(magnitude(largest(x[p]))));
            const bool there = row0 + p < a.n_rows;
            if (there)
                *reinterpret_cast<uint2 *>(a.codes + ((row0 + p) * a.chunks + tile_c) * kF8Block + l * 8) =
                    make_uint2(kept_codes(codes_of(x[p][0], x[p][1], x[p][2], x[p][3], byte), byte), kept_codes(codes_of(x[p][4], x[p][5], x[p][6], x[p][7], byte), byte));
            bytes[p / 4] |= (there ? byte : 0) << (8 * (p % 4));
        }
        if (l == 0 && row0 < a.scale_pitch) *reinterpret_cast<uint2 *>(a.scales + tile_c * a.scale_pitch + row0) = make_uint2(bytes[0], bytes[1]);
    }
    if (!a.codes_t) return;
    uint32_t byte_of[8];
    if (TILES) {
#pragma unroll
        for (int k = 0; k < 8; ++k) byte_of[k] = tile_byte;
    } else {
        uint32_t most[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float v[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) v[p] = x[p][k];
            most[k] = most_of_groups(magnitude(largest(v)));
        }
        if (threadIdx.x % kWave < kTilePieces) {
            most_of_cols[wave][l * 2] = make_uint4(most[0], most[1], most[2], most[3]);
            most_of_cols[wave][l * 2 + 1] = make_uint4(most[4], most[5], most[6], most[7]);
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 m = most_of_cols[w][l * 2 + h];
                most[h * 4] = max(most[h * 4], m.x);
                most[h * 4 + 1] = max(most[h * 4 + 1], m.y);
                most[h * 4 + 2] = max(most[h * 4 + 2], m.z);
                most[h * 4 + 3] = max(most[h * 4 + 3], m.w);
            }
#pragma unroll
        for (int k = 0; k < 8; ++k) byte_of[k] = scale_byte(most[k]);
    }
    // of column 8 l + k the piece of rows 8 r .. is at place r ^ l of line 8 l + (k ^ l mod 2): the lanes of a wave that write the same k share all banks evenly
#pragma unroll
    for (int k = 0; k < 8; ++k)
        turned[(l * 8 + (k ^ l % 2)) * kTilePieces + (r ^ l)] =
            make_uint2(kept_codes(codes_of(x[0][k], x[1][k], x[2][k], x[3][k], byte_of[k]), byte_of[k]), kept_codes(codes_of(x[4][k], x[5][k], x[6][k], x[7][k], byte_of[k]), byte_of[k]));
    if (r == 0 && col < a.scale_pitch_t) {
        uint32_t bytes[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) bytes[k / 4] |= (k < left ? byte_of[k] : 0) << (8 * (k % 4));
        *reinterpret_cast<uint2 *>(a.scales_t + tile_r * a.scale_pitch_t + col) = make_uint2(bytes[0], bytes[1]);
    }
    __syncthreads();
    // 16 rows of a column a lane, 8 lanes a line
#pragma unroll
    for (int i = 0; i < kTile / 32; ++i) {
        const int c = i * 32 + threadIdx.x / 8, part = threadIdx.x % 8, of = c / 8;
        const uint4 both = reinterpret_cast<const uint4 *>(turned)[(of * 8 + (c % 8 ^ of % 2)) * (kTilePieces / 2) + (part ^ of / 2)];
        const int64_t row = tile_c * kTile + c;     // of the transpose
        if (row < a.n_cols) *reinterpret_cast<uint4 *>(a.codes_t + row * a.pitch_t + tile_r * kF8Block + part * 16) = of % 2 ? make_uint4(both.z, both.w, both.x, both.y) : both;
    }
}

struct F8ReadArgs {
    const uint8_t *codes, *scales;
    void *x;
    int64_t ld, n_rows, n_cols, chunks, scale_pitch;
    uint64_t pieces;
    Divider pieces_of_row;
    int64_t written;
};

template <typename T>
__global__ __launch_bounds__(kBlock) void f8_dequantize_kernel(F8ReadArgs a)
{
    const uint64_t at = (uint64_t)workgroup() * kBlock + threadIdx.x;
    if (at >= a.pieces) return;
    const int64_t row = a.pieces_of_row.quotient(at), col = (int64_t)(at - (uint64_t)row * a.pieces_of_row.by) * 8;
    const int left = (int)min(max(a.n_cols - col, (int64_t)0), (int64_t)8), left_written = (int)min(a.written - col, (int64_t)8);
    float v[8] = {};
    if (left > 0) {
        const uint2 word = *reinterpret_cast<const uint2 *>(a.codes + row * a.chunks * kF8Block + col);
        const uint32_t byte = a.scales[col / kF8Block * a.scale_pitch + row];
        const float scale = byte == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, byte == 0 ? 0x400000u : byte << 23);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int w = (int)(h ? word.y : word.x);
            const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), high = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            v[h * 4] = low[0]; v[h * 4 + 1] = low[1]; v[h * 4 + 2] = high[0]; v[h * 4 + 3] = high[1];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < left ? v[k] * scale : 0.0f;
    }
    store_piece<T, 8>((T *)a.x + row * a.ld + col, left_written, v);
}

template <typename T>
hipError_t launch_quantize(const F8Args &a, int32_t blocks, hipStream_t st)
{
    if (!a.codes_t && blocks == ADAQP_F8_ROWS) f8_quantize_rows_kernel<T><<<grid_of((int64_t)((a.blocks + 31) / 32), kBlock), kBlock, 0, st>>>(a);
    else {
        const dim3 grid = grid_of((int64_t)a.tiles_r * a.tiles_c, kBlock);
        if (blocks == ADAQP_F8_TILES) f8_quantize_kernel<T, true><<<grid, kBlock, 0, st>>>(a);
        else                          f8_quantize_kernel<T, false><<<grid, kBlock, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int64_t adaqp_f8_code_bytes(int64_t n_rows, int64_t n_cols)
{
    if (n_rows < 0 || n_cols < 0 || n_rows >= kF8Most || n_cols >= kF8Most) return -1;
    return n_rows * f8_chunks(n_cols) * kF8Block;
}

extern "C" int64_t adaqp_f8_scale_bytes(int64_t n_rows, int64_t n_cols)
{
    if (n_rows < 0 || n_cols < 0 || n_rows >= kF8Most || n_cols >= kF8Most) return -1;
    return f8_chunks(n_cols) * f8_scale_pitch(n_rows);
}

extern "C" int adaqp_f8_quantize(const void *x_dev, int64_t ld, int64_t n_rows, int64_t n_cols, int32_t type, int32_t blocks,
                                 uint8_t *codes_dev, uint8_t *scales_dev, uint8_t *codes_t_dev, uint8_t *scales_t_dev, void *stream)
{
    if (n_rows < 0 || n_cols < 0 || !valid_type(type) || (blocks != ADAQP_F8_ROWS && blocks != ADAQP_F8_TILES)) return ADAQP_EINVAL;
    if (!codes_dev != !scales_dev || !codes_t_dev != !scales_t_dev) return ADAQP_EINVAL;
    if (n_rows >= kF8Most || n_cols >= kF8Most) return ADAQP_ESIZE;
    if (n_rows == 0 || n_cols == 0 || (!codes_dev && !codes_t_dev)) return ADAQP_OK;
    ADAQP_TRY(check_rows(x_dev, ld, n_cols, type));
    if ((codes_dev && !valid_f8(codes_dev, scales_dev)) || (codes_t_dev && !valid_f8(codes_t_dev, scales_t_dev))) return ADAQP_EINVAL;
    if (!countable(n_rows, ld)) return ADAQP_ESIZE;
    const int64_t tiles_r = f8_chunks(n_rows), tiles_c = f8_chunks(n_cols);
    if (n_rows * tiles_c / 32 >= kMostWorkgroups || tiles_r * tiles_c >= kMostWorkgroups) return ADAQP_ESIZE;
    F8Args a{};
    a.x = x_dev; a.ld = ld; a.n_rows = n_rows; a.n_cols = n_cols; a.span = matrix_span(n_rows, ld, n_cols);
    a.chunks = tiles_c;
    a.blocks = (uint64_t)(n_rows * tiles_c);
    a.chunks_of_row = divider(tiles_c, (int64_t)a.blocks);
    a.tiles_r = (uint32_t)tiles_r; a.tiles_c = (uint32_t)tiles_c;
    a.codes = codes_dev; a.scales = scales_dev; a.codes_t = codes_t_dev; a.scales_t = scales_t_dev;
    a.scale_pitch = f8_scale_pitch(n_rows); a.pitch_t = tiles_r * kF8Block; a.scale_pitch_t = f8_scale_pitch(n_cols);
    if (type == ADAQP_F32) ADAQP_HIP_TRY(launch_quantize<float>(a, blocks, (hipStream_t)stream));
    else                   ADAQP_HIP_TRY(launch_quantize<__bf16>(a, blocks, (hipStream_t)stream));
    return ADAQP_OK;
}

extern "C" int adaqp_f8_dequantize(const uint8_t *codes_dev, const uint8_t *scales_dev, int64_t n_rows, int64_t n_cols, void *x_dev, int64_t ld,
                                   int32_t type, void *stream)
{
    if (n_rows < 0 || n_cols < 0 || !valid_type(type)) return ADAQP_EINVAL;
    if (n_rows >= kF8Most || n_cols >= kF8Most) return ADAQP_ESIZE;
    if (n_rows == 0 || n_cols == 0) return ADAQP_OK;
    if (!valid_f8(codes_dev, scales_dev)) return ADAQP_EINVAL;
    ADAQP_TRY(check_rows(x_dev, ld, n_cols, type));
    if (!countable(n_rows, ld)) return ADAQP_ESIZE;
    F8ReadArgs a{};
    a.codes = codes_dev; a.scales = scales_dev; a.x = x_dev; a.ld = ld; a.n_rows = n_rows; a.n_cols = n_cols;
    a.chunks = f8_chunks(n_cols); a.scale_pitch = f8_scale_pitch(n_rows);
    a.written = columns_to_write(x_dev, ld, n_cols, element_bytes(type));
    const int64_t each = (a.written + 7) / 8;
    if (n_rows > kMostWorkgroups * (kBlock / 2) / each) return ADAQP_ESIZE;
    a.pieces = (uint64_t)(n_rows * each);
    a.pieces_of_row = divider(each, (int64_t)a.pieces);
    const dim3 grid = grid_of((int64_t)((a.pieces + kBlock - 1) / kBlock), kBlock);
    if (type == ADAQP_F32) f8_dequantize_kernel<float><<<grid, kBlock, 0, (hipStream_t)stream>>>(a);
    else                   f8_dequantize_kernel<__bf16><<<grid, kBlock, 0, (hipStream_t)stream>>>(a);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}
