// MX matrices: writing them from rows, columns or both, and reading them back (adaqp_dense.h).
//
// A workgroup takes a tile of 128 rows and 128 columns: 16 lanes hold a row's 128 columns, 8 neighbouring ones each (a granule: one Philox call, one
// 32-bit word of codes), 4 lanes a block.  The tile stays in registers for the rows' blocks; for the columns' blocks it goes through the LDS once
// and a lane takes 32 rows of one column.  x is read once whichever of the two forms is wanted.  Both directions are bound by memory: 4 bytes
// read per element of fp32 and 0.53 written per form.
#include "mx4.hpp"
#include "philox.hpp"

namespace adaqp {
namespace {

constexpr uint32_t kMxTag = 0x4d583443u;
constexpr int kTile = 128;
constexpr int kLanes = kTile / 8;                   // of a row
constexpr int kPasses = kTile / (kBlock / kLanes);  // a lane has one row of each

struct MxArgs {
    const void *x;
    int64_t ld, n_rows, n_cols;
    int64_t tiles_c;
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

// The codes of 8 values, low nibble first.  In steps of 1/2 below 2, 1 below 4, 2 beyond, the code counts the steps; all products are by powers of two.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], uint32_t byte, const Rand128 &rnd)
{
    if (byte == 255) return 0;
    const float inv = __builtin_bit_cast(float, (254u - byte) << 23);
    const uint32_t w[4] = {rnd.w0, rnd.w1, rnd.w2, rnd.w3};
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, x[j]);
        const float y = __builtin_bit_cast(float, bits & 0x7FFFFFFFu) * inv;
        const float steps = y < 2.0f ? 2.0f : y < 4.0f ? 1.0f : 0.5f;
        const uint32_t base = y < 2.0f ? 0 : y < 4.0f ? 2 : 4;
        uint32_t code;
        if (STOCHASTIC) {
            const uint32_t r = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
            code = (((uint32_t)(y * (steps * 65536.0f)) + r) >> 16) + base;
        } else {
            code = (uint32_t)rintf(y * steps) + base;
            code = code > 7 ? 7 : code;
        }
        word |= (code | (bits >> 31) << 3) << (4 * j);
    }
    return word;
}

__device__ __forceinline__ Rand128 random_words(uint64_t seed, int64_t row, int64_t granule)
{
    return philox4x32_10((uint32_t)granule, (uint32_t)row, 0u, kMxTag, (uint32_t)seed, (uint32_t)(seed >> 32));
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

template <int PATTERN>
__device__ __forceinline__ uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, PATTERN, 0xF, 0xF, false);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;       // partners of a butterfly over 16 lanes

// 8 columns from col on, zeros from n_cols on.
template <typename T, int VW>
__device__ __forceinline__ void load_granule(const T *row, int64_t col, int64_t n_cols, float (&x)[8])
{
#pragma unroll
    for (int v = 0; v < 8; v += VW) {
        float part[VW];
        if (col + v + VW <= n_cols) load_elements<T, VW>(row + col + v, part);
        else for (int k = 0; k < VW; ++k) part[k] = col + v + k < n_cols ? (float)row[col + v + k] : 0.0f;
#pragma unroll
        for (int k = 0; k < VW; ++k) x[v + k] = part[k];
    }
}

template <typename T, int VW, bool ROWS, bool COLS, bool STOCHASTIC>
__global__ __launch_bounds__(kBlock) void mx4_quantize_kernel(MxArgs a)
{
    __shared__ float tile[COLS ? kTile * kTile : 1];
    const int64_t chunk_c = blockIdx.x % a.tiles_c, chunk_r = blockIdx.x / a.tiles_c;
    const int l = threadIdx.x % kLanes, r = threadIdx.x / kLanes;
    float x[kPasses][8];
    const int64_t col = chunk_c * kTile + l * 8;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int64_t row = chunk_r * kTile + p * (kTile / kPasses) + r;
        if (row < a.n_rows) load_granule<T, VW>((const T *)a.x + row * a.ld, col, a.n_cols, x[p]);
        else for (int k = 0; k < 8; ++k) x[p][k] = 0.0f;
    }
    if (COLS) {
        // columns of rows 32 b .. 32 b + 31 are turned by 16 b: then the lanes of a wave, 16 columns of 4 blocks, read 64 banks
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int row = p * (kTile / kPasses) + r;
            float *to = tile + row * kTile + (l * 8 + 16 * (row / kMxBlock)) % kTile;
#pragma unroll
            for (int k = 0; k < 8; k += 4) *reinterpret_cast<float4 *>(to + k) = make_float4(x[p][k], x[p][k + 1], x[p][k + 2], x[p][k + 3]);
        }
    }
    if (ROWS) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int64_t row = chunk_r * kTile + p * (kTile / kPasses) + r;
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) most = max(most, magnitude(x[p][k]));
            most = max(most, moved<kSwap1>(most));
            most = max(most, moved<kSwap2>(most));
            const uint32_t byte = scale_byte<STOCHASTIC>(most);
            Rand128 rnd{};
            if (STOCHASTIC) rnd = random_words(a.seed, row, col / 8);
            const uint32_t word = codes_of<STOCHASTIC>(x[p], byte, rnd);
            uint32_t scales = byte << (8 * (l / 4));
            scales |= moved<kMirror8>(scales);
            scales |= moved<kMirror16>(scales);
            if (row < a.n_rows) {
                *reinterpret_cast<uint32_t *>(a.codes + row * a.pitch + chunk_c * kMxChunkBytes + l * 4) = word;
                if (l == 0) *reinterpret_cast<uint32_t *>(a.scales + (chunk_c * a.n_rows + row) * 4) = scales;
            }
        }
    }
    if (COLS) {
        __syncthreads();
        const int b = threadIdx.x % 4;                          // block of 32 rows
#pragma unroll
        for (int c = threadIdx.x / 4; c < kTile; c += kBlock / 4) {
            const int64_t row = chunk_c * kTile + c;            // of the transpose
            if (row >= a.n_cols) break;
            const float *from = tile + b * kMxBlock * kTile + (c + 16 * b) % kTile;
            float v[4][8];
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < kMxBlock; ++k) {
                v[k / 8][k % 8] = from[k * kTile];
                most = max(most, magnitude(v[k / 8][k % 8]));
            }
            const uint32_t byte = scale_byte<STOCHASTIC>(most);
            uint32_t word[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                Rand128 rnd{};
                if (STOCHASTIC) rnd = random_words(a.seed + 1, row, chunk_r * (kTile / 8) + b * 4 + g);
                word[g] = codes_of<STOCHASTIC>(v[g], byte, rnd);
            }
            uint32_t scales = byte << (8 * b);
            scales |= moved<kSwap1>(scales);
            scales |= moved<kSwap2>(scales);
            *reinterpret_cast<uint4 *>(a.codes_t + row * a.pitch_t + chunk_r * kMxChunkBytes + b * 16) = make_uint4(word[0], word[1], word[2], word[3]);
            if (b == 0) *reinterpret_cast<uint32_t *>(a.scales_t + (chunk_r * a.n_cols + row) * 4) = scales;
        }
    }
}

// 8 values of one word of codes.
__device__ __forceinline__ void values_of(uint32_t word, uint32_t byte, float (&v)[8])
{
    const float scale = __builtin_bit_cast(float, byte == 0 ? 0x400000u : byte << 23);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t code = word >> (4 * j) & 7u, exponent = code >> 1, odd = code & 1u;
        // 0, 1/2, then (1 + odd / 2) 2^(exponent - 1)
        const uint32_t bits = exponent ? (126u + exponent) << 23 | odd << 22 : odd ? 126u << 23 : 0u;
        const float m = __builtin_bit_cast(float, bits | (word >> (4 * j + 3) & 1u) << 31) * scale;
        v[j] = byte == 255 ? __builtin_nanf("") : m;
    }
}

template <typename T, int VW, bool WHOLE>
__global__ __launch_bounds__(kBlock) void mx4_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, int64_t n_rows, int64_t n_cols, int64_t written,
                                                                int64_t pitch, T *x, int64_t ld, int64_t granules)
{
    const int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const int64_t row = at / granules, g = at % granules;
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
    const bool rows = a.codes, cols = a.codes_t;
    auto go = [&](auto stochastic) {
        constexpr bool S = decltype(stochastic)::value;
        if (rows && cols) mx4_quantize_kernel<T, VW, true, true, S><<<(uint32_t)blocks, kBlock, 0, st>>>(a);
        else if (rows)    mx4_quantize_kernel<T, VW, true, false, S><<<(uint32_t)blocks, kBlock, 0, st>>>(a);
        else              mx4_quantize_kernel<T, VW, false, true, S><<<(uint32_t)blocks, kBlock, 0, st>>>(a);
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
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    constexpr int VW = 16 / sizeof(T);
    const bool wide = whole || (aligned_to(x, 16) && ld % VW == 0);
    auto go = [&](auto vw, auto lines) {
        mx4_dequantize_kernel<T, decltype(vw)::value, decltype(lines)::value>
            <<<(uint32_t)blocks, kBlock, 0, st>>>(codes, scales, n_rows, n_cols, written, mx_pitch(n_cols), (T *)x, ld, granules);
    };
    if (whole)     go(std::integral_constant<int, VW>(), std::true_type());
    else if (wide) go(std::integral_constant<int, VW>(), std::false_type());
    else           go(std::integral_constant<int, 1>(), std::false_type());
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
    MxArgs a{x_dev, ld, n_rows, n_cols, mx_chunks(n_cols), seed, codes_dev, scales_dev, codes_t_dev, scales_t_dev, mx_pitch(n_cols), mx_pitch(n_rows)};
    const int64_t blocks = a.tiles_c * mx_chunks(n_rows);
    if (blocks > 0x7FFFFFFF) return ADAQP_ESIZE;
    // a vector may not be past the last column unless the row's lines are the matrix's own; load_granule takes the last columns one by one
    int vw = (int)(16 / element_bytes(type));
    while (vw > 1 && (!aligned_to(x_dev, vw * element_bytes(type)) || ld % vw != 0)) vw /= 2;
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
    if ((n_cols + 127) / 8 * n_rows / kBlock >= 0x7FFFFFFF) return ADAQP_ESIZE;
    if (type == ADAQP_F32) ADAQP_HIP_TRY((launch_dequantize<float>(codes_dev, scales_dev, n_rows, n_cols, x_dev, ld, (hipStream_t)stream)));
    else                   ADAQP_HIP_TRY((launch_dequantize<__bf16>(codes_dev, scales_dev, n_rows, n_cols, x_dev, ld, (hipStream_t)stream)));
    return ADAQP_OK;
}
