// What products on the matrix cores do with their sums (mx4_matmul.hip, f8_matmul.hip): 32 x 32 parts of a tile to memory, parts of k added up.
#pragma once

#include "elements.hpp"

namespace adaqp {
namespace {

typedef float tile_sums __attribute__((ext_vector_type(16)));

// Of a wave's sheet of 32 rows: FN * 32 columns, and the rows 4 apart that a store takes are in different banks.
constexpr int sheet_pitch(int fn) { return fn * 32 + 8; }

// Stores a wave's sums at (row0, col0); no wave reads operands in `lds` any more.  They go through it, where rows can be stored in vectors, so that a lane has 16 bytes of a
// row: stored as they are, a tile of 256 x 256 took 10 us for it, fp32 or bf16, and 7 and 5 this way.
template <typename T, int FM, int FN, typename Args>
__device__ __forceinline__ void store_tile(const Args &g, const tile_sums (&sums)[FM][FN], int64_t split, int64_t row0, int64_t col0, float *lds)
{
    __builtin_amdgcn_sched_barrier(0);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int rows = (int)min(g.m - row0, (int64_t)(FM * 32)), cols = (int)min(g.n - col0, (int64_t)(FN * 32)), written = (int)min(g.written - col0, (int64_t)(FN * 32));
    T *out = (T *)g.out + (split * g.m + row0) * g.ldo + col0;
    constexpr int VW = 16 / sizeof(T);
    if (g.whole_vectors) {
        constexpr int kSheet = FN * 32, kPitch = sheet_pitch(FN), kLanes = kSheet / VW, kAtOnce = kWave / kLanes;
        float *sheet = lds + wave * (32 * kPitch);
        const int col = lane % kLanes * VW, line = lane / kLanes;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) sheet[(q / 4 * 8 + h * 4 + q % 4) * kPitch + j * 32 + r] = sums[i][j][q];
#pragma unroll
            for (int at = 0; at < 32; at += kAtOnce) {
                float v[VW];
                load_elements<float, VW>(sheet + (at + line) * kPitch + col, v);
#pragma unroll
                for (int k = 0; k < VW; ++k) v[k] = col + k < cols ? v[k] : 0.0f;
                const int row = i * 32 + at + line;
                if (row < rows && col < written) store_elements<T, VW, false>(out + row * g.ldo + col, v);
            }
        }
        return;
    }
    // lane's part of a place, and the wave's
    const int64_t mine = (int64_t)(h * 4) * g.ldo + r;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int row = i * 32 + q / 4 * 8 + q % 4;
            if (row + h * 4 >= rows) continue;
            T *to = out + row * g.ldo + mine;
#pragma unroll
            for (int j = 0; j < FN; ++j)
                if (j * 32 + r < written) to[j * 32] = j * 32 + r < cols ? (T)sums[i][j][q] : (T)0.0f;
        }
}

// The splits' sums, in order; columns from n to `written` are zeros.  A workgroup of 64 columns and four rows.
template <typename T>
__global__ __launch_bounds__(kBlock) void join_parts_kernel(const float *parts, int n_parts, int64_t m, int64_t n, int64_t written, T *out, int64_t ldo)
{
    constexpr int kAtOnce = 8;
    const int64_t col = (int64_t)blockIdx.x * kWave + threadIdx.x % kWave;
    if (col >= written) return;
    for (int64_t row = (int64_t)blockIdx.y * kWavesPerBlock + threadIdx.x / kWave; row < m; row += (int64_t)gridDim.y * kWavesPerBlock) {
        const float *from = parts + row * n + min(col, n - 1);
        float sum = 0.0f;
        for (int s = 0; s < n_parts; s += kAtOnce) {
            float v[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) v[k] = from[min(s + k, n_parts - 1) * m * n];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (s + k < n_parts) sum += v[k];
        }
        out[row * ldo + col] = col < n ? (T)sum : (T)0.0f;
    }
}

}  // namespace
}  // namespace adaqp
