// Tiles of a matrix in the LDS for the matrix cores: of each row one 128-byte line, loaded from memory without passing registers.
// The eight 16-byte parts of a line lie at (part ^ row mod 8), so that 32 lanes that read the same part of 32 rows use all banks.
#pragma once

#include "common.hpp"

namespace adaqp {

constexpr int kLine = 128;

// What lanes load whose row or line does not exist.
__device__ const uint4 zero_part = {0, 0, 0, 0};
__device__ __forceinline__ const void *zeros() { return &zero_part; }

// Of each lane 16 or 4 bytes, to lds + lane * that; lds is the wave's.  (The builtin takes its size as a literal only.)
__device__ __forceinline__ void load_to_lds_16(const void *from, void *lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}
__device__ __forceinline__ void load_to_lds_4(const void *from, void *lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)lds, 4, 0, 0);
}

// This wave's loads are in the LDS, and after the barrier every wave's.
__device__ __forceinline__ void landed()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Line `line` of ROWS rows from row0 on, zeros where the matrix has no such row or its pitch (bytes, a multiple of 16) ends.  All waves of a workgroup of kBlock.
template <int ROWS>
__device__ __forceinline__ void load_lines(const uint8_t *matrix, int64_t row0, int64_t n_rows, int64_t pitch, int64_t line, uint8_t *lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
#pragma unroll
    for (int i = 0; i < ROWS / 32; ++i) {
        const int first = wave * (ROWS / kWavesPerBlock) + i * 8;       // 8 rows of 8 parts
        const int64_t row = row0 + first + lane / 8, at = line * kLine + (lane % 8 ^ lane / 8) * 16;
        load_to_lds_16(row < n_rows && at < pitch ? (const void *)(matrix + row * pitch + at) : zeros(), lds + first * kLine);
    }
}

__device__ __forceinline__ const uint8_t *line_part(const uint8_t *lds, int row, int part) { return lds + row * kLine + (part ^ row % 8) * 16; }

}  // namespace adaqp
