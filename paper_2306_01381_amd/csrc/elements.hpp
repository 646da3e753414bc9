// Matrix elements of the dense operators (adaqp_dense.h): vectors of fp32 or bf16 in memory, fp32 in registers; sums over lanes of a wave.
#pragma once

#include "adaqp_dense.h"
#include "common.hpp"
#include "grid.hpp"

namespace adaqp {

template <typename T, int N> using vec_of = T __attribute__((ext_vector_type(N)));

// N neighbouring elements, aligned to their size together.
template <typename T, int N>
__device__ __forceinline__ void load_elements(const T *p, float (&dst)[N])
{
    const vec_of<T, N> v = *reinterpret_cast<const vec_of<T, N> *>(p);
#pragma unroll
    for (int k = 0; k < N; ++k) dst[k] = (float)v[k];
}

// The same, aligned to one element only: one access all the same, the memory system takes any alignment.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) loose_of { vec_of<T, N> v; };

template <typename T, int N>
__device__ __forceinline__ void load_loose(const T *p, float (&dst)[N])
{
    const vec_of<T, N> v = reinterpret_cast<const loose_of<T, N> *>(p)->v;
#pragma unroll
    for (int k = 0; k < N; ++k) dst[k] = (float)v[k];
}

template <typename T, int N>
__device__ __forceinline__ vec_of<T, N> rounded(const float (&src)[N])
{
    vec_of<T, N> v;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (T)src[k];             // to nearest even
    return v;
}

template <typename T, int N, bool STREAM>
__device__ __forceinline__ void store_elements(T *p, const float (&src)[N])
{
    const vec_of<T, N> v = rounded<T, N>(src);
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<vec_of<T, N> *>(p));
    else                  *reinterpret_cast<vec_of<T, N> *>(p) = v;
}

template <typename T, int N>
__device__ __forceinline__ void store_loose(T *p, const float (&src)[N])
{
    reinterpret_cast<loose_of<T, N> *>(p)->v = rounded<T, N>(src);
}

// The sum over the LANES neighbouring lanes that share lane / LANES, in all of them, without the LDS: exchanges inside rows of 16 lanes by DPP,
// between rows by gfx950's half swaps.  Both partners add the same two numbers, so every lane has the same bits.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v)
{
    static_assert(LANES >= 1 && LANES <= kWave && (LANES & (LANES - 1)) == 0, "a power of two of lanes");
    auto moved = [](float x, auto pattern) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int32_t, x), decltype(pattern)::value, 0xF, 0xF, false));
    };
    if constexpr (LANES >= 2) v += moved(v, std::integral_constant<int, 0xB1>());      // quad_perm [1, 0, 3, 2]
    if constexpr (LANES >= 4) v += moved(v, std::integral_constant<int, 0x4E>());      // quad_perm [2, 3, 0, 1]
    if constexpr (LANES >= 8) v += moved(v, std::integral_constant<int, 0x141>());     // row_half_mirror
    if constexpr (LANES >= 16) v += moved(v, std::integral_constant<int, 0x140>());    // row_mirror
    if constexpr (LANES >= 32) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto w = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = __builtin_bit_cast(float, (uint32_t)w[0]) + __builtin_bit_cast(float, (uint32_t)w[1]);
    }
    if constexpr (LANES >= 64) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        v = __builtin_bit_cast(float, (uint32_t)w[0]) + __builtin_bit_cast(float, (uint32_t)w[1]);
    }
    return v;
}

// A kernel's workgroup among those of grid_of().
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }
__device__ __forceinline__ uint32_t workgroups() { return gridDim.y * gridDim.x; }

inline dim3 grid_of(int64_t workgroups, int32_t threads, uint32_t z = 1)
{
    const GridSize g = grid_size(workgroups, threads);
    return dim3(g.x, g.y, z);
}

// Workgroups are dealt to the eight XCDs in turn: the place of a workgroup in a grid (a multiple of eight) such that neighbouring places share an XCD.
__device__ __forceinline__ uint32_t xcd_neighbour(uint32_t block, uint32_t blocks) { return block % 8 * (blocks / 8) + block / 8; }

inline bool valid_type(int32_t type) { return type == ADAQP_F32 || type == ADAQP_BF16; }

inline int64_t element_bytes(int32_t type) { return type == ADAQP_F32 ? 4 : 2; }

// Rows that begin and end on 128-byte lines.
inline bool whole_lines(const void *base, int64_t ld, int64_t bytes) { return aligned_to(base, 128) && ld * bytes % 128 == 0; }

// The most elements (at most 16 bytes) that a vector may have so that rows of `cols` elements are whole vectors, each on a multiple of its size.
inline int vector_elements(const void *base, int64_t ld, int64_t cols, int64_t bytes)
{
    int n = (int)(16 / bytes);
    while (n > 1 && (!aligned_to(base, n * bytes) || ld % n != 0 || cols % n != 0)) n /= 2;
    return n;
}

}  // namespace adaqp
