// Rows of matrices in pieces of N neighbouring columns, wherever they begin (adaqp_train.h): a piece is read as one vector, aligned to an element only, where that stays in
// the matrix, also where it passes the row's end: what it reads of the next row is not used.
#pragma once

#include "elements.hpp"

namespace adaqp {

// n / by, by a multiplication where all n are below 2^31.
struct Divider {
    uint32_t factor, shift, by;
    __device__ __forceinline__ int64_t quotient(uint64_t n) const
    {
        return factor ? (uint64_t)(uint32_t)n * factor >> shift : n / by;
    }
};

// `most`: n is below it.  With 2^(bits - 1) < by <= 2^bits, factor = ceil(2^(31 + bits) / by) is below 2^32 and by * factor - 2^(31 + bits) below by <= 2^bits, so that
// n * factor / 2^(31 + bits) passes n / by by less than 1 / by.
inline Divider divider(int64_t by, int64_t most)
{
    int bits = 0;
    while (((int64_t)1 << bits) < by) ++bits;
    const uint64_t factor = (((uint64_t)1 << (31 + bits)) + by - 1) / by;
    return Divider{most <= ((int64_t)1 << 31) ? (uint32_t)factor : 0, (uint32_t)(31 + bits), (uint32_t)by};
}

// Elements from a matrix's first to its last.
inline int64_t matrix_span(int64_t n_rows, int64_t ld, int64_t cols) { return n_rows > 0 ? (n_rows - 1) * ld + cols : 0; }

// Vectors aligned to an element only, for accesses that say so to the caches.
template <typename T, int N> using loose_vec = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));

// Whether a matrix of this span, read or written once, drives more out of the 256 MiB of cache before the memory than it brings there.  Smaller ones may themselves be read from it.
inline bool passes_caches(int64_t span, int64_t bytes) { return span * bytes > ((int64_t)192 << 20); }

// The N elements at `at`, of which the first n are the row's; the others are anything.  ONCE: nothing reads them soon again.
template <typename T, int N, bool ONCE = false>
__device__ __forceinline__ void load_piece(const T *base, int64_t at, int n, int64_t span, float (&v)[N])
{
    if (at + N <= span) {
        if constexpr (ONCE) {
            const loose_vec<T, N> w = __builtin_nontemporal_load(reinterpret_cast<const loose_vec<T, N> *>(base + at));
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = (float)w[k];
        } else load_loose<T, N>(base + at, v);
    } else
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = k < n ? (float)base[at + k] : 0.0f;
}

// The first n of N elements, n >= 0.
template <typename T, int N, bool ONCE = false>
__device__ __forceinline__ void store_piece(T *to, int n, const float (&v)[N])
{
    if (n >= N) {
        if constexpr (ONCE) {
            const loose_vec<T, N> w = rounded<T, N>(v);
            __builtin_nontemporal_store(w, reinterpret_cast<loose_vec<T, N> *>(to));
        } else store_loose<T, N>(to, v);
    } else
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < n) to[k] = (T)v[k];
}

// Columns of an output that are written.
inline int64_t columns_to_write(const void *out, int64_t ld, int64_t cols, int64_t bytes)
{
    const int64_t line = 128 / bytes;
    return whole_lines(out, ld, bytes) ? (cols + line - 1) / line * line : cols;
}

inline int check_rows(const void *p, int64_t ld, int64_t cols, int32_t type)
{
    return p && ld >= cols && aligned_to(p, element_bytes(type)) ? ADAQP_OK : ADAQP_EINVAL;
}

// Whole rows of a matrix lie below 2^60 elements: places in it can be counted in 64 bits.
inline bool countable(int64_t n_rows, int64_t ld) { return ld < ((int64_t)1 << 60) / (n_rows > 0 ? n_rows : 1); }

constexpr int32_t kMostDim = (int32_t)1 << 30;

}  // namespace adaqp
