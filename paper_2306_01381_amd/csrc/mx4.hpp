// MX matrices (adaqp_dense.h): 32 values of 4 bits that share a power of two.
#pragma once

#include "elements.hpp"

namespace adaqp {

constexpr int kMxBlock = ADAQP_MX4_BLOCK;
constexpr int kMxChunk = 128;                       // columns of a scale word
constexpr int kMxChunkBytes = kMxChunk / 2;
constexpr int64_t kMxMost = (int64_t)1 << 31;       // rows or columns

inline int64_t mx_chunks(int64_t cols) { return (cols + kMxChunk - 1) / kMxChunk; }
inline int64_t mx_pitch(int64_t cols) { return mx_chunks(cols) * kMxChunkBytes; }

// Arrays of an MX matrix that has elements.
inline bool valid_mx(const void *codes, const void *scales) { return codes && scales && aligned_to(codes, 16) && aligned_to(scales, 16); }

}  // namespace adaqp
