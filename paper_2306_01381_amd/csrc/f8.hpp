// Matrices in 8 bits (adaqp_train.h): e4m3 codes, a power of two for 128 columns of a row.
#pragma once

#include "adaqp_train.h"
#include "elements.hpp"

namespace adaqp {

constexpr int kF8Block = ADAQP_F8_BLOCK;
constexpr int64_t kF8Most = (int64_t)1 << 31;       // rows or columns

inline int64_t f8_chunks(int64_t cols) { return (cols + kF8Block - 1) / kF8Block; }
inline int64_t f8_scale_pitch(int64_t rows) { return (rows + 15) / 16 * 16; }

// Arrays of an 8-bit matrix that has elements.
inline bool valid_f8(const void *codes, const void *scales) { return codes && scales && aligned_to(codes, 16) && aligned_to(scales, 16); }

}  // namespace adaqp
