// What the kernels of orthogonalised updates share: numbers held as two of fp16, and the small form's call.
#pragma once

#include "elements.hpp"

namespace adaqp {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef float sums16 __attribute__((ext_vector_type(16)));

constexpr int kMostSteps = 64;

// One matrix, or several of one shape, small enough for a workgroup each (orthogonalize_small.hip).
struct SmallUpdate {
    const void *g;
    void *out;
    int64_t ldg, stride_g, ldo, stride_o;
    int32_t n_rows, n_cols, written, n_steps;
    double eps;
    int power;                                      // of X in the first step
    float of_gram[kMostSteps], of_poly[kMostSteps], linear[kMostSteps], diagonal[kMostSteps], of_step[kMostSteps];     // factors of a step's sums, as for the products of large ones
};

bool small_update_fits(int64_t n_rows, int64_t n_cols);
hipError_t launch_small_update(const SmallUpdate &u, int32_t n_matrices, int32_t type, hipStream_t st);

__device__ __forceinline__ void split(float v, _Float16 &hi, _Float16 &lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

__device__ __forceinline__ double block_sum(double v, double *lds)
{
    for (int other = 1; other < kWave; other *= 2) v += __shfl_xor(v, other);
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// 1 / (norm + eps) of a matrix with this sum of squares.  fp32 elements that are finite keep the sum finite in 64 bits; one that is not makes the whole matrix NaN, where 1 / inf
// would make zeros of the others.
__device__ __forceinline__ double one_over_norm(double sum, double eps) { return __builtin_isfinite(sum) ? 1.0 / (sqrt(sum) + eps) : __builtin_nan(""); }

}  // namespace adaqp
