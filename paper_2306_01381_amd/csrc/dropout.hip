// Dropout (adaqp_train.h): y = add + keep * x / (1 - p), the choices from a counter-based generator.
//
// A lane has pieces of 8 columns: one Philox call, whose 128 bits are their 16-bit numbers.  Nothing is stored of the choices.  Bound by memory: of 20 vector
// instructions an element (bf16, with a residual) 5 are the generator's; they keep the units busy in 47 % of the cycles.  Measured: 376 000 x 256 bf16 with a residual 104 us (578 MB, 5.5 TB/s; a copy of 1 GiB runs at 5.2), 2000 x 128 fp32 3.3 us.
#include "adaqp_train.h"
#include "philox.hpp"
#include "rows.hpp"

namespace adaqp {
namespace {

constexpr uint32_t kDropTag = 0x44524f50u;

struct DropArgs {
    const void *x, *add;
    void *y;
    const uint64_t *counter;
    int64_t ldx, lda, ldy, n_rows, span_x, span_add, first_row;
    uint64_t seed, pieces;                          // of all rows
    Divider pieces_of_row;
    int32_t dim, written;
    uint32_t threshold;
    float factor;
};

template <typename T, bool ADD>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropArgs a)
{
    constexpr int kEach = 2;
    const uint64_t seed = a.seed + (a.counter ? *a.counter : 0);
    const uint64_t first = (uint64_t)workgroup() * (kBlock * kEach) + threadIdx.x;
    int64_t row[kEach];
    int32_t col[kEach];
    float x[kEach][8], add[kEach][8];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint64_t at = min(first + e * kBlock, a.pieces - 1);
        row[e] = a.pieces_of_row.quotient(at);
        col[e] = (int32_t)(at - (uint64_t)row[e] * a.pieces_of_row.by) * 8;
        load_piece<T, 8>((const T *)a.x, row[e] * a.ldx + col[e], a.dim - col[e], a.span_x, x[e]);
        if (ADD) load_piece<T, 8>((const T *)a.add, row[e] * a.lda + col[e], a.dim - col[e], a.span_add, add[e]);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint64_t number = (uint64_t)a.first_row + (uint64_t)row[e];
        const Rand128 r = philox4x32_10((uint32_t)col[e] / 8, (uint32_t)number, (uint32_t)(number >> 32), kDropTag, (uint32_t)seed, (uint32_t)(seed >> 32));
        const uint32_t w[4] = {r.w0, r.w1, r.w2, r.w3};
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t number16 = k % 2 ? w[k / 2] >> 16 : w[k / 2] & 0xFFFFu;
            y[k] = number16 >= a.threshold ? x[e][k] * a.factor : 0.0f;
            if (ADD) y[k] += add[e][k];
            if (col[e] + k >= a.dim) y[k] = 0.0f;
        }
        if (first + e * kBlock < a.pieces) store_piece<T, 8>((T *)a.y + row[e] * a.ldy + col[e], a.written - col[e], y);
    }
}

template <typename T>
hipError_t launch(const DropArgs &a, hipStream_t st)
{
    const dim3 grid = grid_of((int64_t)((a.pieces + 2 * kBlock - 1) / (2 * kBlock)), kBlock);
    if (a.add) dropout_kernel<T, true><<<grid, kBlock, 0, st>>>(a);
    else       dropout_kernel<T, false><<<grid, kBlock, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_dropout(const void *x_dev, int64_t ldx, const void *add_dev, int64_t lda, int64_t n_rows, int32_t dim, int32_t type, double p, uint64_t seed,
                             int64_t first_row, const uint64_t *counter_dev, void *y_dev, int64_t ldy, void *stream)
{
    if (n_rows < 0 || dim <= 0 || !valid_type(type) || !(p >= 0.0 && p <= 1.0) || first_row < 0 || !aligned_to(counter_dev, 8)) return ADAQP_EINVAL;
    if (dim > kMostDim) return ADAQP_ESIZE;
    if (n_rows == 0) return ADAQP_OK;
    ADAQP_TRY(check_rows(x_dev, ldx, dim, type));
    ADAQP_TRY(check_rows(y_dev, ldy, dim, type));
    if (add_dev) ADAQP_TRY(check_rows(add_dev, lda, dim, type));
    if ((y_dev == x_dev && ldy != ldx) || (y_dev == add_dev && ldy != lda)) return ADAQP_EINVAL;
    if (!countable(n_rows, ldx) || !countable(n_rows, ldy) || (add_dev && !countable(n_rows, lda))) return ADAQP_ESIZE;
    DropArgs a{};
    a.x = x_dev; a.add = add_dev; a.y = y_dev; a.counter = counter_dev;
    a.ldx = ldx; a.lda = lda; a.ldy = ldy; a.n_rows = n_rows; a.first_row = first_row; a.seed = seed; a.dim = dim;
    a.span_x = matrix_span(n_rows, ldx, dim);
    a.span_add = matrix_span(n_rows, lda, dim);
    a.written = (int32_t)columns_to_write(y_dev, ldy, dim, element_bytes(type));
    const int64_t each = ((int64_t)a.written + 7) / 8;
    if (n_rows > kMostWorkgroups * kBlock / each) return ADAQP_ESIZE;
    a.pieces = (uint64_t)(n_rows * each);
    a.pieces_of_row = divider(each, (int64_t)a.pieces);
    a.threshold = (uint32_t)(p * 65536.0 + 0.5);
    a.factor = a.threshold < 65536 ? (float)(65536.0 / (65536.0 - a.threshold)) : 0.0f;
    if (type == ADAQP_F32) ADAQP_HIP_TRY((launch<float>(a, (hipStream_t)stream)));
    else                   ADAQP_HIP_TRY((launch<__bf16>(a, (hipStream_t)stream)));
    return ADAQP_OK;
}
