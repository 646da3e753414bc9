// Layer norm, forward and backward (adaqp_dense.h).
//
// A row is read once: LPR lanes hold it in registers, NV vectors of VW elements each (vector v * LPR + l in lane l), so that mean, centred
// squares and result need no second pass over memory, and the variance is that of the centred values.  Rows of up to 64 lanes' vectors lie
// within a wave (64 / LPR rows in one), longer ones take the 256 lanes of a workgroup; rows beyond the registers of those are walked in memory.
// Both directions are bound by memory: 8 and 12 bytes for about 8 and 15 operations on an element of fp32.  Measured: 58 000 x 602 fp32 forward 47 us (280 MB,
// 6.0 TB/s), 306 000 x 256 fp32 backward with the gradients of gamma and beta 171 and 5 us (942 MB, 5.4 TB/s); a copy of 1 GiB runs at 5.2 TB/s.  bf16, 58 000 x 602, forward 28 us
// (140 MB, 5.0 TB/s), backward 61 with both kernels (209 MB, 3.4 TB/s): a group of lanes waits for a row, reduces it and only then asks for its next.
//
// Rows of bf16 that begin anywhere are read and written in vectors all the same, aligned to two bytes: 40 000 x 1937 forward 74 us, with an element a
// lane 170.  Their last vector ends with the row and begins inside the one before; what both have counts once in the sums.
//
// The gradients of gamma and beta are sums over rows.  A lane keeps the same columns for all its rows, so it adds them up in
// registers; a workgroup leaves one row of sums, and a second kernel adds those in order.
#include "elements.hpp"

namespace adaqp {
namespace {

constexpr int kMostBlocks = 2048;       // of the backward pass: each leaves a row of sums

struct NormArgs {
    const void *x, *dy;
    void *out;                          // y or dx
    const float *gamma, *beta, *stats_in;
    float *stats;
    float *partial;                     // [blocks][2][dim], or NULL
    int64_t n_rows, ldx, lddy, ldo;
    int32_t dim;
    int32_t n_vec;                      // vectors that hold columns, the last perhaps not full
    int32_t n_vec_out;                  // that are written
    float eps;
};

// Sum over the lanes of a row.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float *lds)
{
    if constexpr (LPR <= kWave) return lane_sum<LPR>(v);
    else {
        static_assert(LPR == kBlock, "a row is a wave's or a workgroup's");
        v = lane_sum<kWave>(v);
        __syncthreads();                // what was read from lds before is done with
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        return (lds[0] + lds[1]) + (lds[2] + lds[3]);
    }
}

// How rows lie: PLAIN, whole vectors on multiples of their size; LINES, whole 128-byte lines (zeros behind the columns), dim a multiple of the vector;
// LINES_TAIL, the same with a vector that holds the last columns and padding; LOOSE, aligned to an element, the last vector moved back to end with the row.
enum Rows { PLAIN, LINES, LINES_TAIL, LOOSE };

// The columns of vector i: from `col` on; of its VW elements those from `first` to before `end` are its own.
template <Rows MODE, int VW>
struct Columns {
    int32_t col;
    int first, end;
    __device__ __forceinline__ Columns(int32_t i, int32_t dim) : col(i * VW), first(0), end(VW)
    {
        if (MODE == LINES_TAIL) end = min(VW, dim - col);
        if (MODE == LOOSE) {
            col = min(col, dim - VW);
            first = i * VW - col;
        }
    }
    __device__ __forceinline__ float own(int k, float v) const { return (MODE == LINES_TAIL && k >= end) || (MODE == LOOSE && k < first) ? 0.0f : v; }

    // f(whole) with an integral constant: whether all elements are the vector's own.  One lane of a row has a vector where they are not: the others do without the
    // selections.
    template <typename F>
    __device__ __forceinline__ void with(F f) const
    {
        if (MODE == PLAIN || MODE == LINES || (first == 0 && end == VW)) f(std::true_type());
        else                                                             f(std::false_type());
    }
};

template <typename T, int VW, Rows MODE>
__device__ __forceinline__ void load_columns(const T *row, const Columns<MODE, VW> &c, float (&v)[VW])
{
    if (MODE == LOOSE) load_loose<T, VW>(row + c.col, v);
    else               load_elements<T, VW>(row + c.col, v);
    if (MODE == LINES_TAIL && c.end < VW)
#pragma unroll
        for (int k = 0; k < VW; ++k) v[k] = c.own(k, v[k]);
}

template <typename T, int VW, Rows MODE>
__device__ __forceinline__ void store_columns(T *row, const Columns<MODE, VW> &c, const float (&v)[VW])
{
    if constexpr (MODE == LOOSE) store_loose<T, VW>(row + c.col, v);
    else                         store_elements<T, VW, MODE != PLAIN>(row + c.col, v);
}

template <Rows MODE, int VW>
__device__ __forceinline__ void load_params(const float *p, int32_t i, int32_t n_vec, int32_t dim, float other, float (&v)[VW])
{
#pragma unroll
    for (int k = 0; k < VW; ++k) v[k] = other;
    if (!p || i >= n_vec) return;
    const Columns<MODE, VW> c(i, dim);
    if (c.end == VW) {
        constexpr int W = VW < 4 ? VW : 4;
#pragma unroll
        for (int k = 0; k < VW; k += W) {
            float part[W];
            load_loose<float, W>(p + c.col + k, part);
#pragma unroll
            for (int j = 0; j < W; ++j) v[k + j] = part[j];
        }
    } else {
#pragma unroll
        for (int k = 0; k < VW; ++k)
            if (k < c.end) v[k] = p[c.col + k];
    }
}

template <typename T, int VW, int LPR, int NV, Rows MODE>
__global__ __launch_bounds__(kBlock) void layernorm_forward_kernel(NormArgs a)
{
    constexpr int kRows = kBlock / LPR;
    __shared__ float lds[kBlock / kWave];
    const int l = threadIdx.x % LPR, r = threadIdx.x / LPR;
    float gamma[NV][VW], beta[NV][VW];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        load_params<MODE, VW>(a.gamma, v * LPR + l, a.n_vec, a.dim, 1.0f, gamma[v]);
        load_params<MODE, VW>(a.beta, v * LPR + l, a.n_vec, a.dim, 0.0f, beta[v]);
    }
    const float dim = (float)a.dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + r; row < a.n_rows; row += (int64_t)gridDim.x * kRows) {
        const T *x = (const T *)a.x + row * a.ldx;
        float h[NV][VW];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t i = v * LPR + l;
            if (i < a.n_vec) load_columns<T, VW, MODE>(x, Columns<MODE, VW>(i, a.dim), h[v]);
            else for (int k = 0; k < VW; ++k) h[v][k] = 0.0f;
        }
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (MODE == LOOSE) {
                const Columns<MODE, VW> c(v * LPR + l, a.dim);
                c.with([&](auto whole) {
#pragma unroll
                    for (int k = 0; k < VW; ++k) sum += whole ? h[v][k] : c.own(k, h[v][k]);
                });
            } else {
#pragma unroll
                for (int k = 0; k < VW; ++k) sum += h[v][k];
            }
        }
        const float mean = row_sum<LPR>(sum, lds) / dim;
        sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t i = v * LPR + l;
            if (i < a.n_vec) {
                const Columns<MODE, VW> c(i, a.dim);
                c.with([&](auto whole) {
#pragma unroll
                    for (int k = 0; k < VW; ++k) {
                        h[v][k] -= mean;
                        const float d = whole ? h[v][k] : c.own(k, h[v][k]);
                        sum = fmaf(d, d, sum);
                    }
                });
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<LPR>(sum, lds) / dim + a.eps);
        if (a.stats && l == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = rstd;
        }
        T *y = (T *)a.out + row * a.ldo;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t i = v * LPR + l;
            float o[VW];
            if (i < a.n_vec) {
                const Columns<MODE, VW> c(i, a.dim);
#pragma unroll
                for (int k = 0; k < VW; ++k) o[k] = fmaf(h[v][k] * rstd, gamma[v][k], beta[v][k]);
                if (MODE == LINES_TAIL && c.end < VW)
#pragma unroll
                    for (int k = 0; k < VW; ++k) o[k] = c.own(k, o[k]);
                store_columns<T, VW, MODE>(y, c, o);
            } else if (MODE != LOOSE && i < a.n_vec_out) {
#pragma unroll
                for (int k = 0; k < VW; ++k) o[k] = 0.0f;
                store_elements<T, VW, MODE != PLAIN>(y + i * VW, o);
            }
        }
    }
}

template <typename T, int VW, int LPR, int NV, Rows MODE>
__global__ __launch_bounds__(kBlock) void layernorm_backward_kernel(NormArgs a)
{
    constexpr int kRows = kBlock / LPR, kCols = LPR * NV * VW;
    __shared__ float lds[kRows * kCols];
    const int l = threadIdx.x % LPR, r = threadIdx.x / LPR;
    float gamma[NV][VW], dgamma[NV][VW], dbeta[NV][VW];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        load_params<MODE, VW>(a.gamma, v * LPR + l, a.n_vec, a.dim, 1.0f, gamma[v]);
#pragma unroll
        for (int k = 0; k < VW; ++k) dgamma[v][k] = dbeta[v][k] = 0.0f;
    }
    const float dim = (float)a.dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + r; row < a.n_rows; row += (int64_t)gridDim.x * kRows) {
        const T *x = (const T *)a.x + row * a.ldx, *dy = (const T *)a.dy + row * a.lddy;
        float h[NV][VW], g[NV][VW];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t i = v * LPR + l;
            if (i < a.n_vec) {
                load_columns<T, VW, MODE>(x, Columns<MODE, VW>(i, a.dim), h[v]);
                load_columns<T, VW, MODE>(dy, Columns<MODE, VW>(i, a.dim), g[v]);
            }
        }
        const float mean = a.stats_in[2 * row], rstd = a.stats_in[2 * row + 1];
        float first = 0.0f, second = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t i = v * LPR + l;
            if (i < a.n_vec) {
                const Columns<MODE, VW> c(i, a.dim);
                c.with([&](auto whole) {
#pragma unroll
                    for (int k = 0; k < VW; ++k) {
                        h[v][k] = (h[v][k] - mean) * rstd;
                        const float own_h = whole ? h[v][k] : c.own(k, h[v][k]), d = whole ? g[v][k] : c.own(k, g[v][k]);
                        dgamma[v][k] = fmaf(d, own_h, dgamma[v][k]);
                        dbeta[v][k] += d;
                        g[v][k] *= gamma[v][k];
                        const float own_g = whole ? g[v][k] : c.own(k, g[v][k]);
                        first += own_g;
                        second = fmaf(own_g, own_h, second);
                    }
                });
            }
        }
        if (a.out) {
            first = row_sum<LPR>(first, lds) / dim;
            second = row_sum<LPR>(second, lds) / dim;
            T *dx = (T *)a.out + row * a.ldo;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int32_t i = v * LPR + l;
                float o[VW];
                if (i < a.n_vec) {
                    const Columns<MODE, VW> c(i, a.dim);
#pragma unroll
                    for (int k = 0; k < VW; ++k) o[k] = rstd * (g[v][k] - fmaf(h[v][k], second, first));
                    if (MODE == LINES_TAIL && c.end < VW)
#pragma unroll
                        for (int k = 0; k < VW; ++k) o[k] = c.own(k, o[k]);
                    store_columns<T, VW, MODE>(dx, c, o);
                } else if (MODE != LOOSE && i < a.n_vec_out) {
#pragma unroll
                    for (int k = 0; k < VW; ++k) o[k] = 0.0f;
                    store_elements<T, VW, MODE != PLAIN>(dx + i * VW, o);
                }
            }
        }
    }
    if (!a.partial) return;
    float *to = a.partial + (int64_t)blockIdx.x * 2 * a.dim;
    const int32_t last = (a.n_vec - 1) * VW;        // column of the last vector, which a LOOSE one may be behind
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int k = 0; k < VW; ++k) lds[r * kCols + (v * LPR + l) * VW + k] = which ? dbeta[v][k] : dgamma[v][k];
        __syncthreads();
        for (int32_t col = threadIdx.x; col < a.dim; col += kBlock) {
            const int32_t at = MODE == LOOSE && col >= last ? col + last + VW - a.dim : col;
            float sum = 0.0f;
            for (int q = 0; q < kRows; ++q) sum += lds[q * kCols + at];
            to[which * a.dim + col] = sum;
        }
    }
}

// Rows longer than a workgroup's registers: several passes over the row, which lies in the caches after the first.
template <typename T>
__global__ __launch_bounds__(kBlock) void layernorm_forward_long_kernel(NormArgs a)
{
    __shared__ float lds[kBlock / kWave];
    const float dim = (float)a.dim;
    for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx;
        float sum = 0.0f;
        for (int32_t j = threadIdx.x; j < a.dim; j += kBlock) sum += (float)x[j];
        const float mean = row_sum<kBlock>(sum, lds) / dim;
        sum = 0.0f;
        for (int32_t j = threadIdx.x; j < a.dim; j += kBlock) sum = fmaf((float)x[j] - mean, (float)x[j] - mean, sum);
        const float rstd = 1.0f / sqrtf(row_sum<kBlock>(sum, lds) / dim + a.eps);
        if (a.stats && threadIdx.x == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = rstd;
        }
        T *y = (T *)a.out + row * a.ldo;
        for (int32_t j = threadIdx.x; j < a.n_vec_out; j += kBlock)
            y[j] = j < a.dim ? (T)fmaf(((float)x[j] - mean) * rstd, a.gamma ? a.gamma[j] : 1.0f, a.beta ? a.beta[j] : 0.0f) : (T)0.0f;
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void layernorm_backward_long_kernel(NormArgs a)
{
    __shared__ float lds[kBlock / kWave];
    const float dim = (float)a.dim;
    float *to = a.partial ? a.partial + (int64_t)blockIdx.x * 2 * a.dim : nullptr;
    for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx, *dy = (const T *)a.dy + row * a.lddy;
        const float mean = a.stats_in[2 * row], rstd = a.stats_in[2 * row + 1];
        float first = 0.0f, second = 0.0f;
        for (int32_t j = threadIdx.x; j < a.dim; j += kBlock) {
            const float d = (float)dy[j], g = d * (a.gamma ? a.gamma[j] : 1.0f), h = ((float)x[j] - mean) * rstd;
            first += g;
            second = fmaf(g, h, second);
            if (to) {                   // a column is one thread's in every row
                to[j] = fmaf(d, h, row == blockIdx.x ? 0.0f : to[j]);
                to[a.dim + j] = d + (row == blockIdx.x ? 0.0f : to[a.dim + j]);
            }
        }
        if (!a.out) continue;
        first = row_sum<kBlock>(first, lds) / dim;
        second = row_sum<kBlock>(second, lds) / dim;
        T *dx = (T *)a.out + row * a.ldo;
        for (int32_t j = threadIdx.x; j < a.n_vec_out; j += kBlock) {
            const float h = j < a.dim ? ((float)x[j] - mean) * rstd : 0.0f;
            const float g = j < a.dim ? (float)dy[j] * (a.gamma ? a.gamma[j] : 1.0f) : 0.0f;
            dx[j] = j < a.dim ? (T)(rstd * (g - fmaf(h, second, first))) : (T)0.0f;
        }
    }
}

// dgamma and dbeta: the sums over n_blocks rows of [2][dim], 32 columns a workgroup.
__global__ __launch_bounds__(1024) void layernorm_params_kernel(const float *partial, int32_t n_blocks, int32_t dim, float *dgamma, float *dbeta)
{
    constexpr int kCols = 32, kSlices = 1024 / kCols;
    __shared__ float lds[kSlices][kCols];
    const int c = threadIdx.x % kCols, slice = threadIdx.x / kCols;
    const int64_t col = (int64_t)workgroup() * kCols + c, width = 2 * (int64_t)dim;
    float sum = 0.0f;
    if (col < width) {
#pragma unroll 8
        for (int b = slice; b < n_blocks; b += kSlices) sum += partial[b * width + col];
    }
    lds[slice][c] = sum;
    __syncthreads();
    if (slice != 0 || col >= width) return;
    for (int s = 1; s < kSlices; ++s) sum += lds[s][c];
    if (col < dim) dgamma[col] = sum;
    else           dbeta[col - dim] = sum;
}

// How a launch holds its rows.
struct NormShape {
    int vw, lpr, nv;                    // lpr 0: rows walked in memory
    int64_t blocks;                     // of the backward pass
};

constexpr int kLongLanes = 0;
constexpr int32_t kMostColumns = 1 << 30;       // so that counting them in steps stays within 32 bits

// Lanes per row: the fewest of 8, 16, 32, 64 that have at most four vectors each, then 64 with up to eight, then a workgroup.
// `cols`: that are read or written.
NormShape norm_shape(int64_t n_rows, int64_t cols, int vw)
{
    NormShape s{vw, kLongLanes, 0, 0};
    const int64_t n_vec = (cols + vw - 1) / vw;
    if (n_vec <= 64 * 8) {
        s.lpr = 8;
        while (s.lpr < 64 && n_vec > s.lpr * 4) s.lpr *= 2;
        s.nv = s.lpr == 64 && n_vec <= 64 * 3 ? 3 : n_vec <= s.lpr * 4 ? 4 : n_vec <= s.lpr * 6 ? 6 : 8;
    } else if (n_vec <= kBlock * 8 && vw * 8 <= 32) {
        s.lpr = kBlock;
        s.nv = n_vec <= kBlock * 4 ? 4 : 8;
    }
    const int64_t rows = s.lpr ? kBlock / s.lpr : 1;
    s.blocks = (n_rows + rows - 1) / rows;
    const int64_t most = s.nv * s.vw <= 8 ? kMostBlocks : kMostBlocks / 2;
    if (s.blocks > most) s.blocks = most;
    return s;
}

// f(integral constants for vw, lpr, nv)
template <typename T, int VW, typename F>
void with_shape(const NormShape &s, F f)
{
    using std::integral_constant;
    using W = integral_constant<int, VW>;
    if (s.lpr == 8)       f(W(), integral_constant<int, 8>(), integral_constant<int, 4>());
    else if (s.lpr == 16) f(W(), integral_constant<int, 16>(), integral_constant<int, 4>());
    else if (s.lpr == 32) f(W(), integral_constant<int, 32>(), integral_constant<int, 4>());
    else if (s.lpr == 64) {
        if (s.nv == 3)      f(W(), integral_constant<int, 64>(), integral_constant<int, 3>());
        else if (s.nv == 4) f(W(), integral_constant<int, 64>(), integral_constant<int, 4>());
        else if (VW <= 4 && s.nv == 6) f(W(), integral_constant<int, 64>(), integral_constant<int, VW <= 4 ? 6 : 4>());
        else if (VW <= 4) f(W(), integral_constant<int, 64>(), integral_constant<int, VW <= 4 ? 8 : 4>());
    } else if (VW <= 4) {
        if (s.nv == 4)    f(W(), integral_constant<int, kBlock>(), integral_constant<int, 4>());
        else              f(W(), integral_constant<int, kBlock>(), integral_constant<int, VW <= 4 ? 8 : 4>());
    }
}

template <typename T>
constexpr int most_elements() { return 16 / (int)sizeof(T); }

int32_t columns_written(bool whole, int32_t dim, int64_t bytes)
{
    const int32_t line = (int32_t)(128 / bytes);
    return whole ? (dim + line - 1) / line * line : dim;
}

// Vectors for all matrices of a call, how rows lie, and whether those that are written have whole lines.
struct NormLayout { int vw; Rows mode; bool whole; };

NormLayout norm_layout(const void *x, int64_t ldx, const void *dy, int64_t lddy, const void *out, int64_t ldo, int32_t dim, int64_t bytes)
{
    NormLayout n;
    // Vectors of 8 bf16 up to 2048 columns, beyond which the registers do not suffice; backward, which keeps five numbers a column, 4 up to 1024 (us with 8 and 4:
    // 58 000 x 602 87, 61; 24 000 x 301 21, 18; 40 000 x 1937 118, 166; forward 306 000 x 256 66, 99).
    const int most = (int)(16 / bytes), wide = dim > 2048 || (dy && dim <= 1024) ? 4 : 8;
    n.whole = out && whole_lines(out, ldo, bytes);
    n.mode = PLAIN;
    const bool all = whole_lines(x, ldx, bytes) && (!dy || whole_lines(dy, lddy, bytes)) && (!out || n.whole);
    if (all) {
        n.vw = most < wide ? most : wide;                   // rows own their lines: the last vector may reach into the padding
        n.mode = dim % n.vw ? LINES_TAIL : LINES;
        return n;
    }
    n.vw = vector_elements(x, ldx, dim, bytes);
    if (dy) { const int w = vector_elements(dy, lddy, dim, bytes); if (w < n.vw) n.vw = w; }
    if (out) { const int w = vector_elements(out, ldo, dim, bytes); if (w < n.vw) n.vw = w; }
    if (n.vw > wide) n.vw = wide;
    if (bytes == 2 && n.vw <= 2 && dim >= 8 && !n.whole) {
        n.vw = wide;
        n.mode = LOOSE;
    }
    return n;
}

template <typename T, bool BACKWARD>
hipError_t launch_norm(NormArgs a, const NormLayout &n, const NormShape &s, hipStream_t st)
{
    const int32_t written = columns_written(n.whole, a.dim, sizeof(T));
    if (!s.lpr) {
        a.n_vec_out = written;
        if (BACKWARD) layernorm_backward_long_kernel<T><<<(uint32_t)s.blocks, kBlock, 0, st>>>(a);
        else          layernorm_forward_long_kernel<T><<<(uint32_t)(a.n_rows < 4096 ? a.n_rows : 4096), kBlock, 0, st>>>(a);
        return hipGetLastError();
    }
    a.n_vec = (a.dim + s.vw - 1) / s.vw;
    a.n_vec_out = (written + s.vw - 1) / s.vw;
    auto go = [&](auto vw, auto lpr, auto nv) {
        constexpr int VW = decltype(vw)::value, LPR = decltype(lpr)::value, NV = decltype(nv)::value;
        const int64_t rows = kBlock / LPR;
        int64_t blocks = BACKWARD ? s.blocks : (a.n_rows + rows - 1) / rows;
        if (blocks > 2048) blocks = 2048;
        auto run = [&](auto mode) {
            constexpr Rows MODE = decltype(mode)::value;
            if constexpr (BACKWARD) layernorm_backward_kernel<T, VW, LPR, NV, MODE><<<(uint32_t)blocks, kBlock, 0, st>>>(a);
            else                    layernorm_forward_kernel<T, VW, LPR, NV, MODE><<<(uint32_t)blocks, kBlock, 0, st>>>(a);
        };
        constexpr bool kWide = VW * (int)sizeof(T) == 16 || (VW == 4 && sizeof(T) == 2);
        if (n.mode == PLAIN) run(std::integral_constant<Rows, PLAIN>());
        if constexpr (kWide) {
            if (n.mode == LINES) run(std::integral_constant<Rows, LINES>());
            if (n.mode == LINES_TAIL) run(std::integral_constant<Rows, LINES_TAIL>());
            if constexpr (sizeof(T) == 2)
                if (n.mode == LOOSE) run(std::integral_constant<Rows, LOOSE>());
        }
    };
    if (s.vw == 1)      with_shape<T, 1>(s, go);
    else if (s.vw == 2) with_shape<T, 2>(s, go);
    else if (s.vw == 4) with_shape<T, 4>(s, go);
    else if constexpr (most_elements<T>() == 8) with_shape<T, 8>(s, go);
    return hipGetLastError();
}

int check_matrix(const void *p, int64_t ld, int64_t cols, int32_t type)
{
    return p && ld >= cols && aligned_to(p, element_bytes(type)) ? ADAQP_OK : ADAQP_EINVAL;
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_layernorm_forward(const void *x_dev, int64_t ldx, int64_t n_rows, int32_t dim, int32_t type,
                                       const float *gamma_dev, const float *beta_dev, float eps,
                                       void *y_dev, int64_t ldy, float *stats_dev, void *stream)
{
    if (n_rows < 0 || dim <= 0 || !valid_type(type) || !(eps >= 0.0f && eps <= 3.402823466e+38f)) return ADAQP_EINVAL;
    if (!aligned_to(gamma_dev, 4) || !aligned_to(beta_dev, 4) || !aligned_to(stats_dev, 4)) return ADAQP_EINVAL;
    if (dim > kMostColumns) return ADAQP_ESIZE;
    if (n_rows == 0) return ADAQP_OK;
    ADAQP_TRY(check_matrix(x_dev, ldx, dim, type));
    ADAQP_TRY(check_matrix(y_dev, ldy, dim, type));
    if (x_dev == y_dev && ldx != ldy) return ADAQP_EINVAL;
    NormArgs a{};
    a.x = x_dev; a.out = y_dev; a.gamma = gamma_dev; a.beta = beta_dev; a.stats = stats_dev;
    a.n_rows = n_rows; a.ldx = ldx; a.ldo = ldy; a.dim = dim; a.eps = eps;
    const NormLayout n = norm_layout(x_dev, ldx, nullptr, 0, y_dev, ldy, dim, element_bytes(type));
    const NormShape s = norm_shape(n_rows, columns_written(n.whole, dim, element_bytes(type)), n.vw);
    if (type == ADAQP_F32) ADAQP_HIP_TRY((launch_norm<float, false>(a, n, s, (hipStream_t)stream)));
    else                   ADAQP_HIP_TRY((launch_norm<__bf16, false>(a, n, s, (hipStream_t)stream)));
    return ADAQP_OK;
}

extern "C" int adaqp_layernorm_workspace_bytes(int64_t n_rows, int32_t dim, int64_t *bytes_out)
{
    if (!bytes_out || n_rows < 0 || dim <= 0) return ADAQP_EINVAL;
    if (dim > kMostColumns) return ADAQP_ESIZE;
    const int64_t blocks = n_rows < kMostBlocks ? n_rows : kMostBlocks;
    *bytes_out = (blocks * 2 * dim * 4 + 255) / 256 * 256;
    return ADAQP_OK;
}

extern "C" int adaqp_layernorm_backward(const void *x_dev, int64_t ldx, const void *dy_dev, int64_t lddy, int64_t n_rows, int32_t dim,
                                        int32_t type, const float *stats_dev, const float *gamma_dev, void *dx_dev, int64_t lddx,
                                        float *dgamma_dev, float *dbeta_dev, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (n_rows < 0 || dim <= 0 || !valid_type(type) || !dgamma_dev != !dbeta_dev) return ADAQP_EINVAL;
    if (!aligned_to(gamma_dev, 4) || !aligned_to(stats_dev, 4) || !aligned_to(dgamma_dev, 4) || !aligned_to(dbeta_dev, 4)) return ADAQP_EINVAL;
    if (dim > kMostColumns) return ADAQP_ESIZE;
    if (n_rows > 0) {
        if (!stats_dev) return ADAQP_EINVAL;
        ADAQP_TRY(check_matrix(x_dev, ldx, dim, type));
        ADAQP_TRY(check_matrix(dy_dev, lddy, dim, type));
        if (dx_dev) ADAQP_TRY(check_matrix(dx_dev, lddx, dim, type));
        if ((dx_dev == x_dev && lddx != ldx) || (dx_dev == dy_dev && lddx != lddy)) return ADAQP_EINVAL;
        if (dgamma_dev) {
            int64_t need;
            ADAQP_TRY(adaqp_layernorm_workspace_bytes(n_rows, dim, &need));
            if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
            if (workspace_bytes < need) return ADAQP_ESIZE;
        }
    }
    NormShape s{};
    if (n_rows > 0 && (dx_dev || dgamma_dev)) {
        NormArgs a{};
        a.x = x_dev; a.dy = dy_dev; a.out = dx_dev; a.gamma = gamma_dev; a.stats_in = stats_dev;
        a.partial = dgamma_dev ? (float *)workspace_dev : nullptr;
        a.n_rows = n_rows; a.ldx = ldx; a.lddy = lddy; a.ldo = lddx; a.dim = dim;
        const NormLayout n = norm_layout(x_dev, ldx, dy_dev, lddy, dx_dev, lddx, dim, element_bytes(type));
        s = norm_shape(n_rows, columns_written(n.whole, dim, element_bytes(type)), n.vw);
        if (type == ADAQP_F32) ADAQP_HIP_TRY((launch_norm<float, true>(a, n, s, (hipStream_t)stream)));
        else                   ADAQP_HIP_TRY((launch_norm<__bf16, true>(a, n, s, (hipStream_t)stream)));
    }
    if (dgamma_dev) {
        const int64_t blocks = (2 * (int64_t)dim + 31) / 32;
        layernorm_params_kernel<<<grid_of(blocks, 1024), 1024, 0, (hipStream_t)stream>>>((const float *)workspace_dev, (int32_t)s.blocks, dim, dgamma_dev,
                                                                                    dbeta_dev);
        ADAQP_HIP_TRY(hipGetLastError());
    }
    return ADAQP_OK;
}
