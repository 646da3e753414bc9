// Newton-Schulz steps on the matrix cores (adaqp_dense.h).
//
// With n <= m a step is three products: A = X X^T (n x n over m), Q = a I + b A + c A A (n x n over n) and X <- Q X (n x m over n).  A and Q are symmetric,
// so only the tiles on and below the diagonal are computed and each is stored twice.
//
// fp32 products run at a sixteenth of the fp16 rate on this machine, and fp16 has 11 bits.  Every matrix is therefore held as hi + lo, two
// fp16 numbers with 22 bits together, in units of a power of two that keeps the entries below 2^14 (the host knows a bound on the singular values after
// every step), and a product is hi hi + hi lo + lo hi, summed in fp32: what is left out is below 2^-22 of a term.  Memory holds lines of 128 bytes: 32 hi,
// then the 32 lo of the same columns, which is what a step of the products' loop takes of a row.  Both X and its transpose are kept, since the loop
// runs along rows of both operands.
#include <math.h>

#include "elements.hpp"
#include "lines.hpp"

namespace adaqp {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float sums16 __attribute__((ext_vector_type(16)));

constexpr int kPad = 64;                            // rows and columns of the held matrices are multiples
constexpr int kNormBlocks = 256;                    // of a matrix, at most
constexpr int kMostPower = 14;
constexpr int64_t kMostSize = (int64_t)1 << 20;

// Where (row, col) of a held matrix lies: hi there, lo 64 bytes on.
__device__ __forceinline__ int64_t held_at(int64_t row, int64_t col, int64_t pitch) { return row * pitch + col / 32 * kLine + col % 32 * 2; }

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

// Sums of squares of a share of each matrix: blocks [x] of matrix [y], runs of kBlock columns of a row.
template <typename T>
__global__ __launch_bounds__(kBlock) void update_norm_kernel(const T *g, int64_t ldg, int64_t stride, int64_t n_rows, int64_t n_cols, double *partial)
{
    __shared__ double lds[kWavesPerBlock];
    g += blockIdx.y * stride;
    const uint32_t runs = (uint32_t)((n_cols + kBlock - 1) / kBlock);
    const int64_t total = n_rows * runs;
    double sum = 0.0;
#pragma unroll 4
    for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
        const uint32_t row = (uint32_t)((uint64_t)at / runs), col = ((uint32_t)at - row * runs) * kBlock + threadIdx.x;
        const double v = col < n_cols ? (double)(float)g[row * ldg + col] : 0.0;
        sum = fma(v, v, sum);
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// G / (norm + eps) in units of 2^-power as held matrices: as it lies (`same`) and transposed (`other`), zeros up to the padded sizes.  A workgroup takes 64 x 64.
template <typename T>
__global__ __launch_bounds__(kBlock) void update_split_kernel(const T *g, int64_t ldg, int64_t stride, int64_t n_rows, int64_t n_cols, const double *partial,
                                                              int n_partial, double eps, int power, uint8_t *same, uint8_t *other, int64_t pitch_same,
                                                              int64_t pitch_other, int64_t held_bytes)
{
    __shared__ double lds[kWavesPerBlock];
    __shared__ float tile[kPad][kPad + 1];
    g += blockIdx.z * stride;
    same += blockIdx.z * held_bytes;
    other += blockIdx.z * held_bytes;
    constexpr int kEach = kPad * kPad / kBlock;
    const int64_t row0 = (int64_t)blockIdx.y * kPad, col0 = (int64_t)blockIdx.x * kPad;
    const int c = threadIdx.x % kPad, r0 = threadIdx.x / kPad;
    float v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t row = row0 + r0 + i * (kBlock / kPad), col = col0 + c;
        v[i] = row < n_rows && col < n_cols ? (float)g[row * ldg + col] : 0.0f;
    }
    const double total = block_sum((int)threadIdx.x < n_partial ? partial[blockIdx.z * n_partial + threadIdx.x] : 0.0, lds);
    const double scale = ldexp(1.0 / (sqrt(total) + eps), power);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = r0 + i * (kBlock / kPad);
        const int64_t row = row0 + r, col = col0 + c;
        v[i] = row < n_rows && col < n_cols ? (float)((double)v[i] * scale) : 0.0f;       // behind the edge also where the scale is not finite
        tile[r][c] = v[i];
        _Float16 hi, lo;
        split(v[i], hi, lo);
        uint8_t *to = same + held_at(row, col, pitch_same);
        *reinterpret_cast<_Float16 *>(to) = hi;
        *reinterpret_cast<_Float16 *>(to + 64) = lo;
    }
    __syncthreads();
    for (int r = threadIdx.x / kPad; r < kPad; r += kBlock / kPad) {
        _Float16 hi, lo;
        split(tile[c][r], hi, lo);
        uint8_t *to = other + held_at(col0 + r, row0 + c, pitch_other);
        *reinterpret_cast<_Float16 *>(to) = hi;
        *reinterpret_cast<_Float16 *>(to + 64) = lo;
    }
}

enum Product { GRAM, POLY, STEP, LAST };

struct ProductArgs {
    const uint8_t *p, *q;                           // D = p q^T
    int64_t rows, cols;                             // of D, padded
    int64_t lines;                                  // of a row of p and q that hold columns
    int64_t pitch;                                  // of p and q
    uint8_t *same, *other;                          // D and its transpose, held
    int64_t pitch_same, pitch_other;
    int64_t bytes_p, bytes_q, bytes_d;              // from matrix to matrix
    float scale;                                    // of the sums in the units of what is stored
    float diagonal, linear;                         // POLY: what is added, of I and of p, in those units
    void *out;                                      // LAST: D itself
    int64_t ldo, stride_o, out_rows, out_cols, written;
    int64_t tiles_r, tiles_c;
};

template <Product KIND, typename T, int TILE, int STAGES>
__global__ __launch_bounds__(kBlock) void update_product_kernel(ProductArgs g)
{
    constexpr bool kSymmetric = KIND == GRAM || KIND == POLY;
    constexpr int F = TILE / 64;                    // 32 x 32 parts of a wave, both ways
    __shared__ struct { uint8_t p[TILE * kLine], q[TILE * kLine]; } stage[STAGES];
    int64_t tr, tc;
    if (kSymmetric) {                               // tiles below and on the diagonal, row by row
        tr = (int64_t)((sqrtf(8.0f * blockIdx.x + 1.0f) - 1.0f) * 0.5f);
        while (tr * (tr + 1) / 2 > blockIdx.x) --tr;
        while ((tr + 1) * (tr + 2) / 2 <= blockIdx.x) ++tr;
        tc = blockIdx.x - tr * (tr + 1) / 2;
    } else {
        const TilePlace place = tile_place(blockIdx.x, gridDim.x, (uint32_t)g.tiles_r, (uint32_t)g.tiles_c, 1);
        if (place.part < 0) return;
        tr = place.row;
        tc = place.col;
    }
    const uint8_t *p = g.p + blockIdx.y * g.bytes_p, *q = g.q + blockIdx.y * g.bytes_q;
    const int64_t row0 = tr * TILE, col0 = tc * TILE, pitch = g.pitch;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int wr = wave / 2 * (TILE / 2), wc = wave % 2 * (TILE / 2);

    sums16 sums[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[i][j][e] = 0.0f;

    const TileLoads<TILE> of_p(row0, g.rows, pitch), of_q(col0, g.cols, pitch);
    constexpr int kLoads = 2 * TileLoads<TILE>::kLoads;
    const uint8_t *from_p = p + row0 * pitch, *from_q = q + col0 * pitch;
    // Load i of a line of both operands.
    auto load = [&](int i, int line, const auto &s) {
        if (i < kLoads / 2) of_p.template load<false>(i, from_p + (int64_t)line * kLine, TileLoads<TILE>::place(s.p));
        else                of_q.template load<false>(i - kLoads / 2, from_q + (int64_t)line * kLine, TileLoads<TILE>::place(s.q));
    };
    // The operands of half a line, 16 columns: read from the LDS while the half before is multiplied.
    struct Half { half8 ph[F], pl[F], qh[F], ql[F]; } half[2];
    auto read = [&](const auto &s, int k, Half &to) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            to.ph[i] = *reinterpret_cast<const half8 *>(line_part(s.p, wr + i * 32 + r, k * 2 + h));
            to.pl[i] = *reinterpret_cast<const half8 *>(line_part(s.p, wr + i * 32 + r, 4 + k * 2 + h));
            to.qh[i] = *reinterpret_cast<const half8 *>(line_part(s.q, wc + i * 32 + r, k * 2 + h));
            to.ql[i] = *reinterpret_cast<const half8 *>(line_part(s.q, wc + i * 32 + r, 4 + k * 2 + h));
        }
    };
    // `between(p)` is done behind product p of the half's 3 F F.
    auto multiply = [&](const Half &f, auto between) {
#pragma unroll
        for (int w = 0; w < 3; ++w)                 // the small ones first
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int j = 0; j < F; ++j) {
                    sums[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w == 0 ? f.pl[i] : f.ph[i], w == 1 ? f.ql[j] : f.qh[j], sums[i][j], 0, 0, 0);
                    between((w * F + i) * F + j);
                }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto nothing = [](int) {};

    // Up to STAGES lines are under way.  A line's second half is multiplied behind the barrier after which the next line is in the LDS and its own buffer
    // free, and the loads into that buffer are issued between its products.  No branches: across one the compiler would take products to the other side
    // of the barrier.
    const int lines = (int)g.lines;
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < lines)
#pragma unroll
            for (int l = 0; l < kLoads; ++l) load(l, s, stage[s]);
    if (lines >= STAGES) arrived<kLoads * (STAGES - 1)>();
    else                 arrived<0>();
    read(stage[0], 0, half[0]);
    int now = 0;
    auto one = [&](int line, auto more) {
        constexpr bool kMore = decltype(more)::value;
        const auto &s = stage[now];
        now = now + 1 == STAGES ? 0 : now + 1;
        read(s, 1, half[1]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[0], nothing);
        arrived<kMore ? kLoads * (STAGES - 2) : 0>();
        read(stage[now], 0, half[0]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[1], [&](int p) {
            if constexpr (kMore) {
#pragma unroll
                for (int l = p * kLoads / (3 * F * F); l < (p + 1) * kLoads / (3 * F * F); ++l) load(l, line + STAGES, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    };
    int line = 0;
    for (; line + STAGES < lines; ++line) one(line, std::true_type());
    for (; line < lines; ++line) one(line, std::false_type());

    uint8_t *same = g.same + blockIdx.y * g.bytes_d, *other = g.other + blockIdx.y * g.bytes_d;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int64_t col = col0 + wc + j * 32 + r;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int64_t row = row0 + wr + i * 32 + e / 4 * 8 + h * 4;
                if (row >= g.rows || col >= g.cols) continue;
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[k] = sums[i][j][e + k] * g.scale;
                    if (KIND == POLY) {
                        const uint8_t *from = p + held_at(row + k, col, pitch);
                        const float a = (float)*reinterpret_cast<const _Float16 *>(from) + (float)*reinterpret_cast<const _Float16 *>(from + 64);
                        v[k] = fmaf(g.linear, a, v[k]) + (row + k == col ? g.diagonal : 0.0f);
                    }
                }
                if constexpr (KIND == LAST) {
                    T *out = (T *)g.out + blockIdx.y * g.stride_o;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (row + k < g.out_rows && col < g.written) out[(row + k) * g.ldo + col] = col < g.out_cols ? (T)v[k] : (T)0.0f;
                } else {
                    half4 hi, lo;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        _Float16 a, b;
                        split(v[k], a, b);
                        hi[k] = a;
                        lo[k] = b;
                        uint8_t *to = same + held_at(row + k, col, g.pitch_same);
                        *reinterpret_cast<_Float16 *>(to) = a;
                        *reinterpret_cast<_Float16 *>(to + 64) = b;
                    }
                    if (!kSymmetric || tr != tc) {  // of a tile on the diagonal both halves are there
                        uint8_t *to = other + held_at(col, row, g.pitch_other);
                        *reinterpret_cast<half4 *>(to) = hi;
                        *reinterpret_cast<half4 *>(to + 64) = lo;
                    }
                }
            }
        }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void update_scale_kernel(const T *g, int64_t ldg, int64_t stride, int64_t n_rows, int64_t n_cols, const double *partial,
                                                              int n_partial, double eps, T *out, int64_t ldo, int64_t stride_o, int64_t written)
{
    __shared__ double lds[kWavesPerBlock];
    const double total = block_sum((int)threadIdx.x < n_partial ? partial[blockIdx.y * n_partial + threadIdx.x] : 0.0, lds);
    const double scale = 1.0 / (sqrt(total) + eps);
    g += blockIdx.y * stride;
    out += blockIdx.y * stride_o;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < n_rows * written; at += (int64_t)gridDim.x * kBlock) {
        const int64_t row = at / written, col = at % written;
        out[row * ldo + col] = col < n_cols ? (T)(float)((double)(float)g[row * ldg + col] * scale) : (T)0.0f;
    }
}

int64_t padded(int64_t v) { return (v + kPad - 1) / kPad * kPad; }

// Bytes from row to row of a held matrix: an odd number of lines, so that the same line of all rows is spread over the L2's channels.
int64_t held_pitch(int64_t cols) { return (cols / 32 | 1) * kLine; }

struct UpdateLayout {
    bool flip;                                      // more rows than columns: X is the transpose
    int64_t n, m;                                   // padded, n of the smaller
    int64_t big, small;                             // bytes of X and of A
    int64_t norm_blocks;
    int64_t partial_at, x_at, a_at, q_at, bytes;    // X, its transpose, both again for the next step
};

UpdateLayout update_layout(int32_t n_matrices, int64_t n_rows, int64_t n_cols)
{
    UpdateLayout u;
    u.flip = n_rows > n_cols;
    u.n = padded(u.flip ? n_cols : n_rows);
    u.m = padded(u.flip ? n_rows : n_cols);
    const int64_t of_x = u.n * held_pitch(u.m), of_xt = u.m * held_pitch(u.n);
    u.big = of_x > of_xt ? of_x : of_xt;
    u.small = u.n * held_pitch(u.n);
    u.norm_blocks = (n_rows * ((n_cols + kBlock - 1) / kBlock) + 3) / 4;
    if (u.norm_blocks > kNormBlocks) u.norm_blocks = kNormBlocks;
    u.partial_at = 0;
    u.x_at = (n_matrices * u.norm_blocks * 8 + 255) / 256 * 256;
    u.a_at = u.x_at + 4 * n_matrices * u.big;
    u.q_at = u.a_at + n_matrices * u.small;
    u.bytes = u.q_at + n_matrices * u.small;
    return u;
}

// The largest |x q(x^2)| and |q(x^2)| over 0 <= x <= most, q(y) = a + b y + c y^2: at the ends or where a derivative is zero.
void bounds(double a, double b, double c, double most, double *of_step, double *of_q)
{
    const double end = most * most;
    auto q = [&](double y) { return fabs(a + b * y + c * y * y); };
    double step = most * q(end), quadratic = fmax(q(0.0), q(end));
    auto at = [&](double y, bool both) {
        if (!(y > 0.0 && y < end)) return;
        step = fmax(step, sqrt(y) * q(y));
        if (both) quadratic = fmax(quadratic, q(y));
    };
    if (c != 0.0) {
        at(-b / (2.0 * c), true);
        const double root = 9.0 * b * b - 20.0 * a * c;             // a + 3 b y + 5 c y^2 = 0
        if (root >= 0.0) {
            at((-3.0 * b + sqrt(root)) / (10.0 * c), false);
            at((-3.0 * b - sqrt(root)) / (10.0 * c), false);
        }
    } else if (b != 0.0) at(-a / (3.0 * b), false);
    *of_step = step;
    *of_q = quadratic;
}

// The power of two whose units keep numbers up to `most` (with what rounding adds) below 2^14 and a bit.
int power_for(double most)
{
    int e;
    frexp(fmax(most, 1e-6) * 1.001, &e);            // most <= 2^e
    return kMostPower - e;
}

template <Product KIND, typename T>
hipError_t launch_product(ProductArgs g, int32_t n_matrices, hipStream_t st)
{
    constexpr bool kSymmetric = KIND == GRAM || KIND == POLY;
    auto tiles = [&](int64_t t) {
        g.tiles_r = (g.rows + t - 1) / t;
        g.tiles_c = (g.cols + t - 1) / t;
        return (kSymmetric ? g.tiles_r * (g.tiles_r + 1) / 2 : g.tiles_r * g.tiles_c);
    };
    const int64_t large = tiles(128);
    if (large * n_matrices >= 256) {
        update_product_kernel<KIND, T, 128, 2><<<dim3((uint32_t)(kSymmetric ? large : tile_blocks(large, 1)), (uint32_t)n_matrices), kBlock, 0, st>>>(g);
    } else {
        const int64_t small = tiles(64);
        update_product_kernel<KIND, T, 64, 4><<<dim3((uint32_t)(kSymmetric ? small : tile_blocks(small, 1)), (uint32_t)n_matrices), kBlock, 0, st>>>(g);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t orthogonalize(const T *g, int64_t ldg, int64_t stride_g, T *out, int64_t ldo, int64_t stride_o, int32_t n_matrices, int64_t n_rows, int64_t n_cols,
                         int32_t n_steps, const float *coef, const int *x_power, const int *a_power, const int *q_power, float eps, uint8_t *work, hipStream_t st)
{
    const UpdateLayout u = update_layout(n_matrices, n_rows, n_cols);
    double *partial = (double *)(work + u.partial_at);
    const int64_t line = 128 / sizeof(T);
    const int64_t written = whole_lines(out, ldo, sizeof(T)) && stride_o * (int64_t)sizeof(T) % 128 == 0 ? (n_cols + line - 1) / line * line : n_cols;
    update_norm_kernel<T><<<dim3((uint32_t)u.norm_blocks, (uint32_t)n_matrices), kBlock, 0, st>>>(g, ldg, stride_g, n_rows, n_cols, partial);
    if (hipError_t e = hipGetLastError()) return e;
    if (n_steps == 0) {
        const int64_t blocks = (n_rows * written + kBlock - 1) / kBlock;
        update_scale_kernel<T><<<dim3((uint32_t)(blocks < 2048 ? blocks : 2048), (uint32_t)n_matrices), kBlock, 0, st>>>(
            g, ldg, stride_g, n_rows, n_cols, partial, (int)u.norm_blocks, eps, out, ldo, stride_o, written);
        return hipGetLastError();
    }
    const int64_t lines_n = u.n / 32, lines_m = u.m / 32, pitch_n = held_pitch(u.n), pitch_m = held_pitch(u.m);
    uint8_t *x[2], *xt[2], *a = work + u.a_at, *q = work + u.q_at;
    for (int i = 0; i < 2; ++i) {
        x[i] = work + u.x_at + 2 * i * n_matrices * u.big;
        xt[i] = x[i] + n_matrices * u.big;
    }
    update_split_kernel<T><<<dim3((uint32_t)(padded(n_cols) / kPad), (uint32_t)(padded(n_rows) / kPad), (uint32_t)n_matrices), kBlock, 0, st>>>(
        g, ldg, stride_g, n_rows, n_cols, partial, (int)u.norm_blocks, eps, x_power[0], u.flip ? xt[0] : x[0], u.flip ? x[0] : xt[0],
        u.flip ? pitch_n : pitch_m, u.flip ? pitch_m : pitch_n, u.big);
    if (hipError_t e = hipGetLastError()) return e;
    for (int32_t s = 0; s < n_steps; ++s) {
        const int now = s % 2;
        const float *abc = coef + 3 * s;
        ProductArgs gram{};
        gram.p = gram.q = x[now];
        gram.rows = gram.cols = u.n;
        gram.lines = lines_m;
        gram.pitch = pitch_m;
        gram.same = gram.other = a;
        gram.pitch_same = gram.pitch_other = pitch_n;
        gram.bytes_p = gram.bytes_q = u.big;
        gram.bytes_d = u.small;
        gram.scale = ldexpf(1.0f, a_power[s] - 2 * x_power[s]);
        if (hipError_t e = launch_product<GRAM, float>(gram, n_matrices, st)) return e;
        ProductArgs poly = gram;
        poly.p = poly.q = a;
        poly.lines = lines_n;
        poly.pitch = pitch_n;
        poly.same = poly.other = q;
        poly.bytes_p = poly.bytes_q = u.small;
        poly.scale = ldexpf(abc[2], q_power[s] - 2 * a_power[s]);
        poly.linear = ldexpf(abc[1], q_power[s] - a_power[s]);
        poly.diagonal = ldexpf(abc[0], q_power[s]);
        if (hipError_t e = launch_product<POLY, float>(poly, n_matrices, st)) return e;
        ProductArgs step{};
        step.lines = lines_n;
        step.pitch = pitch_n;
        if (s + 1 < n_steps) {                      // X^T Q, stored both ways
            step.p = xt[now];
            step.q = q;
            step.rows = u.m;
            step.cols = u.n;
            step.same = xt[1 - now];
            step.other = x[1 - now];
            step.pitch_same = pitch_n;
            step.pitch_other = pitch_m;
            step.bytes_p = step.bytes_d = u.big;
            step.bytes_q = u.small;
            step.scale = ldexpf(1.0f, x_power[s + 1] - x_power[s] - q_power[s]);
            if (hipError_t e = launch_product<STEP, float>(step, n_matrices, st)) return e;
        } else {                                    // as it lies in out
            step.p = u.flip ? xt[now] : q;
            step.q = u.flip ? q : xt[now];
            step.rows = u.flip ? u.m : u.n;
            step.cols = u.flip ? u.n : u.m;
            step.bytes_p = u.flip ? u.big : u.small;
            step.bytes_q = u.flip ? u.small : u.big;
            step.out = out;
            step.ldo = ldo;
            step.stride_o = stride_o;
            step.out_rows = n_rows;
            step.out_cols = n_cols;
            step.written = written;
            step.scale = ldexpf(1.0f, -x_power[s] - q_power[s]);
            if (hipError_t e = launch_product<LAST, T>(step, n_matrices, st)) return e;
        }
    }
    return hipSuccess;
}

int check_sizes(int32_t n_matrices, int64_t n_rows, int64_t n_cols)
{
    if (n_matrices < 0 || n_rows < 0 || n_cols < 0) return ADAQP_EINVAL;
    return n_matrices > 65535 || n_rows >= kMostSize || n_cols >= kMostSize ? ADAQP_ESIZE : ADAQP_OK;
}

constexpr int kMostSteps = 64;

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_orthogonalize_workspace_bytes(int32_t n_matrices, int64_t n_rows, int64_t n_cols, int64_t *bytes_out)
{
    if (!bytes_out) return ADAQP_EINVAL;
    ADAQP_TRY(check_sizes(n_matrices, n_rows, n_cols));
    *bytes_out = n_matrices && n_rows && n_cols ? update_layout(n_matrices, n_rows, n_cols).bytes : 0;
    return ADAQP_OK;
}

extern "C" int adaqp_orthogonalize(const void *g_dev, int64_t ldg, int64_t stride_g, void *out_dev, int64_t ldo, int64_t stride_o,
                                   int32_t n_matrices, int64_t n_rows, int64_t n_cols, int32_t type, int32_t n_steps, const float *coef_host, float eps,
                                   void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    ADAQP_TRY(check_sizes(n_matrices, n_rows, n_cols));
    if (!valid_type(type) || n_steps < 0 || (n_steps > 0 && !coef_host) || !(eps >= 0.0f && eps <= 3.402823466e+38f)) return ADAQP_EINVAL;
    if (n_steps > kMostSteps) return ADAQP_ESIZE;
    int x_power[kMostSteps + 1], a_power[kMostSteps], q_power[kMostSteps];
    double most = 1.0;
    for (int32_t s = 0; s < n_steps; ++s) {
        double step, quadratic;
        bounds(coef_host[3 * s], coef_host[3 * s + 1], coef_host[3 * s + 2], most, &step, &quadratic);
        if (!(step <= ADAQP_ORTHOGONALIZE_MOST)) return ADAQP_EINVAL;
        x_power[s] = power_for(most);
        a_power[s] = power_for(most * most);
        q_power[s] = power_for(quadratic);
        x_power[s + 1] = power_for(step);
        most = fmax(step, 1e-6);
    }
    if (n_matrices == 0 || n_rows == 0 || n_cols == 0) return ADAQP_OK;
    const int64_t bytes = element_bytes(type);
    if (!g_dev || !out_dev || ldg < n_cols || ldo < n_cols || !aligned_to(g_dev, bytes) || !aligned_to(out_dev, bytes)) return ADAQP_EINVAL;
    if (n_matrices > 1 && (stride_g < n_rows * ldg || stride_o < n_rows * ldo)) return ADAQP_EINVAL;
    if (g_dev == out_dev && (ldg != ldo || (n_matrices > 1 && stride_g != stride_o))) return ADAQP_EINVAL;
    const UpdateLayout u = update_layout(n_matrices, n_rows, n_cols);
    if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
    if (workspace_bytes < u.bytes) return ADAQP_ESIZE;
    if (type == ADAQP_F32)
        ADAQP_HIP_TRY((orthogonalize<float>((const float *)g_dev, ldg, stride_g, (float *)out_dev, ldo, stride_o, n_matrices, n_rows, n_cols, n_steps, coef_host,
                                            x_power, a_power, q_power, eps, (uint8_t *)workspace_dev, (hipStream_t)stream)));
    else
        ADAQP_HIP_TRY((orthogonalize<__bf16>((const __bf16 *)g_dev, ldg, stride_g, (__bf16 *)out_dev, ldo, stride_o, n_matrices, n_rows, n_cols, n_steps,
                                             coef_host, x_power, a_power, q_power, eps, (uint8_t *)workspace_dev, (hipStream_t)stream)));
    return ADAQP_OK;
}
