// Orthogonalised updates of matrices that fit a CU's LDS with their products (adaqp_dense.h): one workgroup each does all steps.
//
// The same arithmetic as in orthogonalize.hip: operands as two fp16 numbers, three of the four partial products, fp32 sums.  Launched product by product a matrix of
// 64 x 64 waits 17 times about 4 us for products that take a tenth of that (66 us); here its five steps need no memory but their input and output (32 us; 41 x 256 41
// against 75, 16 x 16 25).  What is left are the waits within a step, for barriers and the LDS.  X is held once, by
// rows of lines (32 hi, 32 lo); where a product runs along its columns, lanes gather them.  A row's end is 16 bytes apart from the next one's begin modulo 256,
// so that 16 rows read at one place use all banks.
#include <math.h>

#include "orthogonalize.hpp"

namespace adaqp {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kLds = 156 * 1024;
constexpr int kLineBytes = 128;

__host__ __device__ constexpr int pitch_of(int cols) { return cols * 4 + 16; }

// Sizes of the smaller side that the kernel is made for, 32-column tiles NT of them, and the larger side's tiles a wave may have.
constexpr int most_tiles(int nt) { return 4 / nt; }

struct SmallPlan { int nt; int64_t m; };            // m: the larger side, a multiple of 32

SmallPlan small_plan(int64_t n_rows, int64_t n_cols)
{
    const int64_t n = n_rows < n_cols ? n_rows : n_cols, m = ((n_rows < n_cols ? n_cols : n_rows) + 31) / 32 * 32;
    SmallPlan p{n <= 32 ? 1 : n <= 64 ? 2 : 0, m};
    if (p.nt == 0 || m / 32 > kWaves * most_tiles(p.nt)) return SmallPlan{0, m};
    const int64_t sums = (kWaves / (p.nt * p.nt) - 1) * p.nt * p.nt * 4096, poly = p.nt * 32 * pitch_of(p.nt * 32);
    if (p.nt * 32 * pitch_of((int)m) + poly + (sums > poly ? sums : poly) > kLds) return SmallPlan{0, m};
    return p;
}

// The three partial products of 16 columns.
__device__ __forceinline__ sums16 multiply(half8 ah, half8 al, half8 bh, half8 bl, sums16 sums)
{
    sums = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, sums, 0, 0, 0);
    sums = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, sums, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, sums, 0, 0, 0);
}

__device__ __forceinline__ sums16 no_sums()
{
    sums16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.0f;
    return s;
}

// Row of sum e of a 32 x 32 tile; its column is lane % 32.
__device__ __forceinline__ int sum_row(int e) { return e / 4 * 8 + threadIdx.x % kWave / 32 * 4 + e % 4; }

__device__ __forceinline__ void put_held(uint8_t *rows, int pitch, int row, int col, float v)
{
    _Float16 hi, lo;
    split(v, hi, lo);
    uint8_t *to = rows + row * pitch + col / 32 * kLineBytes + col % 32 * 2;
    *reinterpret_cast<_Float16 *>(to) = hi;
    *reinterpret_cast<_Float16 *>(to + 64) = lo;
}

__device__ __forceinline__ float get_held(const uint8_t *rows, int pitch, int row, int col)
{
    const uint8_t *from = rows + row * pitch + col / 32 * kLineBytes + col % 32 * 2;
    return (float)*reinterpret_cast<const _Float16 *>(from) + (float)*reinterpret_cast<const _Float16 *>(from + 64);
}

// D = R R^T for held rows R of `lines` lines; finish(row, col, sum) with each of D's elements.  `sums`: room for all but the first part of each tile.
template <int NT, typename F>
__device__ __forceinline__ void square(const uint8_t *rows, int pitch, int lines, float *sums, F finish)
{
    constexpr int kTiles = NT * NT, kParts = kWaves / kTiles;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int tile = wave % kTiles, part = wave / kTiles;
    const uint8_t *a = rows + (tile / NT * 32 + r) * pitch + h * 16, *b = rows + (tile % NT * 32 + r) * pitch + h * 16;
    sums16 s = no_sums();
    for (int line = part; line < lines; line += kParts) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = line * kLineBytes + k * 32;
            s = multiply(*reinterpret_cast<const half8 *>(a + at), *reinterpret_cast<const half8 *>(a + at + 64), *reinterpret_cast<const half8 *>(b + at),
                         *reinterpret_cast<const half8 *>(b + at + 64), s);
        }
    }
    if (part > 0)
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[((part - 1) * kTiles + tile) * 1024 + e * kWave + lane] = s[e];
    __syncthreads();
    if (part == 0)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float v = s[e];
#pragma unroll
            for (int q = 0; q < kParts - 1; ++q) v += sums[(q * kTiles + tile) * 1024 + e * kWave + lane];
            finish(tile / NT * 32 + sum_row(e), tile % NT * 32 + r, v);
        }
    __syncthreads();
}

template <typename T, int NT>
__global__ __launch_bounds__(kThreads) void small_update_kernel(SmallUpdate u, int m)
{
    constexpr int kN = NT * 32, kOwn = most_tiles(NT), kPolyPitch = pitch_of(kN);
    __shared__ __align__(16) uint8_t lds[kLds];
    __shared__ double squares[kWaves];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int pitch = pitch_of(m), lines = m / 32;
    uint8_t *x = lds, *a = lds + kN * pitch, *q = a + kN * kPolyPitch;  // the parts' sums lie where Q will
    const T *g = (const T *)u.g + blockIdx.x * u.stride_g;
    T *out = (T *)u.out + blockIdx.x * u.stride_o;
    const bool flip = u.n_rows > u.n_cols;

    // G in fp32 to where X will be, several elements of a thread under way; then row by row, each a wave's, what X is of it
    constexpr int kAtOnce = 12;
    const int total = u.n_rows * u.n_cols, stride_row = kThreads / u.n_cols, stride_col = kThreads % u.n_cols;
    int row = threadIdx.x / u.n_cols, col = threadIdx.x % u.n_cols;
    double sum = 0.0;
    for (int first = threadIdx.x; first < total; first += kThreads * kAtOnce) {
        float v[kAtOnce];
        int to[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const bool there = first + k * kThreads < total;
            v[k] = (float)g[(there ? row : 0) * u.ldg + (there ? col : 0)];
            to[k] = there ? (flip ? col * pitch + row * 4 : row * pitch + col * 4) : -1;
            row += stride_row;
            col += stride_col;
            if (col >= u.n_cols) {
                col -= u.n_cols;
                ++row;
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (to[k] >= 0) {
                *reinterpret_cast<float *>(x + to[k]) = v[k];
                sum = fma((double)v[k], (double)v[k], sum);
            }
    }
    for (int other = 1; other < kWave; other *= 2) sum += __shfl_xor(sum, other);
    if (lane == 0) squares[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += squares[w];
    const double scale = ldexp(one_over_norm(sum, u.eps), u.power);
    const int n_there = flip ? u.n_cols : u.n_rows, m_there = flip ? u.n_rows : u.n_cols;
    for (int i = wave; i < kN; i += kWaves) {
        constexpr int kMost = kOwn * kWaves * 32 / kWave;
        float v[kMost];
#pragma unroll
        for (int k = 0; k < kMost; ++k) v[k] = k * kWave < m && i < n_there && k * kWave + lane < m_there ? *reinterpret_cast<const float *>(x + i * pitch + (k * kWave + lane) * 4) : 0.0f;
        // the row is written over as another type: without this the compiler may move a lane's writes before another lane's reads
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int k = 0; k < kMost; ++k)
            if (k * kWave + lane < m) put_held(x, pitch, i, k * kWave + lane, i < n_there && k * kWave + lane < m_there ? (float)((double)v[k] * scale) : 0.0f);
    }
    __syncthreads();

    for (int step = 0; step < u.n_steps; ++step) {
        square<NT>(x, pitch, lines, (float *)q, [&](int row, int col, float v) { put_held(a, kPolyPitch, row, col, v * u.of_gram[step]); });
        // Q goes where the parts' sums were: those of this product are read before any of it is written
        constexpr int kTiles = NT * NT;
        sums16 poly = no_sums();
        const int tile = wave % kTiles;
        if (wave < kTiles) {
#pragma unroll
            for (int at = 0; at < NT * 2; ++at) {
                const int place = at / 2 * kLineBytes + at % 2 * 32 + h * 16;
                const uint8_t *left = a + (tile / NT * 32 + r) * kPolyPitch + place, *right = a + (tile % NT * 32 + r) * kPolyPitch + place;
                poly = multiply(*reinterpret_cast<const half8 *>(left), *reinterpret_cast<const half8 *>(left + 64), *reinterpret_cast<const half8 *>(right),
                                *reinterpret_cast<const half8 *>(right + 64), poly);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = tile / NT * 32 + sum_row(e), col = tile % NT * 32 + r;
                put_held(q, kPolyPitch, row, col,
                         fmaf(u.linear[step], get_held(a, kPolyPitch, row, col), poly[e] * u.of_poly[step]) + (row == col ? u.diagonal[step] : 0.0f));
            }
        }
        __syncthreads();
        // X <- Q X: a wave's 32-column tiles are w, w + 8, ...
        sums16 next[kOwn][NT];
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            const int t = wave + o * kWaves;
#pragma unroll
            for (int i = 0; i < NT; ++i) next[o][i] = no_sums();
            if (t >= lines) continue;
#pragma unroll
            for (int at = 0; at < NT * 2; ++at) {
                half8 bh, bl;                       // column r of tile t, rows 16 at + 8 h on
                const uint8_t *from = x + (at * 16 + h * 8) * pitch + t * kLineBytes + r * 2;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    bh[k] = *reinterpret_cast<const _Float16 *>(from + k * pitch);
                    bl[k] = *reinterpret_cast<const _Float16 *>(from + k * pitch + 64);
                }
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const uint8_t *left = q + (i * 32 + r) * kPolyPitch + at / 2 * kLineBytes + at % 2 * 32 + h * 16;
                    next[o][i] = multiply(*reinterpret_cast<const half8 *>(left), *reinterpret_cast<const half8 *>(left + 64), bh, bl, next[o][i]);
                }
            }
        }
        __syncthreads();                            // X has been read
        const bool last = step + 1 == u.n_steps;
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            const int t = wave + o * kWaves;
            if (t >= lines) continue;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float v = next[o][i][e] * u.of_step[step];
                    if (last) *reinterpret_cast<float *>(x + (i * 32 + sum_row(e)) * pitch + (t * 32 + r) * 4) = v;
                    else      put_held(x, pitch, i * 32 + sum_row(e), t * 32 + r, v);
                }
        }
        __syncthreads();
    }
    for (row = wave; row < u.n_rows; row += kWaves)
        for (col = lane; col < u.written; col += kWave) {
            const int i = flip ? col : row, j = flip ? row : col;
            out[row * u.ldo + col] = col < u.n_cols ? (T)*reinterpret_cast<const float *>(x + i * pitch + j * 4) : (T)0.0f;
        }
}

}  // namespace

bool small_update_fits(int64_t n_rows, int64_t n_cols) { return small_plan(n_rows, n_cols).nt != 0; }

hipError_t launch_small_update(const SmallUpdate &u, int32_t n_matrices, int32_t type, hipStream_t st)
{
    const SmallPlan p = small_plan(u.n_rows, u.n_cols);
    if (type == ADAQP_F32) {
        if (p.nt == 1) small_update_kernel<float, 1><<<(uint32_t)n_matrices, kThreads, 0, st>>>(u, (int)p.m);
        else           small_update_kernel<float, 2><<<(uint32_t)n_matrices, kThreads, 0, st>>>(u, (int)p.m);
    } else {
        if (p.nt == 1) small_update_kernel<__bf16, 1><<<(uint32_t)n_matrices, kThreads, 0, st>>>(u, (int)p.m);
        else           small_update_kernel<__bf16, 2><<<(uint32_t)n_matrices, kThreads, 0, st>>>(u, (int)p.m);
    }
    return hipGetLastError();
}

}  // namespace adaqp
