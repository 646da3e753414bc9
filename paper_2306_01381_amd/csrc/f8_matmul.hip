// Products of 8-bit matrices on the matrix cores (adaqp_train.h): out = a b^T, both operands rows of k columns.
//
// gfx950's scaled products take e4m3 codes and a power of two for 32 of them; here 128 share one, so that the lanes of a row bring the same byte, and which of a row's columns a lane
// brings does not matter as long as it is the same in both operands.  But they add up the products of eight columns to 14 bits of the largest before they go on in fp32: what is
// below 2^-13 of it is cut off (found with two products of 2^16 and 2^t: t = 3 arrives, t = 2 does not, 16 x 16 and unscaled instructions the same).  That is 3e-5 of a typical result: nothing beside
// the 2^-9 of a bf16 output, for which they are taken, but 500 roundings of an fp32 one.  For those, and where time is not the matrix cores', codes become bf16 in the
// registers, with their power of two, which is exact, and the products are bf16's, exact in fp32, at half the rate.
//
// A workgroup of four waves takes a tile of BM x BN outputs, a quarter each wave, and walks k in steps of 64 columns, half a line
// of 128 bytes of a row.  Up to STAGES steps' codes are on their way from memory straight into the LDS; a step's operands are read from there into registers while the step before is multiplied.
//
// Where the tiles are few, k is split over workgroups; the parts' sums, fp32, are added in order by a second kernel.  With at most 32 rows nothing is used
// twice but those: a workgroup takes 32 columns of out, its eight waves share the lines of k and read them into registers.
//
// What bounds it: large products the matrix cores, power and waits.  8192 x 8192 x 4096, bf16 out, takes 227 to 254 us (2.2 to 2.4 PFLOP/s; zeros, which draw less, 182); the matrix cores are busy in 54 % of the cycles, at a clock that falls
// to 1.9 GHz; of a tile's 57 us its first loads and its stores take 6, with the matrix cores idle.  With fp32 outputs 425 to 465 us, 1.2 to 1.3 PFLOP/s, what a library's bf16 product reaches on this card (1.2); the matrix cores are
// busy in 63 % of the cycles, the vector units, for the most part with conversions, in 31 %.  Shallow products the output: 179 000 x 256, k = 300, bf16 out, 34 us (149 MB, 4.3 TB/s).  Deep ones the operands
// and the conversions: 256 x 602, k = 58 000, fp32 out, 26 us and 5 to add up the parts.  Few rows their waits: 5 x 8192, k = 4096, 8 us (34 MB, 4.2 TB/s).
#include "f8.hpp"
#include "lines.hpp"
#include "products.hpp"

namespace adaqp {
namespace {

constexpr int kStep = kLine / 2;                    // columns, and bytes
constexpr int64_t kMostDepth = (int64_t)1 << 24;    // columns of the operands: a tile's places in them are 32-bit

typedef int f8_codes __attribute__((ext_vector_type(8)));
typedef __bf16 bf16_values __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f8_codes codes_of(const int4 (&half)[2])
{
    return f8_codes{half[0].x, half[0].y, half[0].z, half[0].w, half[1].x, half[1].y, half[1].z, half[1].w};
}

// Half of 16 codes in units of the block's power of two.  The conversion goes by the scale's exponent; 255 gives NaN.
__device__ __forceinline__ bf16_values values_of(const int4 &codes, int half, int byte)
{
    const float scale = __builtin_bit_cast(float, byte << 23);
    const uint32_t w[2] = {(uint32_t)(half ? codes.z : codes.x), (uint32_t)(half ? codes.w : codes.y)};
    bf16_values v;
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const auto pair = k % 4 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k / 4], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k / 4], scale, false);
        v[k] = pair[0];
        v[k + 1] = pair[1];
    }
    return v;
}

struct F8MulArgs {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    void *out;
    int64_t m, n, ldo;
    int64_t written;                                // columns of out: n, or its whole lines
    int64_t pitch;                                  // of a row of codes, both operands
    int64_t scale_pitch_a, scale_pitch_b;
    int64_t steps, steps_per_split, splits;         // steps_per_split is even
    int64_t tiles_m, tiles_n;
    bool whole_vectors;                             // rows of out begin and end on 16 bytes
};

constexpr int kScalePlaces = kWave * 4;             // a load's

template <int BM, int BN>
struct alignas(32) F8Stage {
    uint8_t a[BM * kStep], b[BN * kStep];
    uint8_t scale_a[kScalePlaces], scale_b[kScalePlaces];
};

// Of half lines the four 16-byte parts lie at (part ^ row / 4 mod 4): four rows fill the banks.
__device__ __forceinline__ const uint8_t *half_part(const uint8_t *lds, int row, int part) { return lds + row * kStep + (part ^ row / 4 % 4) * 16; }

// A wave's loads of a step: the same number in every wave.  Even waves load a's scales, odd ones b's.
template <int BM, int BN>
struct F8Loads {
    static_assert(BM <= kScalePlaces && BN <= kScalePlaces, "a load of scales has them all");
    static constexpr int kA = BM / 64, kB = BN / 64, kLoads = kA + kB + 1;
    uint32_t a[kA], b[kB], scale;
    const uint8_t *from_a, *from_b, *from_scale;
    int64_t scale_stride;
    int wave;

    __device__ __forceinline__ F8Loads(const F8MulArgs &g, int64_t row0, int64_t col0, int64_t begin)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int lane = threadIdx.x % kWave;
        from_a = g.a_codes + row0 * g.pitch + begin * kStep;
        from_b = g.b_codes + col0 * g.pitch + begin * kStep;
        auto places = [&](auto &to, int rows, int64_t left) {           // 16 rows of four parts a load
            const uint32_t last = (uint32_t)min((int64_t)rows, left) - 1;
#pragma unroll
            for (int i = 0; i < rows / 64; ++i) to[i] = min((uint32_t)(wave * (rows / 4) + i * 16 + lane / 4), last) * (uint32_t)g.pitch + (lane % 4 ^ lane / 16) * 16;
        };
        places(a, BM, g.m - row0);
        places(b, BN, g.n - col0);
        const bool of_b = wave % 2;
        scale_stride = of_b ? g.scale_pitch_b : g.scale_pitch_a;
        const int64_t first = of_b ? col0 : row0;
        from_scale = (of_b ? g.b_scales : g.a_scales) + begin / 2 * scale_stride + first;
        scale = (uint32_t)min((int64_t)lane * 4, scale_stride - first - 4);
    }

    __device__ __forceinline__ void load(int i, int step, const F8Stage<BM, BN> &s) const
    {
        if (i < kA)           load_to_lds_16(from_a + (int64_t)step * kStep, a[i], __builtin_amdgcn_readfirstlane(lds_offset(s.a) + (wave * (BM / 4) + i * 16) * kStep));
        else if (i < kA + kB) load_to_lds_16(from_b + (int64_t)step * kStep, b[i - kA], __builtin_amdgcn_readfirstlane(lds_offset(s.b) + (wave * (BN / 4) + (i - kA) * 16) * kStep));
        else                  load_to_lds_4(from_scale + step / 2 * scale_stride, scale, __builtin_amdgcn_readfirstlane(lds_offset(wave % 2 ? s.scale_b : s.scale_a)));
    }
};

template <typename T, bool EXACT, int BM, int BN, int STAGES>
__global__ __launch_bounds__(kBlock) void f8_matmul_kernel(F8MulArgs g)
{
    constexpr int FM = BM / 64, FN = BN / 64;       // 32 x 32 parts of a wave
    __shared__ F8Stage<BM, BN> stage[STAGES];
    static_assert(alignof(decltype(stage)) % alignof(vec_of<float, 16 / sizeof(T)>) == 0 && alignof(decltype(stage)) % alignof(int4) == 0, "operands and sheets are read in vectors");
    static_assert(sizeof(stage) >= kWavesPerBlock * 32 * sheet_pitch(FN) * 4, "the sheets lie where the operands were");
    static_assert(STAGES >= 2, "a step is read while the one before is multiplied");
    using Loads = F8Loads<BM, BN>;
    const TilePlace place = tile_place(workgroup(), workgroups(), (uint32_t)g.tiles_m, (uint32_t)g.tiles_n, (uint32_t)g.splits);
    if (place.part < 0) return;
    const int64_t row0 = place.row * BM, col0 = place.col * BN;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int wm = wave / 2 * (BM / 2), wn = wave % 2 * (BN / 2);
    const int64_t begin = place.part * g.steps_per_split;
    const int steps = (int)min(g.steps_per_split, g.steps - begin);
    const Loads loads(g, row0, col0, begin);

    tile_sums sums[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) sums[i][j][q] = 0.0f;

    // A step's operands and scales.
    struct Step { int4 a[FM][2], b[FN][2]; int sa[FM], sb[FN]; } part[2];
    // Read `i` of a step, in the order in which products need them.
    constexpr int kReads = FM + FN, kProducts = FM * FN, kReadsAtOnce = (kReads + kProducts - 1) / kProducts;
    auto read = [&](const F8Stage<BM, BN> &s, int i, Step &to) {
        if (i >= 1 && i <= FN) {
            const int j = i - 1, row = wn + j * 32 + r;
#pragma unroll
            for (int p = 0; p < 2; ++p) to.b[j][p] = *reinterpret_cast<const int4 *>(half_part(s.b, row, p * 2 + h));
            to.sb[j] = s.scale_b[row];
        } else {
            const int j = i == 0 ? 0 : i - FN, row = wm + j * 32 + r;
#pragma unroll
            for (int p = 0; p < 2; ++p) to.a[j][p] = *reinterpret_cast<const int4 *>(half_part(s.a, row, p * 2 + h));
            to.sa[j] = s.scale_a[row];
        }
    };
    // The operands of a quarter of a step, as bf16.
    struct Quarter { bf16_values a[FM], b[FN]; } quarter[2];
    auto convert = [&](const Step &f, int q, int i, Quarter &to) {
        if (i >= 1 && i <= FN) to.b[i - 1] = values_of(f.b[i - 1][q / 2], q % 2, f.sb[i - 1]);
        else                   to.a[i == 0 ? 0 : i - FN] = values_of(f.a[i == 0 ? 0 : i - FN][q / 2], q % 2, f.sa[i == 0 ? 0 : i - FN]);
    };

    // Up to STAGES steps are under way.  Behind the barrier the next step is in the LDS and this one's buffer free: its operands are in registers.  Reads of the one and loads into the other
    // lie one by one between the products.  No branches: across one the compiler would take products to the other side of the barrier.
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < steps)
#pragma unroll
            for (int l = 0; l < Loads::kLoads; ++l) loads.load(l, s, stage[s]);
    if (steps >= STAGES) arrived<Loads::kLoads * (STAGES - 1)>();
    else                 arrived<0>();
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(stage[0], i, part[0]);
    if (EXACT)
#pragma unroll
        for (int i = 0; i < kReads; ++i) convert(part[0], 0, i, quarter[0]);
    int now = 0;
    // `more`: step + STAGES exists, and with it STAGES - 1 steps' loads are under way behind this step
    auto one = [&](int step, const Step &f, Step &to, auto more) {
        constexpr bool kMore = decltype(more)::value;
        const F8Stage<BM, BN> &s = stage[now];
        now = now + 1 == STAGES ? 0 : now + 1;
        const F8Stage<BM, BN> &next = stage[now];
        arrived<kMore ? Loads::kLoads * (STAGES - 2) : 0>();
        __builtin_amdgcn_sched_barrier(0);
        // what is done behind product p of the first kProducts
        auto between = [&](int p) {
#pragma unroll
            for (int i = p * kReadsAtOnce; i < (p + 1) * kReadsAtOnce && i < kReads; ++i) read(next, i, to);
            if constexpr (kMore) {
#pragma unroll
                for (int l = p * Loads::kLoads / kProducts; l < (p + 1) * Loads::kLoads / kProducts; ++l) loads.load(l, step + STAGES, s);
            }
        };
        if constexpr (EXACT) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const Quarter &now_of = quarter[q % 2];
                Quarter &next_of = quarter[(q + 1) % 2];
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) {
                        const int p = i * FN + j;
                        sums[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now_of.a[i], now_of.b[j], sums[i][j], 0, 0, 0);
                        if (q == 0) between(p);
#pragma unroll
                        for (int c = p * kReadsAtOnce; c < (p + 1) * kReadsAtOnce && c < kReads; ++c) convert(q < 3 ? f : to, (q + 1) % 4, c, next_of);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    sums[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes_of(f.a[i]), codes_of(f.b[j]), sums[i][j], 0, 0, 0, f.sa[i], 0, f.sb[j]);
                    between(i * FN + j);
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
    };
    int step = 0;
    for (; step + 1 + STAGES < steps; step += 2) {
        one(step, part[0], part[1], std::true_type());
        one(step + 1, part[1], part[0], std::true_type());
    }
    // the rest: at most STAGES + 1 steps, of which the first may still load one
    if (step + STAGES < steps) {
        one(step, part[0], part[1], std::true_type());
        ++step;
        part[0] = part[1];
    }
    for (; step + 1 < steps; step += 2) {
        one(step, part[0], part[1], std::false_type());
        one(step + 1, part[1], part[0], std::false_type());
    }
    if (step < steps) one(step, part[0], part[1], std::false_type());
    arrived<0>();                                   // what was read behind the last step, too: the sheets lie there
    store_tile<T, FM, FN>(g, sums, place.part, row0 + wm, col0 + wn, reinterpret_cast<float *>(stage));
}

constexpr int kFewRows = 32, kFewWaves = 8;

// At most 32 rows: 32 columns of out, wave w takes the lines w, w + 8, ... of its part of k.
template <typename T>
__global__ __launch_bounds__(kFewWaves * kWave) void f8_few_rows_kernel(F8MulArgs g)
{
    constexpr int kLines = 2;                       // under way
    __shared__ float parts[kFewWaves][kFewRows * 32];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int64_t col0 = (int64_t)workgroup() * 32;
    const int64_t row_a = min((int64_t)r, g.m - 1), row_b = min(col0 + r, g.n - 1);
    const int64_t begin = blockIdx.z * g.steps_per_split / 2, end = min(begin + g.steps_per_split / 2, (g.steps + 1) / 2);        // lines
    tile_sums sums;
#pragma unroll
    for (int q = 0; q < 16; ++q) sums[q] = 0.0f;
    for (int64_t line0 = begin + wave; line0 < end; line0 += kFewWaves * kLines) {
        int4 a[kLines][4], b[kLines][4];
        int sa[kLines], sb[kLines];
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
            const int64_t line = min(line0 + i * kFewWaves, end - 1);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                a[i][q] = *reinterpret_cast<const int4 *>(g.a_codes + row_a * g.pitch + line * kLine + (q * 2 + h) * 16);
                b[i][q] = *reinterpret_cast<const int4 *>(g.b_codes + row_b * g.pitch + line * kLine + (q * 2 + h) * 16);
            }
            sa[i] = g.a_scales[line * g.scale_pitch_a + row_a];
            sb[i] = g.b_scales[line * g.scale_pitch_b + row_b];
        }
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
            if (line0 + i * kFewWaves >= end) break;
#pragma unroll
            for (int q = 0; q < 8; ++q)
                sums = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values_of(a[i][q / 2], q % 2, sa[i]), values_of(b[i][q / 2], q % 2, sb[i]), sums, 0, 0, 0);
        }
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) parts[wave][(q / 4 * 8 + h * 4 + q % 4) * 32 + r] = sums[q];
    __syncthreads();
    for (int at = threadIdx.x; at < (int)g.m * 32; at += kFewWaves * kWave) {
        const int64_t row = at / 32, col = col0 + at % 32;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) sum += parts[w][at];
        if (col < g.written) ((T *)g.out)[(blockIdx.z * g.m + row) * g.ldo + col] = col < g.n ? (T)sum : (T)0.0f;
    }
}

enum F8Tile { F8_FEW_ROWS, F8_64_64, F8_128_64, F8_128_128, F8_256_256 };

struct F8Shape {
    F8Tile tile;
    int64_t tiles_m, tiles_n, steps, splits, steps_per_split, bytes;
};

// us of tiles of 256 x 256 (four steps under way), 128 x 128 (three; with four, and two workgroups a CU instead of three, 40 for 33 in the first line) and 128 x 64 (three), bf16 outputs:
//     179 000 x 256 x 300    46   33   38       8192 x 8192 x 256    52   38   44       8192 x 8192 x 640    72   66   85
//     8192 x 8192 x 1024     87   98  130       4096^3               63   88  124       3584 x 3584 x 4096   52   75   97
//     2048 x 4096 x 4096     48   45   63       1024 x 4096 x 4096   44   25   32       2304^3               30   25   27
// A large tile takes 0.72 of the time of its four middle ones where the CUs are full, and a round of large tiles that does not fill them takes as long: 256 x 256 where its rounds so counted are fewer.
// k is split where tiles of 64 x 64 leave half of the CUs idle, or a quarter with 8192 columns and more, so that middle tiles fill the CUs once (256 x 602, k = 58 000, 10 tiles: 16, 24, 32, 48 parts 24, 20, 24, 21 us without the
// joining), in parts of at least 16 steps; shorter ones in tiles of 64 x 64 (512 x 512, k = 8192, 13 us with the joining, middle tiles 18).
F8Shape f8_shape(int64_t m, int64_t n, int64_t k)
{
    F8Shape s{};
    auto tiles = [&](F8Tile t, int64_t rows, int64_t cols) {
        s.tile = t;
        s.tiles_m = (m + rows - 1) / rows;
        s.tiles_n = (n + cols - 1) / cols;
        return s.tiles_m * s.tiles_n;
    };
    s.steps = (k + kStep - 1) / kStep;
    s.splits = 1;
    s.steps_per_split = (s.steps + 1) / 2 * 2;
    auto split = [&](int64_t splits) {
        if (splits < 2) return;
        s.steps_per_split = ((s.steps + splits - 1) / splits + 1) / 2 * 2;
        s.splits = (s.steps + s.steps_per_split - 1) / s.steps_per_split;
        s.bytes = s.splits > 1 ? (s.splits * m * n * 4 + 255) / 256 * 256 : 0;
    };
    if (m == 0 || n == 0) return s;
    if (m <= kFewRows) {
        const int64_t blocks = tiles(F8_FEW_ROWS, kFewRows, 32), most = s.steps / (4 * kFewWaves);
        split(256 / blocks < most ? 256 / blocks : most);
        return s;
    }
    auto padded = [&](int64_t rows, int64_t cols) { return (double)((m + rows - 1) / rows * rows) * (double)((n + cols - 1) / cols * cols); };
    auto fits = [&](int64_t rows, int64_t cols) { return padded(rows, cols) < 1.1 * padded(rows == 256 ? 128 : rows, cols / 2); };
    const int64_t large = tiles(F8_256_256, 256, 256), middle = tiles(F8_128_128, 128, 128);
    if (s.steps >= 14 && fits(256, 256) && (large + 255) / 256 * 256 * 4 * 18 < middle * 25) {
        tiles(F8_256_256, 256, 256);
        return s;
    }
    if (fits(128, 128) && tiles(F8_128_128, 128, 128) >= 256) return s;
    if (tiles(F8_128_64, 128, 64) >= 256) return s;
    const int64_t small = tiles(F8_64_64, 64, 64);
    if (s.steps < (small >= 128 ? 128 : 32)) return s;
    const double least = 1.25 * padded(64, 64);
    const F8Tile tile = padded(128, 128) <= least ? F8_128_128 : padded(128, 64) <= least ? F8_128_64 : F8_64_64;
    const int64_t blocks = tile == F8_128_128 ? tiles(tile, 128, 128) : tile == F8_128_64 ? tiles(tile, 128, 64) : small;
    const int64_t wanted = (tile == F8_128_128 ? 256 : 512) / blocks;
    if (tile == F8_64_64 || s.steps < wanted * 16) {
        tiles(F8_64_64, 64, 64);
        split(480 / small < s.steps / 16 ? 480 / small : s.steps / 16);
    } else split(wanted);
    return s;
}

template <typename T, bool EXACT>
void launch_tiles(const F8MulArgs &g, const F8Shape &s, hipStream_t st)
{
    const dim3 blocks = grid_of(tile_blocks(s.tiles_m * s.tiles_n, s.splits), kBlock);
    switch (s.tile) {
        case F8_FEW_ROWS: f8_few_rows_kernel<T><<<grid_of((g.written + 31) / 32, kFewWaves * kWave, (uint32_t)s.splits), kFewWaves * kWave, 0, st>>>(g); break;
        case F8_64_64:    f8_matmul_kernel<T, EXACT, 64, 64, 4><<<blocks, kBlock, 0, st>>>(g); break;
        case F8_128_64:   f8_matmul_kernel<T, EXACT, 128, 64, 3><<<blocks, kBlock, 0, st>>>(g); break;
        case F8_128_128:  f8_matmul_kernel<T, EXACT, 128, 128, 3><<<blocks, kBlock, 0, st>>>(g); break;
        case F8_256_256:  f8_matmul_kernel<T, EXACT, 256, 256, 4><<<blocks, kBlock, 0, st>>>(g); break;
    }
}

int check_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return ADAQP_EINVAL;
    return m >= kF8Most || n >= kF8Most || k > kMostDepth || (m + 63) / 64 * ((n + 63) / 64) >= 0x3FFFFFFF ? ADAQP_ESIZE : ADAQP_OK;
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_f8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t *bytes_out)
{
    if (!bytes_out) return ADAQP_EINVAL;
    ADAQP_TRY(check_sizes(m, n, k));
    *bytes_out = f8_shape(m, n, k).bytes;
    return ADAQP_OK;
}

extern "C" int adaqp_f8_matmul(const uint8_t *a_codes_dev, const uint8_t *a_scales_dev, int64_t m,
                               const uint8_t *b_codes_dev, const uint8_t *b_scales_dev, int64_t n, int64_t k,
                               void *out_dev, int64_t ldo, int32_t type, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    ADAQP_TRY(check_sizes(m, n, k));
    if (!valid_type(type)) return ADAQP_EINVAL;
    if (m == 0 || n == 0) return ADAQP_OK;
    if (!out_dev || ldo < n || !aligned_to(out_dev, element_bytes(type))) return ADAQP_EINVAL;
    if (k > 0 && (!valid_f8(a_codes_dev, a_scales_dev) || !valid_f8(b_codes_dev, b_scales_dev))) return ADAQP_EINVAL;
    const F8Shape s = f8_shape(m, n, k);
    if (s.splits > 1) {
        if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
        if (workspace_bytes < s.bytes) return ADAQP_ESIZE;
    }
    F8MulArgs g{a_codes_dev, a_scales_dev, b_codes_dev, b_scales_dev, out_dev, m, n, ldo, 0, f8_chunks(k) * kF8Block, f8_scale_pitch(m), f8_scale_pitch(n),
                s.steps, s.steps_per_split, s.splits, s.tiles_m, s.tiles_n, false};
    const hipStream_t st = (hipStream_t)stream;
    const int64_t line = 128 / element_bytes(type);
    const int64_t written = whole_lines(out_dev, ldo, element_bytes(type)) ? (n + line - 1) / line * line : n;
    const int64_t vector = 16 / element_bytes(type);
    g.written = s.splits > 1 ? n : written;
    g.whole_vectors = aligned_to(out_dev, 16) && ldo % vector == 0 && written % vector == 0;
    if (s.splits > 1) {
        g.out = workspace_dev;
        g.ldo = n;
        g.whole_vectors = n % 4 == 0;
        if (type == ADAQP_F32) launch_tiles<float, true>(g, s, st);
        else                   launch_tiles<float, false>(g, s, st);
        ADAQP_HIP_TRY(hipGetLastError());
        const int64_t rows = (m + kWavesPerBlock - 1) / kWavesPerBlock;
        const dim3 grid((uint32_t)((written + kWave - 1) / kWave), (uint32_t)(rows < 65535 ? rows : 65535));
        if (type == ADAQP_F32) join_parts_kernel<float><<<grid, kBlock, 0, st>>>((const float *)workspace_dev, (int)s.splits, m, n, written, (float *)out_dev, ldo);
        else                   join_parts_kernel<__bf16><<<grid, kBlock, 0, st>>>((const float *)workspace_dev, (int)s.splits, m, n, written, (__bf16 *)out_dev, ldo);
    } else if (type == ADAQP_F32) launch_tiles<float, true>(g, s, st);
    else                          launch_tiles<__bf16, false>(g, s, st);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}
