// Products of MX matrices on the matrix cores (adaqp_dense.h): out = a b^T, both operands rows of k columns.
//
// gfx950's scaled products take 4-bit codes and a power of two for 32 of them as they lie in memory: nothing is unpacked.  A workgroup of four waves
// takes a tile of BM x BN outputs, a quarter each wave, and walks k in steps of 256 columns, a line of 128 bytes of a row.  The next step's codes and
// scales go from memory straight into the LDS while the current one is multiplied.
//
// Where the tiles are few, k is split over workgroups; the parts' sums, fp32, are added in order by a second kernel.  With at most 32 rows nothing is used
// twice but those: a workgroup takes 32 columns of out, its eight waves share the lines of k and read them into registers, as many at a time as they can.
//
// What bounds it: large products the waits of a tile that has a CU to itself.  8192 x 8192 x 4096, fp32 out, takes 171 to 190 us with the clock that a run finds (about 3 PFLOP/s).  Of a tile's
// 43 us its loop takes 33, at 73 % of what the matrix cores reach on random codes from registers alone (6.1 PFLOP/s): a wave has a SIMD to itself and nothing to fill its waits with.
// Its first loads take 3 and its stores 7, with the matrix cores idle.  Power is a fifth: zeros, which draw less, take 141 us (61 at their rate from registers, 9.0 PFLOP/s).
// Shallow products the output: 58 000 x 256, k = 602, 20 us (79 MB, 3.9 TB/s).  Deep ones the operands: 256 x 300, k = 196 000, 29 us and 5 to add up the parts; of 54 MB each line is
// loaded by the 4 or 5 tiles of 64 x 64 that need it.  Few rows their waits: 5 x 8192, k = 4096 and bf16 out, 7 us (17.9 MB, 2.7 TB/s).
#include "lines.hpp"
#include "mx4.hpp"
#include "products.hpp"

namespace adaqp {
namespace {

constexpr int kStepChunks = 2;                      // scale words
constexpr int64_t kMostDepth = (int64_t)1 << 25;    // columns of the operands: a tile's places in them are 32-bit

typedef int mx_codes __attribute__((ext_vector_type(8)));       // of which 4-bit codes fill the first half

struct MulArgs {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    void *out;
    int64_t m, n, ldo;
    int64_t written;                                // columns of out: n, or its whole lines
    int64_t pitch;                                  // of a row of codes, both operands
    int64_t chunks;                                 // scale words of a row
    int64_t steps, steps_per_split, splits;
    int64_t tiles_m, tiles_n;
    bool whole_vectors;                             // rows of out begin and end on 16 bytes
};

template <int BM, int BN>
struct alignas(32) Stage {
    uint8_t a[BM * kLine], b[BN * kLine];
    uint32_t scales[kStepChunks * (BM + BN)];       // [2][BM], then [2][BN]
};

// What lanes load whose scales do not exist: 2^-127, times the other operand's too, leaves nothing of whatever codes.
__device__ const uint32_t smallest_scales = 0;

// A workgroup's loads of a step, the same number in every wave.
template <int BM, int BN>
struct StepLoads {
    static constexpr int kScaleWords = kStepChunks * (BM + BN), kScaleLoads = (kScaleWords + kBlock - 1) / kBlock;
    static constexpr int kLoads = TileLoads<BM>::kLoads + TileLoads<BN>::kLoads + kScaleLoads;
    TileLoads<BM> a;
    TileLoads<BN> b;
    const uint8_t *from_a, *from_b;
    const uint8_t *from_scale[kScaleLoads];
    int64_t scale_stride[kScaleLoads];              // from step to step
    int scale_chunk[kScaleLoads];
    uint32_t scale[kScaleLoads], to_scale[kScaleLoads];
    uint64_t missing;
    int chunks;

    // Of the words [2][BM], [2][BN] a wave's load takes 64; where they do not come out even, some are loaded twice.
    __device__ __forceinline__ StepLoads(const MulArgs &g, int64_t row0, int64_t col0) : a(row0, g.m, g.pitch), b(col0, g.n, g.pitch)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        from_a = g.a_codes + row0 * g.pitch;
        from_b = g.b_codes + col0 * g.pitch;
        chunks = (int)g.chunks;
        missing = (uint64_t)&smallest_scales;
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            int at = (i * kWavesPerBlock + wave) * kWave % kScaleWords;
            to_scale[i] = at * 4;
            const bool of_b = at >= kStepChunks * BM;
            at -= of_b ? kStepChunks * BM : 0;
            const int rows = of_b ? BN : BM;
            const int64_t n = of_b ? g.n : g.m, first = of_b ? col0 : row0;
            scale_chunk[i] = at / rows;
            scale_stride[i] = n * 4 * kStepChunks;
            from_scale[i] = (of_b ? g.b_scales : g.a_scales) + (scale_chunk[i] * n + first) * 4;
            scale[i] = min((uint32_t)(at % rows + threadIdx.x % kWave), (uint32_t)min((int64_t)rows, n - first) - 1) * 4;
        }
    }

    // Load i of a step.  The last step of an odd number of chunks has half a line, and the smallest scales for the other.
    __device__ __forceinline__ void load(int i, int step, const Stage<BM, BN> &s) const
    {
        constexpr int kA = TileLoads<BM>::kLoads, kB = TileLoads<BN>::kLoads;
        const bool half = (step + 1) * kStepChunks > chunks;
        if (i < kA)           a.template load<true>(i, from_a + (int64_t)step * kLine, TileLoads<BM>::place(s.a), half);
        else if (i < kA + kB) b.template load<true>(i - kA, from_b + (int64_t)step * kLine, TileLoads<BN>::place(s.b), half);
        else {
            i -= kA + kB;
            const bool there = step * kStepChunks + scale_chunk[i] < chunks;
            const uint64_t from = (uint64_t)from_scale[i] + step * scale_stride[i], mask = there ? ~(uint64_t)0 : 0;
            load_to_lds_4((const void *)((from & mask) | (missing & ~mask)), scale[i] & (uint32_t)mask,
                          lds_offset(s.scales) + to_scale[i]);
        }
    }
};

template <typename T, int BM, int BN, int STAGES>
__global__ __launch_bounds__(kBlock) void mx4_matmul_kernel(MulArgs g)
{
    constexpr int FM = BM / 64, FN = BN / 64;       // 32 x 32 parts of a wave
    __shared__ Stage<BM, BN> stage[STAGES];
    static_assert(alignof(decltype(stage)) % alignof(vec_of<float, 16 / sizeof(T)>) == 0 && alignof(decltype(stage)) % alignof(int4) == 0, "operands and sheets are read in vectors");
    static_assert(sizeof(stage) >= kWavesPerBlock * 32 * sheet_pitch(FN) * 4, "the sheets lie where the operands were");
    using Loads = StepLoads<BM, BN>;
    const TilePlace place = tile_place(workgroup(), workgroups(), (uint32_t)g.tiles_m, (uint32_t)g.tiles_n, (uint32_t)g.splits);
    if (place.part < 0) return;
    const int64_t split = place.part, row0 = place.row * BM, col0 = place.col * BN;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int wm = wave / 2 * (BM / 2), wn = wave % 2 * (BN / 2);
    const int begin = (int)(split * g.steps_per_split), steps = (int)min(g.steps_per_split, g.steps - begin);
    const Loads loads(g, row0, col0);

    tile_sums sums[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) sums[i][j][q] = 0.0f;

    // The operands of a quarter of a step, 64 columns: read from the LDS while the quarter before is multiplied.
    struct Quarter { int4 a[FM], b[FN]; } quarter[2];
    uint32_t sa[kStepChunks][FM], sb[kStepChunks][FN];      // scales of this lane's rows; the upper half of a wave has the odd blocks
    auto read = [&](const Stage<BM, BN> &s, int at, Quarter &to) {
#pragma unroll
        for (int i = 0; i < FM; ++i) to.a[i] = *reinterpret_cast<const int4 *>(line_part(s.a, wm + i * 32 + r, at * 2 + h));
#pragma unroll
        for (int j = 0; j < FN; ++j) to.b[j] = *reinterpret_cast<const int4 *>(line_part(s.b, wn + j * 32 + r, at * 2 + h));
    };
    auto read_scales = [&](const Stage<BM, BN> &s, int c) {
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[c][i] = s.scales[c * BM + wm + i * 32 + r] >> (8 * h);
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[c][j] = s.scales[kStepChunks * BM + c * BN + wn + j * 32 + r] >> (8 * h);
    };
    // `between(p)` is done behind product p of the quarter's FM * FN.
    auto multiply = [&](const Quarter &f, int at, auto between) {
        const int c = at / 2;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const mx_codes a{f.a[i].x, f.a[i].y, f.a[i].z, f.a[i].w, 0, 0, 0, 0}, b{f.b[j].x, f.b[j].y, f.b[j].z, f.b[j].w, 0, 0, 0, 0};
                sums[i][j] = at % 2 == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, sums[i][j], 4, 4, 0, (int)sa[c][i], 0, (int)sb[c][j])
                                         : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, sums[i][j], 4, 4, 2, (int)sa[c][i], 2, (int)sb[c][j]);
                between(i * FN + j);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto nothing = [](int) {};

    // Up to STAGES steps are under way.  A step's last quarter is multiplied behind the barrier after which the next step is in the LDS and its own buffer
    // free, and the loads into that buffer are issued between its products.  No branches: across one the compiler would take products to the other side
    // of the barrier.
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < steps)
#pragma unroll
            for (int l = 0; l < Loads::kLoads; ++l) loads.load(l, begin + s, stage[s]);
    if (steps >= STAGES) arrived<Loads::kLoads * (STAGES - 1)>();
    else                 arrived<0>();
    read_scales(stage[0], 0);
    read(stage[0], 0, quarter[0]);
    int now = 0;
    auto one = [&](int step, auto more) {
        constexpr bool kMore = decltype(more)::value;
        const Stage<BM, BN> &s = stage[now];
        now = now + 1 == STAGES ? 0 : now + 1;
        read_scales(s, 1);
#pragma unroll
        for (int at = 0; at < 3; ++at) {
            read(s, at + 1, quarter[(at + 1) % 2]);
            __builtin_amdgcn_sched_barrier(0);
            multiply(quarter[at % 2], at, nothing);
        }
        arrived<kMore ? Loads::kLoads * (STAGES - 2) : 0>();
        read_scales(stage[now], 0);
        read(stage[now], 0, quarter[0]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(quarter[1], 3, [&](int p) {
            if constexpr (kMore) {
#pragma unroll
                for (int l = p * Loads::kLoads / (FM * FN); l < (p + 1) * Loads::kLoads / (FM * FN); ++l) loads.load(l, step + STAGES, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    };
    int i = 0;
    for (; i + STAGES < steps; ++i) one(begin + i, std::true_type());
    for (; i < steps; ++i) one(begin + i, std::false_type());

    store_tile<T, FM, FN>(g, sums, split, row0 + wm, col0 + wn, reinterpret_cast<float *>(stage));
}

// The same in steps of half a line, 128 columns and one scale word.  Of tiles of 256 x 256 two steps of a line fit the LDS, and the loads of the next would have to follow one another
// in a quarter of a step if they were to arrive in the rest; of half a line four fit, and loads and reads of the LDS alike lie one by one between the products
// (8192 x 8192 x 4096 fp32 181 us in lines, 176 with the loads spread, 171 with the reads spread).  Short rows have less of an empty half line.
template <int BM, int BN>
struct alignas(32) HalfStage {
    uint8_t a[BM * kLine / 2], b[BN * kLine / 2];
    uint32_t scales[BM + BN];
};

// Of such lines the four 16-byte parts lie at (part ^ row / 4 mod 4): four rows fill the banks.
__device__ __forceinline__ const uint8_t *half_part(const uint8_t *lds, int row, int part) { return lds + row * (kLine / 2) + (part ^ row / 4 % 4) * 16; }

template <int BM, int BN>
struct HalfLoads {
    static constexpr int kA = BM / 64, kB = BN / 64, kScaleLoads = (BM + BN + kBlock - 1) / kBlock, kLoads = kA + kB + kScaleLoads;
    uint32_t a[kA], b[kB], scale[kScaleLoads];
    const uint8_t *from_a, *from_b, *from_scale[kScaleLoads];
    int64_t scale_stride[kScaleLoads];
    uint32_t to_scale[kScaleLoads];
    int wave;

    __device__ __forceinline__ HalfLoads(const MulArgs &g, int64_t row0, int64_t col0, int64_t begin)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int lane = threadIdx.x % kWave;
        from_a = g.a_codes + row0 * g.pitch + begin * (kLine / 2);
        from_b = g.b_codes + col0 * g.pitch + begin * (kLine / 2);
        auto places = [&](auto &to, int rows, int64_t left) {           // 16 rows of four parts a load
            const uint32_t last = (uint32_t)min((int64_t)rows, left) - 1;
#pragma unroll
            for (int i = 0; i < rows / 64; ++i) to[i] = min((uint32_t)(wave * (rows / 4) + i * 16 + lane / 4), last) * (uint32_t)g.pitch + (lane % 4 ^ lane / 16) * 16;
        };
        places(a, BM, g.m - row0);
        places(b, BN, g.n - col0);
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            int at = (i * kWavesPerBlock + wave) * kWave % (BM + BN);
            to_scale[i] = at * 4;
            const bool of_b = at >= BM;
            at -= of_b ? BM : 0;
            const int64_t n = of_b ? g.n : g.m, first = of_b ? col0 : row0;
            scale_stride[i] = n * 4;
            from_scale[i] = (of_b ? g.b_scales : g.a_scales) + (begin * n + first) * 4;
            scale[i] = min((uint32_t)(at + lane), (uint32_t)min((int64_t)(of_b ? BN : BM), n - first) - 1) * 4;
        }
    }

    __device__ __forceinline__ void load(int i, int step, const HalfStage<BM, BN> &s) const
    {
        if (i < kA)           load_to_lds_16(from_a + (int64_t)step * (kLine / 2), a[i], __builtin_amdgcn_readfirstlane(lds_offset(s.a) + (wave * (BM / 4) + i * 16) * (kLine / 2)));
        else if (i < kA + kB) load_to_lds_16(from_b + (int64_t)step * (kLine / 2), b[i - kA], __builtin_amdgcn_readfirstlane(lds_offset(s.b) + (wave * (BN / 4) + (i - kA) * 16) * (kLine / 2)));
        else                  load_to_lds_4(from_scale[i - kA - kB] + step * scale_stride[i - kA - kB], scale[i - kA - kB], lds_offset(s.scales) + to_scale[i - kA - kB]);
    }
};

template <typename T, int BM, int BN, int STAGES>
__global__ __launch_bounds__(kBlock) void mx4_matmul_halves_kernel(MulArgs g)
{
    constexpr int FM = BM / 64, FN = BN / 64;
    __shared__ HalfStage<BM, BN> stage[STAGES];
    static_assert(alignof(decltype(stage)) % alignof(vec_of<float, 16 / sizeof(T)>) == 0 && alignof(decltype(stage)) % alignof(int4) == 0, "operands and sheets are read in vectors");
    static_assert(sizeof(stage) >= kWavesPerBlock * 32 * sheet_pitch(FN) * 4, "the sheets lie where the operands were");
    using Loads = HalfLoads<BM, BN>;
    const TilePlace place = tile_place(workgroup(), workgroups(), (uint32_t)g.tiles_m, (uint32_t)g.tiles_n, (uint32_t)g.splits);
    if (place.part < 0) return;
    const int64_t row0 = place.row * BM, col0 = place.col * BN;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int wm = wave / 2 * (BM / 2), wn = wave % 2 * (BN / 2);
    const int64_t begin = place.part * g.steps_per_split * kStepChunks;
    const int steps = (int)min(g.steps_per_split * kStepChunks, g.chunks - begin);
    const Loads loads(g, row0, col0, begin);

    tile_sums sums[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) sums[i][j][q] = 0.0f;

    struct Part { int4 a[FM], b[FN]; } part[2];     // of 64 columns
    uint32_t next_a[FM], next_b[FN], sa[FM], sb[FN];
    // Read `i` of a part, in the order in which products need them.
    constexpr int kReads = FM + FN;
    auto read = [&](const HalfStage<BM, BN> &s, int at, int i, Part &to) {
        if (i == 0)       to.a[0] = *reinterpret_cast<const int4 *>(half_part(s.a, wm + r, at * 2 + h));
        else if (i <= FN) to.b[i - 1] = *reinterpret_cast<const int4 *>(half_part(s.b, wn + (i - 1) * 32 + r, at * 2 + h));
        else              to.a[i - FN] = *reinterpret_cast<const int4 *>(half_part(s.a, wm + (i - FN) * 32 + r, at * 2 + h));
    };
    auto read_scales = [&](const HalfStage<BM, BN> &s) {
#pragma unroll
        for (int i = 0; i < FM; ++i) next_a[i] = s.scales[wm + i * 32 + r];
#pragma unroll
        for (int j = 0; j < FN; ++j) next_b[j] = s.scales[BM + wn + j * 32 + r];
    };
    auto multiply = [&](const Part &f, int at, auto between) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const mx_codes a{f.a[i].x, f.a[i].y, f.a[i].z, f.a[i].w, 0, 0, 0, 0}, b{f.b[j].x, f.b[j].y, f.b[j].z, f.b[j].w, 0, 0, 0, 0};
                sums[i][j] = at == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, sums[i][j], 4, 4, 0, (int)sa[i], 0, (int)sb[j])
                                     : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, sums[i][j], 4, 4, 2, (int)sa[i], 2, (int)sb[j]);
                between(i * FN + j);
            }
        __builtin_amdgcn_sched_barrier(0);
    };

    // Up to STAGES steps are under way.  A step's second part is multiplied behind the barrier after which the next step is in the LDS and its own buffer free; the loads into
    // that buffer are spread over those products and the first of the next step.
    constexpr int kProducts = FM * FN, kFirst = Loads::kLoads / 2, kReadsAtOnce = (kReads + kProducts - 1) / kProducts;
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < steps)
#pragma unroll
            for (int l = 0; l < (s < STAGES - 1 ? Loads::kLoads : kFirst); ++l) loads.load(l, s, stage[s]);
    if (steps >= STAGES) arrived<Loads::kLoads * (STAGES - 2) + kFirst>();
    else                 arrived<0>();
    read_scales(stage[0]);
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(stage[0], 0, i, part[0]);
    int now = 0, before = STAGES - 1;
    auto one = [&](int step, auto pending, auto more) {
        constexpr bool kPending = decltype(pending)::value, kMore = decltype(more)::value;
        const HalfStage<BM, BN> &s = stage[now], &last = stage[before];
        before = now;
        now = now + 1 == STAGES ? 0 : now + 1;
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = next_a[i] >> (8 * h);      // the upper half of a wave has the odd blocks
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] = next_b[j] >> (8 * h);
        __builtin_amdgcn_sched_barrier(0);
        multiply(part[0], 0, [&](int p) {
#pragma unroll
            for (int i = p * kReadsAtOnce; i < (p + 1) * kReadsAtOnce && i < kReads; ++i) read(s, 1, i, part[1]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kPending) {
#pragma unroll
                for (int l = kFirst + p * (Loads::kLoads - kFirst) / kProducts; l < kFirst + (p + 1) * (Loads::kLoads - kFirst) / kProducts; ++l)
                    loads.load(l, step - 1 + STAGES, last);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        arrived<kPending ? Loads::kLoads * (STAGES - 2) : 0>();
        __builtin_amdgcn_sched_barrier(0);
        multiply(part[1], 1, [&](int p) {
#pragma unroll
            for (int i = p * kReadsAtOnce; i < (p + 1) * kReadsAtOnce && i < kReads; ++i) read(stage[now], 0, i, part[0]);
            if (p == kProducts / 2) read_scales(stage[now]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kMore) {
#pragma unroll
                for (int l = p * kFirst / kProducts; l < (p + 1) * kFirst / kProducts; ++l) loads.load(l, step + STAGES, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    };
    int step = 0;
    for (; step + STAGES < steps; ++step) one(step, std::true_type(), std::true_type());
    if (steps >= STAGES) one(step++, std::true_type(), std::false_type());
    for (; step < steps; ++step) one(step, std::false_type(), std::false_type());
    store_tile<T, FM, FN>(g, sums, place.part, row0 + wm, col0 + wn, reinterpret_cast<float *>(stage));
}

constexpr int kFewRows = 32, kFewWaves = 8;

// At most 32 rows: 32 columns of out, wave w takes the lines w, w + 8, ... of its part of k.
template <typename T>
__global__ __launch_bounds__(kFewWaves * kWave) void mx4_few_rows_kernel(MulArgs g)
{
    constexpr int kLines = 2;                       // under way
    __shared__ float parts[kFewWaves][kFewRows * 32];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
    const int64_t col0 = (int64_t)workgroup() * 32;
    const int64_t row_a = min((int64_t)r, g.m - 1), row_b = min(col0 + r, g.n - 1);
    const int64_t begin = blockIdx.z * g.steps_per_split, end = min(begin + g.steps_per_split, g.steps);
    tile_sums sums;
#pragma unroll
    for (int q = 0; q < 16; ++q) sums[q] = 0.0f;
    for (int64_t step = begin + wave; step < end; step += kFewWaves * kLines) {
        int4 a[kLines][4], b[kLines][4];
        uint32_t sa[kLines][kStepChunks], sb[kLines][kStepChunks];
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
            const int64_t line = min(step + i * kFewWaves, end - 1);
            const bool missing = step + i * kFewWaves >= end;
            const int64_t half = (line + 1) * kStepChunks > g.chunks ? kLine / 2 : 0;  // the line ends there: its first half in the second's place
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t at = line * kLine + (q * 2 + h) * 16 - (q >= 2 ? half : 0);
                a[i][q] = *reinterpret_cast<const int4 *>(g.a_codes + row_a * g.pitch + at);
                b[i][q] = *reinterpret_cast<const int4 *>(g.b_codes + row_b * g.pitch + at);
            }
#pragma unroll
            for (int c = 0; c < kStepChunks; ++c) {
                const int64_t chunk = min(line * kStepChunks + c, g.chunks - 1);
                const bool none = missing || line * kStepChunks + c >= g.chunks;
                const uint32_t wa = *reinterpret_cast<const uint32_t *>(g.a_scales + (chunk * g.m + row_a) * 4);
                const uint32_t wb = *reinterpret_cast<const uint32_t *>(g.b_scales + (chunk * g.n + row_b) * 4);
                sa[i][c] = none ? 0 : wa >> (8 * h);            // the smallest scales: nothing is left of the product
                sb[i][c] = none ? 0 : wb >> (8 * h);
            }
        }
#pragma unroll
        for (int i = 0; i < kLines; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const mx_codes x{a[i][q].x, a[i][q].y, a[i][q].z, a[i][q].w, 0, 0, 0, 0}, y{b[i][q].x, b[i][q].y, b[i][q].z, b[i][q].w, 0, 0, 0, 0};
                sums = q % 2 == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, sums, 4, 4, 0, (int)sa[i][q / 2], 0, (int)sb[i][q / 2])
                                  : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, sums, 4, 4, 2, (int)sa[i][q / 2], 2, (int)sb[i][q / 2]);
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

enum MulTile { FEW_ROWS, TILE_64_64, TILE_128_64, TILE_128_64_HALVES, TILE_128_64_DEEP, TILE_128_128, TILE_256_256 };

struct MulShape {
    MulTile tile;
    int64_t tiles_m, tiles_n, steps, splits, steps_per_split, bytes;
};

// Large tiles read less and small ones overlap more: a workgroup of 256 x 256 fills a CU's LDS by itself, so that nothing runs while it begins and ends; two of
// 128 x 128 or three of 128 x 64 share one.  us for 8192 x 8192 fp32 outputs, k = 256, 1024, 2048, 3200, 4096, 8192: 256 x 256 67, 86, 113, 160, 171, 293;
// 128 x 128 55, 70, 110, 165, 193, 346; 128 x 64 62, 88, 127, 199, 217, 400.  Where the outputs' edges leave more of a larger tile empty than it gains, the smaller:
// 196 000 x 300, k = 256, 128 x 128 48 and 128 x 64 44.  A tile's time must not come in two rounds for a bit more than one: 58 000 x 256, k = 602, 908 tiles of
// 128 x 128, 21.3, with 128 x 64 19.6 (in whole lines 21.0; 8192 x 8192, k = 1024, 107 and 107, k = 2048 in half lines 144, in whole ones 129); 2048 x 2048, k = 2048, 256 tiles of 128 x 128, 14.7 against 13.0.
// k is split where tiles of 64 x 64 leave half of the CUs idle, in parts of at least eight steps, to about 480 workgroups (256 x 300 outputs, k = 196 000: 12, 24,
// 50 parts 29, 26, 34 us); from 25 such tiles on, tiles of 128 x 64 with one more step under way (256 x 602, k = 306 000: 70 us, 64 x 64 more than 78).
MulShape mul_shape(int64_t m, int64_t n, int64_t k)
{
    MulShape s{};
    auto tiles = [&](MulTile t, int64_t rows, int64_t cols) {
        s.tile = t;
        s.tiles_m = (m + rows - 1) / rows;
        s.tiles_n = (n + cols - 1) / cols;
        return s.tiles_m * s.tiles_n;
    };
    s.steps = (mx_chunks(k) + kStepChunks - 1) / kStepChunks;
    s.splits = 1;
    s.steps_per_split = s.steps;
    auto split = [&](int64_t splits) {
        if (splits < 2) return;
        s.steps_per_split = (s.steps + splits - 1) / splits;
        s.splits = (s.steps + s.steps_per_split - 1) / s.steps_per_split;
        s.bytes = s.splits > 1 ? (s.splits * m * n * 4 + 255) / 256 * 256 : 0;
    };
    if (m == 0 || n == 0) return s;
    if (m <= kFewRows) {
        const int64_t blocks = tiles(FEW_ROWS, kFewRows, 32), most = s.steps / (4 * kFewWaves);
        split(256 / blocks < most ? 256 / blocks : most);
        return s;
    }
    auto padded = [&](int64_t rows, int64_t cols) { return (double)((m + rows - 1) / rows * rows) * (double)((n + cols - 1) / cols * cols); };
    if (s.steps >= 12 && padded(256, 256) < 1.1 * padded(128, 128) && tiles(TILE_256_256, 256, 256) >= 512) return s;
    if (padded(128, 128) < 1.1 * padded(128, 64) && tiles(TILE_128_128, 128, 128) >= (s.steps >= 6 ? 512 : 1024)) return s;
    if (tiles(s.steps <= 3 ? TILE_128_64_HALVES : TILE_128_64, 128, 64) >= 256) return s;
    const int64_t small = tiles(TILE_64_64, 64, 64);
    if (small >= 128 || s.steps < 16) return s;
    const int64_t blocks = small >= 25 ? tiles(TILE_128_64_DEEP, 128, 64) : small;
    split(480 / blocks < s.steps / 8 ? 480 / blocks : s.steps / 8);
    return s;
}

template <typename T>
void launch_tiles(const MulArgs &g, const MulShape &s, hipStream_t st)
{
    const dim3 blocks = grid_of(tile_blocks(s.tiles_m * s.tiles_n, s.splits), kBlock);
    switch (s.tile) {
        case FEW_ROWS:         mx4_few_rows_kernel<T><<<grid_of((g.written + 31) / 32, kFewWaves * kWave, (uint32_t)s.splits), kFewWaves * kWave, 0, st>>>(g); break;
        case TILE_64_64:       mx4_matmul_kernel<T, 64, 64, 4><<<blocks, kBlock, 0, st>>>(g); break;
        case TILE_128_64:      mx4_matmul_kernel<T, 128, 64, 2><<<blocks, kBlock, 0, st>>>(g); break;
        case TILE_128_64_HALVES: mx4_matmul_halves_kernel<T, 128, 64, 4><<<blocks, kBlock, 0, st>>>(g); break;
        case TILE_128_64_DEEP: mx4_matmul_kernel<T, 128, 64, 3><<<blocks, kBlock, 0, st>>>(g); break;
        case TILE_128_128:     mx4_matmul_kernel<T, 128, 128, 2><<<blocks, kBlock, 0, st>>>(g); break;
        case TILE_256_256:     mx4_matmul_halves_kernel<T, 256, 256, 4><<<blocks, kBlock, 0, st>>>(g); break;
    }
}

int check_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return ADAQP_EINVAL;
    return m >= kMxMost || n >= kMxMost || k > kMostDepth || (m + 63) / 64 * ((n + 63) / 64) >= 0x3FFFFFFF ? ADAQP_ESIZE : ADAQP_OK;
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_mx4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t *bytes_out)
{
    if (!bytes_out) return ADAQP_EINVAL;
    ADAQP_TRY(check_sizes(m, n, k));
    *bytes_out = mul_shape(m, n, k).bytes;
    return ADAQP_OK;
}

extern "C" int adaqp_mx4_matmul(const uint8_t *a_codes_dev, const uint8_t *a_scales_dev, int64_t m,
                                const uint8_t *b_codes_dev, const uint8_t *b_scales_dev, int64_t n, int64_t k,
                                void *out_dev, int64_t ldo, int32_t type, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    ADAQP_TRY(check_sizes(m, n, k));
    if (!valid_type(type)) return ADAQP_EINVAL;
    if (m == 0 || n == 0) return ADAQP_OK;
    if (!out_dev || ldo < n || !aligned_to(out_dev, element_bytes(type))) return ADAQP_EINVAL;
    if (k > 0 && (!valid_mx(a_codes_dev, a_scales_dev) || !valid_mx(b_codes_dev, b_scales_dev))) return ADAQP_EINVAL;
    const MulShape s = mul_shape(m, n, k);
    if (s.splits > 1) {
        if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
        if (workspace_bytes < s.bytes) return ADAQP_ESIZE;
    }
    MulArgs g{a_codes_dev, a_scales_dev, b_codes_dev, b_scales_dev, out_dev, m, n, ldo, 0, mx_pitch(k), mx_chunks(k), s.steps, s.steps_per_split,
              s.splits, s.tiles_m, s.tiles_n, false};
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
        launch_tiles<float>(g, s, st);
        ADAQP_HIP_TRY(hipGetLastError());
        const int64_t rows = (m + kWavesPerBlock - 1) / kWavesPerBlock;
        const dim3 grid((uint32_t)((written + kWave - 1) / kWave), (uint32_t)(rows < 65535 ? rows : 65535));
        if (type == ADAQP_F32) join_parts_kernel<float><<<grid, kBlock, 0, st>>>((const float *)workspace_dev, (int)s.splits, m, n, written, (float *)out_dev, ldo);
        else                   join_parts_kernel<__bf16><<<grid, kBlock, 0, st>>>((const float *)workspace_dev, (int)s.splits, m, n, written, (__bf16 *)out_dev, ldo);
    } else if (type == ADAQP_F32) launch_tiles<float>(g, s, st);
    else                          launch_tiles<__bf16>(g, s, st);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}
