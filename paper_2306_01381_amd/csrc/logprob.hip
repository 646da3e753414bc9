// Log probabilities of given classes, with entropy, the likeliest classes, and the logits' gradient (adaqp_train.h).
//
// A row is read once.  What is kept of a part of it is (max, others, moment): others = the sum of exp(x_j - max) over all of the part but one largest, moment = the sum of
// (x_j - max) exp(x_j - max).  Two parts join by taking the smaller max's part, and its own largest, down by exp(smaller - larger).  Without the one largest, whose term is 1, log1p of
// the others keeps the digits of probabilities near 1.
//
// The largest logits are kept by a wave: a list in the LDS, and the n_top-th so far.  Only what is above that is added to the list, and the list is cut back to n_top
// when it is full: each of its members counts those above it.
//
// Bound by memory, and with many classes in 16 bits by the vector instructions as much: 13 a logit, one of them an exponential at a quarter of the rate, and 26 in the gradient.  Measured: 58 000 x 41 fp32 6.8 us, its gradient 7.3;
// 4096 x 32 001 bf16 63 us on operands that the caches do not hold (262 MB, 4.2 TB/s, the vector units busy in 74 % of the cycles; 53 to 59 where a part is in the last cache; with a branch for a new largest 95), its gradient 88
// (524 MB, 6.0 TB/s, in part from the last cache, the vector units always busy); 65 536 x 1000 fp32 44 us (5.9 TB/s).  3 x 128 000 bf16 with the 20 likeliest 11.6 us, and 5.1 for
// joining 31 splits of a row: waits, of the cuts of three lists after one another.
#include "adaqp_train.h"
#include "rows.hpp"

namespace adaqp {
namespace {

constexpr float kLog2E = 1.4426950408889634f;
constexpr int kMostTop = ADAQP_LOGPROB_MOST_TOP;
constexpr float kNothing = -200.0f;                 // exp of it is 0 in fp32

__device__ __forceinline__ float exp_of(float u) { return __builtin_amdgcn_exp2f(u * kLog2E); }

struct Part { float max, others, moment; };

__device__ __forceinline__ Part no_part() { return Part{-__builtin_inff(), 0.0f, 0.0f}; }

// Whether any logit of it is above -inf.  (NaN: max is NaN, and this is true.)
__device__ __forceinline__ bool is_part(const Part &p) { return !(p.max == -__builtin_inff()); }

// `low` with its largest counted, in units of exp(max); max is not below low's.
__device__ __forceinline__ void lower(const Part &low, float max, float &others, float &moment)
{
    const float down = low.max - max, e = exp_of(down), clamped = fmaxf(down, kNothing);
    const float sum = (low.others + 1.0f) * e;
    others = sum;
    moment = low.moment * e + clamped * sum;        // sum of (u + down) e^(u + down) over the others and u = 0
}

__device__ __forceinline__ Part join(const Part &a, const Part &b)
{
    if (!is_part(b)) return a;
    if (!is_part(a)) return b;
    const bool first = a.max >= b.max;
    const Part &high = first ? a : b, &low = first ? b : a;
    float others, moment;
    lower(low, high.max, others, moment);
    return Part{high.max != high.max || low.max != low.max ? __builtin_nanf("") : high.max, high.others + others, high.moment + moment};
}

// A lane's logits as they come: of the largest so far and the next, the smaller is counted and the larger kept, so that the largest of all is never counted.  Sums are in units of
// exp(base), a logit that the lane has seen; it moves where they could grow out of fp32.  The difference from base comes before the product with log2(e): it is exact for logits near base however large
// both are, where in fma(x, log2(e), -base log2(e)) the last term's rounding, 2^-24 of |base|, passes the exponents of fp32 from 5e9 on (logits that are masked by a finite number).
struct Running {
    float base, max, others, moment;

    __device__ __forceinline__ void begin()
    {
        base = max = -__builtin_inff();
        others = moment = 0.0f;
    }

    // N logits, not all of which need be there (those are -inf); the largest of them.
    template <int N>
    __device__ __forceinline__ float add(const float (&x)[N])
    {
        float most = x[0];
#pragma unroll
        for (int k = 1; k < N; ++k) most = __builtin_elementwise_maximum(most, x[k]);      // NaN where there is one
        if (!(most <= base + 30.0f)) {              // the lane's first, NaN, or far above
            const Part p = part();
            base = most;
            others = moment = 0.0f;
            if (is_part(p)) {
                const float down = p.max - base, e = exp_of(down), clamped = fmaxf(down, kNothing);
                others = p.others * e;
                moment = p.moment * e + clamped * others;
            }
        }
        if (base == -__builtin_inff()) return most; // all are
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float low = __builtin_elementwise_minimum(max, x[k]);
            max = __builtin_elementwise_maximum(max, x[k]);
            const float u = __builtin_elementwise_maximum(low - base, kNothing), e = exp_of(u);
            others += e;
            moment = __builtin_fmaf(u, e, moment);
        }
        return most;
    }

    __device__ __forceinline__ Part part() const
    {
        if (max == -__builtin_inff()) return no_part();
        const float down = base - max, e = exp_of(down), sum = others * e;
        return Part{max, sum, __builtin_fmaf(fmaxf(down, kNothing), sum, moment * e)};
    }
};

// The largest over LANES neighbouring lanes, NaN where there is one, in all of them.
template <int LANES>
__device__ __forceinline__ float lane_most(float v)
{
    auto moved = [](float x, auto pattern) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int32_t, x), decltype(pattern)::value, 0xF, 0xF, false));
    };
    if constexpr (LANES >= 2) v = __builtin_elementwise_maximum(v, moved(v, std::integral_constant<int, 0xB1>()));     // quad_perm [1, 0, 3, 2]
    if constexpr (LANES >= 4) v = __builtin_elementwise_maximum(v, moved(v, std::integral_constant<int, 0x4E>()));     // quad_perm [2, 3, 0, 1]
    if constexpr (LANES >= 8) v = __builtin_elementwise_maximum(v, moved(v, std::integral_constant<int, 0x141>()));    // row_half_mirror
    if constexpr (LANES >= 16) v = __builtin_elementwise_maximum(v, moved(v, std::integral_constant<int, 0x140>()));   // row_mirror
    if constexpr (LANES >= 32) v = __builtin_elementwise_maximum(v, __shfl_xor(v, 16));
    if constexpr (LANES >= 64) v = __builtin_elementwise_maximum(v, __shfl_xor(v, 32));
    return v;
}

// Over the lanes of a wave, in all of them.
__device__ __forceinline__ Part join_lanes(const Part &p)
{
    const float max = lane_most<kWave>(p.max);
    if (max == -__builtin_inff()) return no_part();
    const uint64_t with = __ballot(p.max == max);
    const bool left_out = with && (int)(threadIdx.x % kWave) == __builtin_ctzll(with);      // one largest is not counted
    const float down = p.max - max, e = exp_of(down);
    const float others = p.others * e + (left_out ? 0.0f : e);
    return Part{max, lane_sum<kWave>(others), lane_sum<kWave>(__builtin_fmaf(fmaxf(down, kNothing), others, p.moment * e))};
}

// ---- the largest --------------------------------------------------------------------------------------------------------------------------

// Logits in descending order and classes in ascending order: larger is earlier.
typedef unsigned long long Place;
__device__ __forceinline__ uint32_t value_key(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);                              // -0 is 0
    if (x != x) return 0xFFFFFFFFu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t key)
{
    if (key == 0xFFFFFFFFu) return __builtin_nanf("");
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ Place place_of(float x, uint32_t index) { return (Place)value_key(x) << 32 | (uint32_t)~index; }

constexpr int kList = 256, kPadding = 8;

// A wave's.
struct Largest {
    Place *list;                                    // kList + kPadding
    int count, n_top;
    Place least;                                    // what is not above it is not among the largest

    __device__ __forceinline__ void begin(Place *lds, int n)
    {
        list = lds;
        count = 0;
        n_top = n;
        least = 0;
    }

    // The n_top largest of the first EACH * 64, in descending order, to the list's beginning.
    template <int EACH>
    __device__ __forceinline__ void rank()
    {
        const int lane = threadIdx.x % kWave;
        Place mine[EACH];
        int above[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            mine[i] = i * kWave + lane < count ? list[i * kWave + lane] : 0;
            above[i] = 0;
        }
        for (int j = 0; j < count; j += kPadding)
#pragma unroll
            for (int k = 0; k < kPadding; ++k) {
                const Place other = list[j + k];
#pragma unroll
                for (int i = 0; i < EACH; ++i) above[i] += other > mine[i] ? 1 : 0;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (mine[i] != 0 && above[i] < n_top) list[above[i]] = mine[i];
    }

    // The list's n_top largest, in descending order, at its beginning.
    __device__ __forceinline__ void cut()
    {
        if (threadIdx.x % kWave < kPadding) list[count + threadIdx.x % kWave] = 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (count <= kWave) rank<1>();
        else                rank<kList / kWave>();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        count = min(count, n_top);
        if (count == n_top) least = list[n_top - 1];
    }

    // Before the first are added: the n_top-th largest of the lanes' best is a bound, so that hardly more than n_top of them are added.
    __device__ __forceinline__ void bound(Place best)
    {
        const uint64_t with = __ballot(best != 0);
        if (__popcll(with) < n_top) return;
        if (best != 0) list[__popcll(with & (((uint64_t)1 << threadIdx.x % kWave) - 1))] = best;
        count = __popcll(with);
        cut();
        least -= 1;                                 // itself is to be added
        count = 0;
    }

    // One place of each lane that has one; there is room for them.
    __device__ __forceinline__ void add(Place place)
    {
        const bool has = place > least;
        const uint64_t with = __ballot(has);
        if (has) list[count + __popcll(with & (((uint64_t)1 << threadIdx.x % kWave) - 1))] = place;
        count += __popcll(with);
    }

    __device__ __forceinline__ void make_room()
    {
        if (count + kWave > kList) cut();
    }

    // N places of each lane that has them; other(k) gives place k once more, for a loop that is not unrolled.
    template <int N, typename F>
    __device__ __forceinline__ void add_all(const Place (&place)[N], F other)
    {
        int more = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) more += __popcll(__ballot(place[k] > least));
        if (more == 0) return;
        if (count + more <= kList) {
#pragma unroll
            for (int k = 0; k < N; ++k) add(place[k]);
        } else {
#pragma unroll 1
            for (int k = 0; k < N; ++k) {
                make_room();
                add(other(k));
            }
        }
    }
};

template <int N>
__device__ __forceinline__ Place best_of(const Place (&place)[N])
{
    Place best = place[0];
#pragma unroll
    for (int k = 1; k < N; ++k) best = place[k] > best ? place[k] : best;
    return best;
}

// ---- forward ------------------------------------------------------------------------------------------------------------------------------

struct ProbArgs {
    const void *logits;
    const int32_t *targets;
    float *logp, *entropy, *stats, *top_logp;
    int32_t *top_class;
    Part *parts;                                    // [rows][splits]
    Place *places;                                  // [rows][splits][n_top]
    int64_t ld, n_rows, span;
    int32_t n_classes, n_top;
    int32_t splits, per_split;                      // classes of a split, a multiple of 8
};

template <typename T>
__device__ __forceinline__ float one_logit(const ProbArgs &a, int64_t row, int32_t j) { return (float)((const T *)a.logits)[row * a.ld + j]; }

// What a row's part comes to.
struct Prob {
    float max, rest, entropy;
    bool none;
    __device__ __forceinline__ float logp(float x) const { return none ? -__builtin_inff() : (x - max) - rest; }
};

__device__ __forceinline__ Prob prob_of(const Part &p)
{
    Prob r;
    r.none = !is_part(p);
    const bool bad = !(p.max < __builtin_inff());
    r.max = p.max;
    r.rest = bad ? __builtin_nanf("") : r.none ? 0.0f : log1pf(p.others);
    r.entropy = r.none ? 0.0f : r.rest - p.moment / (1.0f + p.others);
    return r;
}

// By the first threads of those that hold a row's largest.
template <typename T>
__device__ __forceinline__ void store_row(const ProbArgs &a, int64_t row, const Part &p, int thread, const Place *largest)
{
    const Prob prob = prob_of(p);
    if (thread == 0) {
        if (a.stats) {
            a.stats[row * 2] = p.max;
            a.stats[row * 2 + 1] = prob.rest;
        }
        if (a.entropy) a.entropy[row] = prob.entropy;
        if (a.logp) {
            const int32_t t = a.targets[row];
            a.logp[row] = t >= 0 && t < a.n_classes ? prob.logp(one_logit<T>(a, row, t)) : 0.0f;
        }
    }
    if (thread < a.n_top) {
        const Place place = largest[thread];
        a.top_class[row * a.n_top + thread] = (int32_t)~(uint32_t)place;
        a.top_logp[row * a.n_top + thread] = prob.logp(key_value((uint32_t)(place >> 32)));
    }
}

// A part of a row by a workgroup of WAVES waves, each of which has a contiguous share.
template <typename T, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES * kWave) void logprob_kernel(ProbArgs a)
{
    constexpr int kPieces = 2, kAtOnce = kPieces * kWave * 8;
    __shared__ Place lists[TOP ? WAVES : 1][TOP ? kList + kPadding : 1];
    __shared__ Part parts[WAVES];
    __shared__ int counts[WAVES];
    const uint64_t at = workgroup();
    const int64_t row = at / (uint32_t)a.splits;
    if (row >= a.n_rows) return;
    const int32_t split = (int32_t)(at - row * a.splits), first = split * a.per_split, last = (int32_t)min((int64_t)first + a.per_split, (int64_t)a.n_classes);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int32_t share = ((last - first + WAVES - 1) / WAVES + 7) / 8 * 8, begin = min(first + wave * share, last), end = min(begin + share, last);
    Running running;
    running.begin();
    Largest largest;
    largest.begin(lists[TOP ? wave : 0], a.n_top);
    auto take = [&](int32_t col0, const float (&x)[kPieces * 8]) {
        const float most = running.add<kPieces * 8>(x);
        if constexpr (TOP) {
            if (!__ballot(!(most < key_value((uint32_t)(largest.least >> 32))))) return;        // none reaches the list (NaN does)
            auto number = [&](int k) { return col0 + (k / 8 * kWave + lane) * 8 + k % 8; };
            Place place[kPieces * 8];
#pragma unroll
            for (int k = 0; k < kPieces * 8; ++k) place[k] = number(k) < end ? place_of(x[k], (uint32_t)number(k)) : 0;
            if (col0 == begin) largest.bound(best_of(place));
            largest.add_all(place, [&](int k) { return number(k) < end ? place_of(one_logit<T>(a, row, number(k)), (uint32_t)number(k)) : 0; });
        }
    };
    // what is whole is on its way while what is before it is counted
    typedef loose_vec<T, 8> Raw;
    vec_of<T, 8> next[kPieces];
    auto load = [&](int32_t col0) {
        const T *from = (const T *)a.logits + row * a.ld + col0 + lane * 8;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) next[i] = *reinterpret_cast<const Raw *>(from + i * kWave * 8);
    };
    if (end - begin >= kAtOnce) load(begin);
    for (int32_t col0 = begin; col0 < end; col0 += kAtOnce) {
        float x[kPieces * 8];
        if (end - col0 >= kAtOnce) {
#pragma unroll
            for (int k = 0; k < kPieces * 8; ++k) x[k] = (float)next[k / 8][k % 8];
            if (end - col0 >= 2 * kAtOnce) load(col0 + kAtOnce);
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int32_t col = col0 + (i * kWave + lane) * 8;
                float v[8];
                if (col < end) load_piece<T, 8>((const T *)a.logits, row * a.ld + col, end - col, a.span, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[i * 8 + k] = col + k < end ? v[k] : -__builtin_inff();
            }
        }
        take(col0, x);
    }
    Part p = join_lanes(running.part());
    if (TOP) largest.cut();
    if (lane == 0) {
        parts[wave] = p;
        counts[wave] = largest.count;
    }
    __syncthreads();
    if (wave != 0) return;
    p = join_lanes(lane < WAVES ? parts[lane] : no_part());
    if (TOP) {
        static_assert(WAVES * kMostTop <= kList, "the waves' lists have room");
        for (int w = 1; w < WAVES; ++w) largest.add(lane < counts[w] ? lists[TOP ? w : 0][lane] : 0);
        largest.cut();
    }
    if (a.splits == 1) {
        store_row<T>(a, row, p, lane, lists[0]);
        return;
    }
    if (lane == 0) a.parts[row * a.splits + split] = p;
    if (TOP && lane < a.n_top) a.places[(row * a.splits + split) * a.n_top + lane] = lane < largest.count ? lists[0][lane] : 0;
}

template <int LANES>
__device__ __forceinline__ Place lane_most(Place v)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
        const Place other = (Place)(uint32_t)__shfl_xor((int)(v >> 32), d) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)v, d);
        v = other > v ? other : v;
    }
    return v;
}

// Rows of at most 64 lanes' registers: LANES lanes have one, PIECES pieces of 8 logits each.
template <typename T, int LANES, int PIECES, int EACH, bool TOP>
__global__ __launch_bounds__(kBlock) void logprob_rows_kernel(ProbArgs a)
{
    constexpr int kRows = kBlock / LANES;
    __shared__ Place lists[TOP && LANES == kWave ? kWavesPerBlock : 1][TOP && LANES == kWave ? kList + kPadding : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t row0 = (int64_t)workgroup() * (kRows * EACH) + threadIdx.x / LANES;
    float x[EACH][PIECES * 8];
    int32_t target[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int64_t row = min(row0 + e * kRows, a.n_rows - 1);
        target[e] = a.logp ? a.targets[row] : -1;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int32_t col = (p * LANES + lane) * 8;
            float v[8];
            if (col < a.n_classes) load_piece<T, 8>((const T *)a.logits, row * a.ld + col, a.n_classes - col, a.span, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[e][p * 8 + k] = col + k < a.n_classes ? v[k] : -__builtin_inff();
        }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int64_t row = row0 + e * kRows;
        float most = x[e][0];
#pragma unroll
        for (int k = 1; k < PIECES * 8; ++k) most = __builtin_elementwise_maximum(most, x[e][k]);
        most = lane_most<LANES>(most);
        float others = 0.0f, moment = 0.0f, of_target = 0.0f;
        int equal = 0;                              // logits that are the largest
#pragma unroll
        for (int k = 0; k < PIECES * 8; ++k) {
            const float u = x[e][k] - most;
            const bool is = x[e][k] == most;
            const float v = is ? 0.0f : exp_of(u);
            equal += is ? 1 : 0;
            others += v;
            moment += fmaxf(u, kNothing) * v;
            of_target += (k / 8 * LANES + lane) * 8 + k % 8 == target[e] ? x[e][k] : 0.0f;
        }
        others = lane_sum<LANES>(others) + (lane_sum<LANES>((float)equal) - 1.0f);
        moment = lane_sum<LANES>(moment);
        of_target = lane_sum<LANES>(of_target);
        const Prob prob = prob_of(Part{most, others, moment});
        if (lane == 0 && row < a.n_rows) {
            if (a.stats) {
                a.stats[row * 2] = most;
                a.stats[row * 2 + 1] = prob.rest;
            }
            if (a.entropy) a.entropy[row] = prob.entropy;
            if (a.logp) a.logp[row] = target[e] >= 0 && target[e] < a.n_classes ? prob.logp(of_target) : 0.0f;
        }
        if constexpr (TOP && LANES == kWave) {
            auto number = [&](int k) { return (k / 8 * LANES + lane) * 8 + k % 8; };
            Place place[PIECES * 8];
#pragma unroll
            for (int k = 0; k < PIECES * 8; ++k) place[k] = number(k) < a.n_classes ? place_of(x[e][k], (uint32_t)number(k)) : 0;
            Largest largest;
            largest.begin(lists[threadIdx.x / kWave], a.n_top);
            largest.bound(best_of(place));
            const int64_t there = min(row, a.n_rows - 1);
            largest.add_all(place, [&](int k) { return number(k) < a.n_classes ? place_of(one_logit<T>(a, there, number(k)), (uint32_t)number(k)) : 0; });
            largest.cut();
            if (lane < a.n_top && row < a.n_rows) {
                const Place now = lists[threadIdx.x / kWave][lane];
                a.top_class[row * a.n_top + lane] = (int32_t)~(uint32_t)now;
                a.top_logp[row * a.n_top + lane] = prob.logp(key_value((uint32_t)(now >> 32)));
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        } else if constexpr (TOP) {
            Place place[PIECES * 8], best = 0;
#pragma unroll
            for (int k = 0; k < PIECES * 8; ++k) {
                const int32_t j = (k / 8 * LANES + lane) * 8 + k % 8;
                place[k] = j < a.n_classes ? place_of(x[e][k], (uint32_t)j) : 0;
                best = place[k] > best ? place[k] : best;
            }
            for (int n = 0; n < a.n_top; ++n) {
                const Place now = lane_most<LANES>(best);
                if (lane == n % LANES && row < a.n_rows) {
                    a.top_class[row * a.n_top + n] = (int32_t)~(uint32_t)now;
                    a.top_logp[row * a.n_top + n] = prob.logp(key_value((uint32_t)(now >> 32)));
                }
                if (best == now) {                  // this lane's: its next below
                    best = 0;
#pragma unroll
                    for (int k = 0; k < PIECES * 8; ++k) best = place[k] < now && place[k] > best ? place[k] : best;
                }
            }
        }
    }
}

// The splits of a row, a wave.
template <typename T>
__global__ __launch_bounds__(kWave) void logprob_join_kernel(ProbArgs a)
{
    constexpr int kAtOnce = 16;
    __shared__ Place list[kList + kPadding];
    const int64_t row = workgroup();
    if (row >= a.n_rows) return;
    const int lane = threadIdx.x;
    Part p = no_part();
    for (int32_t s = lane; s < a.splits; s += kWave) p = join(p, a.parts[row * a.splits + s]);
    Largest largest;
    largest.begin(list, a.n_top);
    const int32_t n = a.splits * a.n_top;
    for (int32_t i = 0; i < n; i += kAtOnce * kWave) {
        Place place[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) place[k] = i + k * kWave + lane < n ? a.places[row * n + i + k * kWave + lane] : 0;
        if (i == 0) largest.bound(best_of(place));
        largest.add_all(place, [&](int k) { return i + k * kWave + lane < n ? a.places[row * n + i + k * kWave + lane] : 0; });
    }
    p = join_lanes(p);
    if (a.n_top) largest.cut();
    store_row<T>(a, row, p, lane, list);
}

struct ProbShape {
    int32_t splits, per_split;
    int64_t bytes_parts, bytes;
};

// Rows are split where they are few.
ProbShape prob_shape(int64_t n_rows, int32_t n_classes, int32_t n_top)
{
    ProbShape s{1, (n_classes + 7) / 8 * 8, 0, 0};
    if (n_rows == 0 || n_rows >= 512 || n_classes < 8192) return s;
    const int64_t most = n_classes / 4096, wanted = 512 / n_rows;
    const int64_t splits = wanted < most ? wanted : most;
    if (splits < 2) return s;
    s.per_split = (int32_t)(((n_classes + splits - 1) / splits + 7) / 8 * 8);
    s.splits = (n_classes + s.per_split - 1) / s.per_split;
    s.bytes_parts = (n_rows * s.splits * (int64_t)sizeof(Part) + 255) / 256 * 256;
    s.bytes = s.bytes_parts + (n_rows * s.splits * n_top * (int64_t)sizeof(Place) + 255) / 256 * 256;
    return s;
}

template <typename T, int LANES, int PIECES>
void launch_rows(const ProbArgs &a, hipStream_t st)
{
    constexpr int kEach = PIECES == 1 ? 2 : 1, kRows = kBlock / LANES * kEach;
    const dim3 grid = grid_of((a.n_rows + kRows - 1) / kRows, kBlock);
    if (a.n_top) logprob_rows_kernel<T, LANES, PIECES, kEach, true><<<grid, kBlock, 0, st>>>(a);
    else         logprob_rows_kernel<T, LANES, PIECES, kEach, false><<<grid, kBlock, 0, st>>>(a);
}

template <typename T>
hipError_t launch_forward(const ProbArgs &a, hipStream_t st)
{
    if (a.n_classes <= 32)       launch_rows<T, 4, 1>(a, st);
    else if (a.n_classes <= 64)  launch_rows<T, 8, 1>(a, st);
    else if (a.n_classes <= 128) launch_rows<T, 16, 1>(a, st);
    else if (a.n_classes <= 256) launch_rows<T, 32, 1>(a, st);
    else if (a.n_classes <= 512) launch_rows<T, 64, 1>(a, st);
    else if (a.n_classes <= 1024) launch_rows<T, 64, 2>(a, st);
    else if (a.n_classes <= 2048) launch_rows<T, 64, 4>(a, st);
    else if (a.n_top)             logprob_kernel<T, 4, true><<<grid_of(a.n_rows * a.splits, kBlock), kBlock, 0, st>>>(a);
    else                          logprob_kernel<T, 4, false><<<grid_of(a.n_rows * a.splits, kBlock), kBlock, 0, st>>>(a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.splits == 1) return err;
    logprob_join_kernel<T><<<grid_of(a.n_rows, kWave), kWave, 0, st>>>(a);
    return hipGetLastError();
}

// ---- backward -----------------------------------------------------------------------------------------------------------------------------

struct ProbGradArgs {
    const void *logits;
    void *dlogits;
    const int32_t *targets;
    const float *stats, *entropy, *dlogp, *dentropy;
    int64_t ld, ldd, span;
    uint64_t pieces;
    Divider pieces_of_row;
    int32_t n_classes, written;
    float scale;
};

template <typename T, bool ONCE>
__global__ __launch_bounds__(kBlock) void logprob_gradient_kernel(ProbGradArgs a)
{
    constexpr int kEach = 2;
    // From the last row to the first, and stored past the caches where the logits fill them: what the forward pass read last is still there.  4096 x 32 001 bf16, both passes on the same logits 138 us,
    // from the first row on 142, stored through the caches 168; on others each time 151, 152, 171.
    const uint64_t first = (uint64_t)(workgroups() - 1 - workgroup()) * (kBlock * kEach) + threadIdx.x;
    int64_t row[kEach];
    int32_t col[kEach];
    float x[kEach][8];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint64_t at = min(first + e * kBlock, a.pieces - 1);
        row[e] = a.pieces_of_row.quotient(at);
        col[e] = (int32_t)(at - (uint64_t)row[e] * a.pieces_of_row.by) * 8;
        load_piece<T, 8>((const T *)a.logits, row[e] * a.ld + col[e], a.n_classes - col[e], a.span, x[e]);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int32_t t = a.targets ? a.targets[row[e]] : -1;
        const bool given = t >= 0 && t < a.n_classes;
        const float max = a.stats[row[e] * 2], rest = a.stats[row[e] * 2 + 1];
        const float dlogp = given ? (a.dlogp ? a.dlogp[row[e]] : 1.0f) : 0.0f;
        const float dentropy = a.dentropy ? a.dentropy[row[e]] : 0.0f, entropy = a.dentropy ? a.entropy[row[e]] : 0.0f;
        const bool zeros = max == -__builtin_inff() || !(given || a.dentropy);
        float d[8], other = 0.0f;                   // 1 - p of the target, with its digits where p is near 1
        if (given && t >= col[e] && t < col[e] + 8) {
#pragma unroll
            for (int k = 0; k < 8; ++k) other = col[e] + k == t ? x[e][k] : other;
            other = -expm1f(fmaxf(other - max, kNothing) - rest);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float logp = fmaxf(x[e][k] - max, kNothing) - rest, p = exp_of(logp);
            float v = given ? dlogp * (col[e] + k == t ? other : -p) : 0.0f;
            if (a.dentropy) v -= dentropy * p * (logp + entropy);
            d[k] = zeros || col[e] + k >= a.n_classes ? 0.0f : v * a.scale;
        }
        if (first + e * kBlock < a.pieces) store_piece<T, 8, ONCE>((T *)a.dlogits + row[e] * a.ldd + col[e], a.written - col[e], d);
    }
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_logprob_workspace_bytes(int64_t n_rows, int32_t n_classes, int32_t n_top, int64_t *bytes_out)
{
    if (!bytes_out || n_rows < 0 || n_classes <= 0 || n_top < 0 || n_top > n_classes || n_top > kMostTop) return ADAQP_EINVAL;
    if (n_classes > kMostDim) return ADAQP_ESIZE;
    *bytes_out = prob_shape(n_rows, n_classes, n_top).bytes;
    return ADAQP_OK;
}

extern "C" int adaqp_logprob_forward(const void *logits_dev, int64_t ld, int64_t n_rows, int32_t n_classes, int32_t type, const int32_t *targets_dev,
                                     float *logp_dev, float *entropy_dev, float *stats_dev, int32_t n_top, float *top_logp_dev, int32_t *top_class_dev,
                                     void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (n_rows < 0 || n_classes <= 0 || !valid_type(type) || n_top < 0 || n_top > n_classes || n_top > kMostTop) return ADAQP_EINVAL;
    if (!aligned_to(targets_dev, 4) || !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(stats_dev, 4) || !aligned_to(top_logp_dev, 4) ||
        !aligned_to(top_class_dev, 4)) return ADAQP_EINVAL;
    if (n_classes > kMostDim) return ADAQP_ESIZE;
    if (n_rows == 0) return ADAQP_OK;
    ADAQP_TRY(check_rows(logits_dev, ld, n_classes, type));
    if ((n_top > 0) != (top_logp_dev != nullptr) || (n_top > 0) != (top_class_dev != nullptr) || (logp_dev && !targets_dev)) return ADAQP_EINVAL;
    const ProbShape s = prob_shape(n_rows, n_classes, n_top);
    if (s.bytes > 0) {
        if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
        if (workspace_bytes < s.bytes) return ADAQP_ESIZE;
    }
    if (!countable(n_rows, ld) || n_rows >= kMostWorkgroups / s.splits) return ADAQP_ESIZE;
    ProbArgs a{};
    a.logits = logits_dev; a.targets = targets_dev; a.logp = logp_dev; a.entropy = entropy_dev; a.stats = stats_dev; a.top_logp = top_logp_dev;
    a.top_class = top_class_dev; a.ld = ld; a.n_rows = n_rows; a.n_classes = n_classes; a.n_top = n_top; a.splits = s.splits; a.per_split = s.per_split;
    a.span = matrix_span(n_rows, ld, n_classes);
    a.parts = (Part *)workspace_dev;
    a.places = (Place *)((uint8_t *)workspace_dev + s.bytes_parts);
    if (type == ADAQP_F32) ADAQP_HIP_TRY(launch_forward<float>(a, (hipStream_t)stream));
    else                   ADAQP_HIP_TRY(launch_forward<__bf16>(a, (hipStream_t)stream));
    return ADAQP_OK;
}

extern "C" int adaqp_logprob_backward(const void *logits_dev, int64_t ld, int64_t n_rows, int32_t n_classes, int32_t type, const int32_t *targets_dev,
                                      const float *stats_dev, const float *entropy_dev, const float *dlogp_dev, const float *dentropy_dev, float scale,
                                      void *dlogits_dev, int64_t ldd, void *stream)
{
    if (n_rows < 0 || n_classes <= 0 || !valid_type(type) || !(scale - scale == 0.0f)) return ADAQP_EINVAL;
    if (!aligned_to(targets_dev, 4) || !aligned_to(stats_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(dlogp_dev, 4) || !aligned_to(dentropy_dev, 4)) return ADAQP_EINVAL;
    if (n_classes > kMostDim) return ADAQP_ESIZE;
    if (n_rows == 0) return ADAQP_OK;
    ADAQP_TRY(check_rows(logits_dev, ld, n_classes, type));
    ADAQP_TRY(check_rows(dlogits_dev, ldd, n_classes, type));
    if (!stats_dev || (dentropy_dev && !entropy_dev) || (dlogits_dev == logits_dev && ldd != ld)) return ADAQP_EINVAL;
    if (!countable(n_rows, ld) || !countable(n_rows, ldd)) return ADAQP_ESIZE;
    ProbGradArgs a{};
    a.logits = logits_dev; a.dlogits = dlogits_dev; a.targets = targets_dev; a.stats = stats_dev; a.entropy = entropy_dev; a.dlogp = dlogp_dev;
    a.dentropy = dentropy_dev; a.ld = ld; a.ldd = ldd; a.n_classes = n_classes; a.scale = scale;
    a.span = matrix_span(n_rows, ld, n_classes);
    a.written = (int32_t)columns_to_write(dlogits_dev, ldd, n_classes, element_bytes(type));
    const int64_t each = ((int64_t)a.written + 7) / 8;
    if (n_rows > kMostWorkgroups * kBlock / each) return ADAQP_ESIZE;
    a.pieces = (uint64_t)(n_rows * each);
    a.pieces_of_row = divider(each, (int64_t)a.pieces);
    const dim3 grid = grid_of((int64_t)((a.pieces + 2 * kBlock - 1) / (2 * kBlock)), kBlock);
    const hipStream_t st = (hipStream_t)stream;
    const bool once = passes_caches(a.span, element_bytes(type));
    if (type == ADAQP_F32 && once) logprob_gradient_kernel<float, true><<<grid, kBlock, 0, st>>>(a);
    else if (type == ADAQP_F32)    logprob_gradient_kernel<float, false><<<grid, kBlock, 0, st>>>(a);
    else if (once)                 logprob_gradient_kernel<__bf16, true><<<grid, kBlock, 0, st>>>(a);
    else                           logprob_gradient_kernel<__bf16, false><<<grid, kBlock, 0, st>>>(a);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}
