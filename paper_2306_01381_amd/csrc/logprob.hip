// Log probabilities of given classes, with entropy, the likeliest classes, and the logits' gradient (adaqp_train.h).
//
// A row is read once.  What is kept of a part of it is (max, others, moment): others = the sum of exp(x_j - max) over all of the part but one largest, moment = the sum of
// (x_j - max) exp(x_j - max).  Two parts join by taking the smaller max's part, and its own largest, down by exp(smaller - larger).  Without the one largest, whose term is 1, log1p of
// the others keeps the digits of probabilities near 1.
//
// The largest logits are kept by a wave: a list in the LDS, and the n_top-th so far.  Only what is above that is added to the list, and the list is cut back to n_top
// when it is full: each of its members counts those above it.
#include "adaqp_train.h"
#include "rows.hpp"

namespace adaqp {
namespace {

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
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

// Adds N logits, not all of which are there (those are -inf).
template <int N>
__device__ __forceinline__ void add_logits(Part &p, const float (&x)[N])
{
    float most = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) most = __builtin_elementwise_maximum(most, x[k]);          // NaN where there is one
    if (most <= p.max) {
        if (!is_part(p)) return;                    // all are -inf
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float u = x[k] - p.max, e = exp_of(u);
            p.others += e;
            p.moment += fmaxf(u, kNothing) * e;
        }
        return;
    }
    Part now{most, 0.0f, 0.0f};
    bool one = true;                                // the largest that is not counted is still to come
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float u = x[k] - most;
        const bool is = one && x[k] == most;
        const float e = is ? 0.0f : exp_of(u);
        one = one && !is;
        now.others += e;
        now.moment += fmaxf(u, kNothing) * e;
    }
    p = join(p, now);
}

// Over the lanes of a wave, in all of them.
__device__ __forceinline__ Part join_lanes(Part p)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const Part other{__shfl_xor(p.max, d), __shfl_xor(p.others, d), __shfl_xor(p.moment, d)};
        const bool upper = threadIdx.x & d;         // both lanes join the same two in the same order
        p = upper ? join(other, p) : join(p, other);
    }
    return p;
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

constexpr int kList = 256, kListEach = kList / kWave;

// A wave's.
struct Largest {
    Place *list;
    int count, n_top;
    Place least;                                    // what is not above it is not among the largest

    __device__ __forceinline__ void begin(Place *lds, int n)
    {
        list = lds;
        count = 0;
        n_top = n;
        least = 0;
    }

    // The list's n_top largest, in descending order, at its beginning.
    __device__ __forceinline__ void cut()
    {
        const int lane = threadIdx.x % kWave;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        Place mine[kListEach];
        int above[kListEach];
#pragma unroll
        for (int i = 0; i < kListEach; ++i) {
            mine[i] = i * kWave + lane < count ? list[i * kWave + lane] : 0;
            above[i] = 0;
        }
        for (int j = 0; j < count; ++j) {
            const Place other = list[j];
#pragma unroll
            for (int i = 0; i < kListEach; ++i) above[i] += other > mine[i] ? 1 : 0;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < kListEach; ++i)
            if (i * kWave + lane < count && above[i] < n_top) list[above[i]] = mine[i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        count = min(count, n_top);
        if (count == n_top) least = list[n_top - 1];
    }

    // One place of each lane that has one.
    __device__ __forceinline__ void add(Place place, bool has)
    {
        has = has && place > least;
        uint64_t with = __ballot(has);
        if (!with) return;
        if (count + __popcll(with) > kList) {
            cut();
            has = has && place > least;
            with = __ballot(has);
        }
        if (has) list[count + __popcll(with & (((uint64_t)1 << threadIdx.x % kWave) - 1))] = place;
        count += __popcll(with);
    }
};

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

// What a row's part and largest come to: by the first threads of those that hold them.
template <typename T>
__device__ __forceinline__ void store_row(const ProbArgs &a, int64_t row, const Part &p, int thread, const Place *largest)
{
    const bool none = !is_part(p), bad = !(p.max < __builtin_inff()) && !none;
    const float rest = bad ? __builtin_nanf("") : none ? 0.0f : log1pf(p.others);
    if (thread == 0) {
        if (a.stats) {
            a.stats[row * 2] = p.max;
            a.stats[row * 2 + 1] = rest;
        }
        if (a.entropy) a.entropy[row] = rest - (bad ? rest : p.moment / (1.0f + p.others));
        if (a.logp) {
            const int32_t t = a.targets[row];
            float v = 0.0f;
            if (t >= 0 && t < a.n_classes) v = none ? -__builtin_inff() : (one_logit<T>(a, row, t) - p.max) - rest;
            a.logp[row] = v;
        }
    }
    if (thread < a.n_top) {
        const Place place = largest[thread];
        a.top_class[row * a.n_top + thread] = (int32_t)~(uint32_t)place;
        a.top_logp[row * a.n_top + thread] = none ? -__builtin_inff() : (key_value((uint32_t)(place >> 32)) - p.max) - rest;
    }
}

// A part of a row by a workgroup of WAVES waves, each of which has a contiguous share.
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void logprob_kernel(ProbArgs a)
{
    __shared__ Place lists[WAVES][kList];
    __shared__ Part parts[WAVES];
    __shared__ int counts[WAVES];
    const uint64_t at = workgroup();
    const int64_t row = at / (uint32_t)a.splits;
    if (row >= a.n_rows) return;
    const int32_t split = (int32_t)(at - row * a.splits), first = split * a.per_split, last = (int32_t)min((int64_t)first + a.per_split, (int64_t)a.n_classes);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int32_t share = ((last - first + WAVES - 1) / WAVES + 7) / 8 * 8, begin = min(first + wave * share, last), end = min(begin + share, last);
    Part p = no_part();
    Largest largest;
    largest.begin(lists[wave], a.n_top);
    for (int32_t col0 = begin; col0 < end; col0 += kWave * 8) {
        const int32_t col = col0 + lane * 8;
        float x[8];
        if (col < end) load_piece<T, 8>((const T *)a.logits, row * a.ld + col, end - col, a.span, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = col + k < end ? x[k] : -__builtin_inff();
        add_logits<8>(p, x);
        if (a.n_top) {
#pragma unroll
            for (int k = 0; k < 8; ++k) largest.add(place_of(x[k], (uint32_t)(col + k)), col + k < end);
        }
    }
    p = join_lanes(p);
    if (a.n_top) largest.cut();
    if (lane == 0) {
        parts[wave] = p;
        counts[wave] = largest.count;
    }
    __syncthreads();
    if (wave != 0) return;
    p = parts[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) p = join(p, parts[w]);
    if (a.n_top)
        for (int w = 1; w < WAVES; ++w) {
            const int n = counts[w];
            largest.add(lane < n ? lists[w][lane] : 0, lane < n);
        }
    if (a.n_top) largest.cut();
    if (a.splits == 1) {
        store_row<T>(a, row, p, lane, lists[0]);
        return;
    }
    if (lane == 0) a.parts[row * a.splits + split] = p;
    if (lane < a.n_top) a.places[(row * a.splits + split) * a.n_top + lane] = lane < largest.count ? lists[0][lane] : 0;
}

// The splits of a row, a wave.
template <typename T>
__global__ __launch_bounds__(kWave) void logprob_join_kernel(ProbArgs a)
{
    __shared__ Place list[kList];
    const int64_t row = workgroup();
    if (row >= a.n_rows) return;
    const int lane = threadIdx.x;
    Part p = no_part();
    for (int32_t s = lane; s < a.splits; s += kWave) p = join(p, a.parts[row * a.splits + s]);
    p = join_lanes(p);
    Largest largest;
    largest.begin(list, a.n_top);
    if (a.n_top) {
        const int32_t n = a.splits * a.n_top;
        for (int32_t i = 0; i < n; i += kWave) {
            const Place place = i + lane < n ? a.places[row * n + i + lane] : 0;
            largest.add(place, place != 0);
        }
        largest.cut();
    }
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

template <typename T>
hipError_t launch_forward(const ProbArgs &a, hipStream_t st)
{
    if (a.n_classes <= 2048) logprob_kernel<T, 1><<<grid_of(a.n_rows * a.splits, kWave), kWave, 0, st>>>(a);
    else                     logprob_kernel<T, 4><<<grid_of(a.n_rows * a.splits, kBlock), kBlock, 0, st>>>(a);
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

template <typename T>
__global__ __launch_bounds__(kBlock) void logprob_gradient_kernel(ProbGradArgs a)
{
    constexpr int kEach = 2;
    const uint64_t first = (uint64_t)workgroup() * (kBlock * kEach) + threadIdx.x;
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
        if (first + e * kBlock < a.pieces) store_piece<T, 8>((T *)a.dlogits + row[e] * a.ldd + col[e], a.written - col[e], d);
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
    if (type == ADAQP_F32) logprob_gradient_kernel<float><<<grid, kBlock, 0, (hipStream_t)stream>>>(a);
    else                   logprob_gradient_kernel<__bf16><<<grid, kBlock, 0, (hipStream_t)stream>>>(a);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}
