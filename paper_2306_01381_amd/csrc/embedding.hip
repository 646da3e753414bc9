// Embedding (adaqp_train.h): rows of a table by their ids, a stable sort of ids, and the table's gradient along the sorted ids.
//
// Lookup: a lane has pieces of 8 columns of the output's rows; a wave's lanes read neighbouring pieces of the same table row or of a few.  Bound by memory: 131 072 rows of 50 000 x 1024 fp32 137 us (537 MB
// written, the table read once or more), 512 of bf16 3.7 us.
//
// Sort, of few ids by counting those before each (sort_few_kernel); of more, least significant digit first, at most kMostDigitBits bits a pass, as many passes as the table's size needs.  A pass counts each digit in
// blocks of kSortItems ids and then deals the ids out: a wave takes 64 ids at a time and finds the lanes with its digit by a ballot for each bit, so that equal digits keep their order.  No atomics but the
// counts', which are whole numbers.  Bound by waits, of which each launch is a chain.  us by ids, 20 000 and 50 000 entries: 64 2.8, 4096 5.6, 9001 14, 12 288 18, then by digits 16 000 22, 131 072 25, 306 000 51 (456 000 entries, three
// passes).  One workgroup with all ids in its LDS, pass after pass, took 19 at 9001.
//
// Gradient: the sorted places are cut into chunks.  A group of lanes walks a chunk, adds the rows of equal ids in registers and stores the sum of every run that lies in
// its chunk; of the runs that go on it leaves the parts (the first run's as the chunk's head, the last one's as its tail), and a second kernel adds a tail and the heads
// behind it; where entries have very many ids each one between them adds heads by blocks of 64.  Entries without a row are found by a search of the sorted ids, 64 places a step, and set to zero beside it in the same launch.  Bound by memory: 131 072 ids, 50 000 x 1024 fp32, 142 us (742 MB, 5.2 TB/s; 178 where the
// gradient's rows, which are read once, go through the caches) and 14 for the second kernel, whose longest run has 380 heads; 9001 ids, 20 000 x 301 bf16, 10.7 and 5 us, a chain of waits.  Added to the table instead,
// both launches: 148 us (147 whole) and 17 (18); 306 000 ids of 456 000 x 64, a fifth of them named, 54 (68: the others are not set to zero); 58 000 x 256, each named once, 44 (30: the table is read, too).
#include "adaqp_train.h"
#include "rows.hpp"

namespace adaqp {
namespace {

constexpr int64_t kMostIds = (int64_t)1 << 31;

// ---- lookup ------------------------------------------------------------------------------------------------------------------------------

struct LookArgs {
    const void *table;
    const int32_t *ids;
    void *out;
    int64_t ldt, ldo, span, n_entries;
    uint64_t pieces;
    Divider pieces_of_row;
    int32_t dim, written;
    float scale;
};

template <typename E, typename T, bool ONCE>
__global__ __launch_bounds__(kBlock) void lookup_kernel(LookArgs a)
{
    constexpr int kEach = 2;
    const uint64_t first = (uint64_t)workgroup() * (kBlock * kEach) + threadIdx.x;
    int64_t row[kEach], id[kEach];
    int32_t col[kEach];
    float x[kEach][8];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint64_t at = min(first + e * kBlock, a.pieces - 1);
        row[e] = a.pieces_of_row.quotient(at);
        col[e] = (int32_t)(at - (uint64_t)row[e] * a.pieces_of_row.by) * 8;
        id[e] = a.ids[row[e]];
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const bool there = id[e] >= 0 && id[e] < a.n_entries && col[e] < a.dim;
        if (there) load_piece<E, 8>((const E *)a.table, id[e] * a.ldt + col[e], a.dim - col[e], a.span, x[e]);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[e][k] = there && col[e] + k < a.dim ? x[e][k] * a.scale : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e)
        if (first + e * kBlock < a.pieces) store_piece<T, 8, ONCE>((T *)a.out + row[e] * a.ldo + col[e], a.written - col[e], x[e]);
}

// ---- sort --------------------------------------------------------------------------------------------------------------------------------

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave, kSortEach = 4, kSortItems = kSortThreads * kSortEach;
constexpr int kMostDigitBits = 9, kMostDigits = 1 << kMostDigitBits;
static_assert(2 * kMostDigits == kSortThreads, "two threads have a digit");
constexpr int kFewSortBlocks = 64;                  // up to here every block adds up the counts before its own by itself

struct SortPass {
    const int32_t *ids;                             // of the first pass; NULL: keys and places
    const uint32_t *keys;
    const int32_t *places;
    int32_t *keys_out, *places_out;
    int64_t n, n_entries;
    uint32_t *counts;                               // [blocks][digits]; offsets once they are added up
    uint32_t *totals;                               // [digits], where they are added up by a kernel of its own
    int32_t blocks;
    int shift, bits;
};

__device__ __forceinline__ uint32_t sort_key(const SortPass &p, int64_t at)
{
    if (!p.ids) return p.keys[at];
    const int32_t id = p.ids[at];
    return id >= 0 && id < p.n_entries ? (uint32_t)id : (uint32_t)p.n_entries;
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p)
{
    __shared__ uint32_t count[kMostDigits];
    const uint32_t mask = (1u << p.bits) - 1;
    if (threadIdx.x < kMostDigits) count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * kSortItems;
    uint32_t key[kSortEach];
#pragma unroll
    for (int e = 0; e < kSortEach; ++e) {
        const int64_t at = begin + e * kSortThreads + threadIdx.x;
        key[e] = at < p.n ? sort_key(p, at) : 0;
    }
#pragma unroll
    for (int e = 0; e < kSortEach; ++e)
        if (begin + e * kSortThreads + threadIdx.x < p.n) atomicAdd(&count[key[e] >> p.shift & mask], 1u);
    __syncthreads();
    if (threadIdx.x <= mask) p.counts[(int64_t)blockIdx.x * (mask + 1) + threadIdx.x] = count[threadIdx.x];
}

// Counts to the sums of those before them, digit by digit; totals.  A workgroup has 64 digits, a wave a share of the blocks.
constexpr int kScanThreads = 1024, kScanWaves = kScanThreads / kWave;

__global__ __launch_bounds__(kScanThreads) void sort_scan_kernel(SortPass p)
{
    __shared__ uint32_t part[kScanWaves][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const uint32_t digits = 1u << p.bits, digit = blockIdx.x * kWave + lane;
    const int32_t share = (p.blocks + kScanWaves - 1) / kScanWaves, begin = min(wave * share, p.blocks), end = min(begin + share, p.blocks);
    uint32_t sum = 0;
    if (digit < digits)
#pragma unroll 8
        for (int32_t b = begin; b < end; ++b) sum += p.counts[(int64_t)b * digits + digit];
    part[wave][lane] = sum;
    __syncthreads();
    if (digit >= digits) return;
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w) {
        before += w < wave ? part[w][lane] : 0;
        total += part[w][lane];
    }
    if (wave == 0) p.totals[digit] = total;
#pragma unroll 8
    for (int32_t b = begin; b < end; ++b) {
        const uint32_t c = p.counts[(int64_t)b * digits + digit];
        p.counts[(int64_t)b * digits + digit] = before;
        before += c;
    }
}

// The sum over the threads before this one, of a workgroup of WAVES waves.
template <int WAVES>
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t *lds)
{
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t from = __shfl_up(sum, d);
        if (lane >= d) sum += from;
    }
    if (lane == kWave - 1) lds[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) before += w < wave ? lds[w] : 0;
    return before + sum - v;
}

// How many ids with this one's digit the wave had so far, those of lower lanes among them; count: the wave's, by digit.
__device__ __forceinline__ uint32_t rank_in_wave(uint32_t *count, uint32_t digit, int bits, bool there)
{
    const uint64_t all = __ballot(there);
    uint32_t low = (uint32_t)all, high = (uint32_t)(all >> 32);
#pragma unroll
    for (int b = 0; b < kMostDigitBits; ++b)
        if (b < bits) {
            const int32_t set = (int32_t)(digit << (31 - b)) >> 31;            // all bits, or none
            const uint64_t with = __ballot(set != 0);
            low = __builtin_amdgcn_bitop3_b32(low, (uint32_t)with, (uint32_t)set, 0x90);                   // low & ~(with ^ set)
            high = __builtin_amdgcn_bitop3_b32(high, (uint32_t)(with >> 32), (uint32_t)set, 0x90);
        }
    const uint64_t same = (uint64_t)high << 32 | low;
    const uint64_t lower = same & (((uint64_t)1 << threadIdx.x % kWave) - 1);
    const uint32_t so_far = count[digit];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (there && lower == 0) count[digit] = so_far + (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return so_far + (uint32_t)__popcll(lower);
}

// Few ids: each one's place is the number of those before it, counted.  A workgroup has kCountItems ids and all to compare with in the LDS; its threads share those: thread t has id t mod kCountItems
// and part t / kCountItems of the others.
constexpr int kCountThreads = 1024, kCountItems = 16, kCountSlices = kCountThreads / kCountItems;
constexpr int kFewIds = 12288;

__global__ __launch_bounds__(kCountThreads) void sort_few_kernel(const int32_t *ids, int32_t n, uint32_t n_entries, int32_t *sorted, int32_t *order)
{
    __shared__ uint4 keys[kFewIds / 4];
    __shared__ int32_t part[kCountSlices][kCountItems];
    const int slice = threadIdx.x / kCountItems;
    const int32_t first = blockIdx.x * kCountItems, mine = first + threadIdx.x % kCountItems;
    const int32_t share = ((n + kCountSlices - 1) / kCountSlices + 3) / 4, all = share * kCountSlices;     // in fours; at most kFewIds / 4
    const int32_t begin = slice * share, end = begin + share;
    constexpr int kLoads = kFewIds / 4 / kCountThreads;
    uint32_t v[kLoads][4];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int32_t j = (i * kCountThreads + threadIdx.x) * 4;
        if (j + 4 <= n) {
            const auto four = reinterpret_cast<const loose_of<int32_t, 4> *>(ids + j)->v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = (uint32_t)four[k];
        } else
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = j + k < n ? (uint32_t)ids[j + k] : 0;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int32_t j = i * kCountThreads + threadIdx.x;
        if (j < all) {                              // below zero is large
            auto one = [&](int k) { return j * 4 + k < n ? min(v[i][k], n_entries) : 0x7FFFFFFFu; };      // behind the last: below none
            keys[j] = make_uint4(one(0), one(1), one(2), one(3));
        }
    }
    __syncthreads();
    const uint32_t *flat = reinterpret_cast<const uint32_t *>(keys);
    const uint32_t key = flat[min(mine, n - 1)];
    int32_t before = 0;
    // Of the fours from `at` on: below 2^31 both, k < bound is the sign of k - bound, and 32 of those make a word.
    auto count = [&](int32_t at, int32_t end, uint32_t bound) {
        auto four = [&](uint32_t word, int32_t j) {
            const uint4 k = keys[j];
            word = __builtin_amdgcn_alignbit(word, k.x - bound, 31);
            word = __builtin_amdgcn_alignbit(word, k.y - bound, 31);
            word = __builtin_amdgcn_alignbit(word, k.z - bound, 31);
            return __builtin_amdgcn_alignbit(word, k.w - bound, 31);
        };
        for (; at + 8 <= end; at += 8) {
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) word = four(word, at + i);
            before += __popc(word);
        }
        for (; at < end; ++at) before += __popc(four(0, at));
    };
    // in the workgroup's own ids equal ones are before an id if their place is; in those below all are, above none
    const int32_t own = min(max(first / 4, begin), end), above = min(max((first + kCountItems) / 4, begin), end);
    count(begin, own, key + 1);
    for (int32_t j = own * 4; j < above * 4; ++j) before += flat[j] < (j < mine ? key + 1 : key) ? 1 : 0;
    count(above, end, key);
    part[slice][threadIdx.x % kCountItems] = before;
    __syncthreads();
    if (threadIdx.x >= kCountItems || mine >= n) return;
    int32_t to = 0;
#pragma unroll
    for (int i = 0; i < kCountSlices; ++i) to += part[i][threadIdx.x];
    sorted[to] = (int32_t)key;
    order[to] = mine;
}

__global__ __launch_bounds__(kSortThreads) void sort_deal_kernel(SortPass p)
{
    __shared__ uint32_t count[kSortWaves][kMostDigits];        // of a wave's own ids; then where they go
    __shared__ uint32_t scan[kSortWaves], other[kMostDigits][2];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const uint32_t mask = (1u << p.bits) - 1;
    const int64_t begin = (int64_t)blockIdx.x * kSortItems + wave * (kSortItems / kSortWaves);
    uint32_t key[kSortEach], rank[kSortEach];
    int32_t place[kSortEach];
#pragma unroll
    for (int e = 0; e < kSortEach; ++e) {
        const int64_t at = begin + e * kWave + lane;
        key[e] = at < p.n ? sort_key(p, at) : 0;
        place[e] = at < p.n ? (p.ids ? (int32_t)at : p.places[at]) : 0;
    }
    // this thread's digit: how many of it lie in the blocks before, and in all; two threads share the blocks
    const uint32_t digit = threadIdx.x % kMostDigits;
    uint32_t before = 0, total = 0;
    if (digit <= mask) {
        const uint32_t *of_digit = p.counts + digit;
        if (p.totals) {
            before = of_digit[(int64_t)blockIdx.x * (mask + 1)];
            total = p.totals[digit];
        } else {
            constexpr int kAtOnce = 16;
            for (int32_t b0 = threadIdx.x / kMostDigits; b0 < p.blocks; b0 += 2 * kAtOnce) {
                uint32_t c[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) c[i] = of_digit[(int64_t)min(b0 + 2 * i, p.blocks - 1) * (mask + 1)];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    before += b0 + 2 * i < (int32_t)blockIdx.x ? c[i] : 0;
                    total += b0 + 2 * i < p.blocks ? c[i] : 0;
                }
            }
        }
    }
    for (int i = threadIdx.x; i < kSortWaves * kMostDigits; i += kSortThreads) (&count[0][0])[i] = 0;
    if (threadIdx.x >= kMostDigits) {
        other[digit][0] = before;
        other[digit][1] = total;
    }
    __syncthreads();
    if (threadIdx.x < kMostDigits) {
        if (!p.totals) {
            before += other[digit][0];
            total += other[digit][1];
        }
    } else total = 0;
    before += sum_before<kSortWaves>(total, scan);
#pragma unroll
    for (int e = 0; e < kSortEach; ++e) rank[e] = rank_in_wave(count[wave], key[e] >> p.shift & mask, p.bits, begin + e * kWave + lane < p.n);
    __syncthreads();
    if (threadIdx.x < kMostDigits)
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = count[w][threadIdx.x];
            count[w][threadIdx.x] = before;
            before += c;
        }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kSortEach; ++e)
        if (begin + e * kWave + lane < p.n) {
            const uint32_t to = count[wave][key[e] >> p.shift & mask] + rank[e];
            p.keys_out[to] = (int32_t)key[e];
            p.places_out[to] = place[e];
        }
}

struct SortShape {
    int passes, bits_of_pass;
    int64_t blocks, bytes_keys, bytes_counts, bytes;
};

SortShape sort_shape(int64_t n_ids, int64_t n_entries)
{
    SortShape s{};
    int bits = 1;
    while ((n_entries >> bits) != 0) ++bits;        // of the largest key, n_entries
    s.passes = (bits + kMostDigitBits - 1) / kMostDigitBits;
    s.bits_of_pass = (bits + s.passes - 1) / s.passes;
    s.blocks = (n_ids + kSortItems - 1) / kSortItems;
    s.bytes_keys = s.passes > 1 ? (n_ids * 4 + 255) / 256 * 256 : 0;
    s.bytes_counts = ((s.blocks + 1) * ((int64_t)4 << s.bits_of_pass) + 255) / 256 * 256;
    s.bytes = n_ids > 0 ? 2 * s.bytes_keys + s.bytes_counts : 0;
    return s;
}

// ---- gradient ----------------------------------------------------------------------------------------------------------------------------

constexpr int kLongChunk = 32, kShortChunk = 8;

struct GradArgs {
    const void *dy;
    const int32_t *sorted, *order;
    float *dtable, *parts;                          // [chunks][head, tail][pitch]
    float *block_parts;                             // [chunks / kBlockChunks][pitch]; NULL: there are too few
    int64_t lddy, ldd, span, n_ids, n_entries, chunks, pitch;
    int64_t run_blocks;                             // workgroups that walk chunks; those behind them set entries to zero
    int32_t dim, written;                           // columns of dy; of dtable's rows that are written
    int32_t slabs, chunk;                           // places of a chunk
    int32_t clear;                                  // entries that a wave sets to zero where no id names them
    float scale;
    int accumulate;
};

// Of LANES lanes with V columns each, the runs of a chunk.
template <typename T, int LANES, int V, int CHUNK, bool ONCE>
__device__ __forceinline__ void walk_chunk(const GradArgs &a, int64_t chunk, int32_t col)
{
    constexpr int kAtOnce = 8, kHeld = LANES < CHUNK ? CHUNK / LANES : 1;
    const int64_t begin = chunk * CHUNK;
    const int n = (int)min((int64_t)CHUNK, a.n_ids - begin);
    const int lane = threadIdx.x % LANES, lane0 = threadIdx.x % kWave / LANES * LANES;
    // the chunk's ids and places, in the lanes
    int32_t held_id[kHeld], held_place[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int64_t at = begin + min(i * LANES + lane % CHUNK, n - 1);
        held_id[i] = a.sorted[at];
        held_place[i] = a.order[at];
    }
    auto held = [&](const int32_t (&v)[kHeld], int at) {
        int32_t mine = v[0];
#pragma unroll
        for (int i = 1; i < kHeld; ++i) mine = at / LANES == i ? v[i] : mine;
        if constexpr (LANES == kWave) return __builtin_amdgcn_readlane(mine, at);
        else                          return __shfl(mine, lane0 + at % LANES);
    };
    const int32_t id_before = begin > 0 ? a.sorted[begin - 1] : 0, id_behind = begin + n < a.n_ids ? a.sorted[begin + n] : 0;
    const int left = a.dim - col, left_written = a.written - col;
    float *head = a.parts + chunk * 2 * a.pitch + col;
    float sum[V];
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] = 0.0f;
    int32_t now = held(held_id, 0);
    bool first = begin > 0 && id_before == now;     // the run goes on from the chunk before
    auto leave = [&](bool goes_on) {
        if (first || goes_on) store_piece<float, V>(head + (first ? 0 : a.pitch), left, sum);
        else if (now >= 0 && now < a.n_entries) {
            float *to = a.dtable + now * a.ldd + col;
            float v[V];
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = k < left ? sum[k] * a.scale : 0.0f;
            if (a.accumulate)
#pragma unroll
                for (int k = 0; k < V; ++k) v[k] += k < left ? to[k] : 0.0f;
            store_piece<float, V>(to, a.accumulate ? left : left_written, v);
        }
    };
    for (int at = 0; at < n; at += kAtOnce) {
        int32_t id[kAtOnce];
        float v[kAtOnce][V];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int p = min(at + u, n - 1);
            id[u] = held(held_id, p);
            const int64_t place = held(held_place, p);
            const bool there = at + u < n && place >= 0 && place < a.n_ids && left > 0 && id[u] < a.n_entries;
            if (there) load_piece<T, V, ONCE>((const T *)a.dy, place * a.lddy + col, left, a.span, v[u]);
#pragma unroll
            for (int k = 0; k < V; ++k) v[u][k] = there ? v[u][k] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (id[u] != now) {
                leave(false);
                first = false;
                now = id[u];
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += v[u][k];
        }
    }
    leave(begin + n < a.n_ids && id_behind == now);
}

// How many sorted ids are below each of two bounds, by a wave: it looks at 64 at a time.
__device__ __forceinline__ void places_below(const int32_t *sorted, int64_t n, int64_t bound_a, int64_t bound_b, int64_t &a, int64_t &b)
{
    const int lane = threadIdx.x % kWave;
    a = b = 0;                                      // so many are below for certain; of the `left` behind them perhaps
    for (int64_t left = n; left > 0;) {
        const int64_t step = (left + kWave - 1) / kWave;
        const int64_t at_a = a + (lane + 1) * step - 1, at_b = b + (lane + 1) * step - 1;
        const bool below_a = at_a < n && sorted[min(at_a, n - 1)] < bound_a, below_b = at_b < n && sorted[min(at_b, n - 1)] < bound_b;
        a += __popcll(__ballot(below_a)) * step;
        b += __popcll(__ballot(below_b)) * step;
        left = step - 1;                            // the next one that was looked at is not below
    }
}

// Zeros in the entries of a wave's a.clear, at most 64, that no id names.
__device__ __forceinline__ void clear_entries(const GradArgs &a, int64_t tile, uint8_t *named)
{
    const int lane = threadIdx.x % kWave;
    const int64_t entry0 = tile * a.clear, entry = entry0 + lane;
    if (entry0 >= a.n_entries) return;
    int64_t begin, end;                             // places of the tile's ids
    places_below(a.sorted, a.n_ids, entry0, entry0 + a.clear, begin, end);
    bool is_named = false;
    if (end - begin <= kWave) {
        named[lane] = 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (begin + lane < end) named[a.sorted[begin + lane] - entry0 & (kWave - 1)] = 1;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        is_named = named[lane];
    } else {
        while (begin < end) {                       // the first place of an id that is not below entry
            const int64_t mid = (begin + end) / 2;
            if (a.sorted[mid] < entry) begin = mid + 1;
            else                       end = mid;
        }
        is_named = begin < a.n_ids && a.sorted[begin] == entry;
    }
    uint64_t absent = __ballot(lane < a.clear && entry < a.n_entries && !is_named);
    const float zeros[4] = {};
    while (absent) {
        const int64_t at = entry0 + __builtin_ctzll(absent);
        absent &= absent - 1;
        for (int32_t col = lane * 4; col < a.written; col += kWave * 4) store_piece<float, 4>(a.dtable + at * a.ldd + col, a.written - col, zeros);
    }
}

template <typename T, int LANES, int V, int CHUNK, bool ONCE>
__global__ __launch_bounds__(kBlock) void embedding_runs_kernel(GradArgs a)
{
    __shared__ uint8_t named[kWavesPerBlock][kWave];
    const int64_t at = workgroup();
    if (at >= a.run_blocks) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        if (!a.accumulate) clear_entries(a, (at - a.run_blocks) * kWavesPerBlock + wave, named[wave]);
        return;
    }
    // neighbouring groups have a chunk's slabs: they read the same rows at a time
    constexpr int kGroups = kBlock / LANES;
    const int group = LANES == kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : threadIdx.x / LANES;
    const int64_t flat = at * kGroups + group, chunk = flat / a.slabs, slab = flat - chunk * a.slabs;
    if (chunk < a.chunks) walk_chunk<T, LANES, V, CHUNK, ONCE>(a, chunk, (int32_t)(slab * LANES + threadIdx.x % LANES) * V);       // lanes behind the columns, too: they hold ids
}

constexpr int kBlockChunks = 64;                    // chunks whose heads are added together where one run covers them all

constexpr int kJoinWaves = 8, kJoinCols = kWave * 4, kFewHeads = 16;

// Adds rows begin, begin + step, ... up to last of `from`, of a pitch in floats, in turn.
__device__ __forceinline__ void add_rows(const float *from, int64_t pitch, int64_t begin, int64_t last, int step, float (&sum)[4])
{
    constexpr int kAtOnce = 8;
    for (int64_t c = begin; c <= last; c += step * kAtOnce) {
        float v[kAtOnce][4];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            load_elements<float, 4>(from + min(c + u * step, last) * pitch, v[u]);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[u][k] = c + u * step <= last ? v[u][k] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += v[u][k];
    }
}

// Of chunks [kBlockChunks b, kBlockChunks (b + 1)) that all begin inside the same run, the sum of their heads: few ids with very many places each would leave the next kernel thousands of heads to add in turn.
__global__ __launch_bounds__(kJoinWaves * kWave) void embedding_blocks_kernel(GradArgs a)
{
    __shared__ float part[kJoinWaves][kJoinCols];
    const int64_t at = workgroup(), slab = at % a.slabs, block = at / a.slabs, chunk = block * kBlockChunks;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (chunk + kBlockChunks > a.chunks || chunk == 0) return;
    const int32_t id = a.sorted[chunk * a.chunk];
    if (a.sorted[chunk * a.chunk - 1] != id || a.sorted[(chunk + kBlockChunks - 1) * a.chunk] != id) return;
    const int32_t col = (int32_t)slab * kJoinCols + lane * 4;
    float sum[4] = {};
    if (col < a.dim) add_rows(a.parts + col, 2 * a.pitch, chunk + wave, chunk + kBlockChunks - 1, kJoinWaves, sum);
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][k * kWave + lane] = sum[k];
    __syncthreads();
    if (wave != 0 || col >= a.dim) return;
    float v[4] = {};
#pragma unroll
    for (int i = 0; i < kJoinWaves; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += part[i][k * kWave + lane];
    store_elements<float, 4, false>(a.block_parts + block * a.pitch + col, v);
}

// Of each run that begins in a chunk and goes on behind it: the chunk's tail and the heads of the chunks that it covers, those of whole blocks together.  A wave has a chunk; where the heads are many all waves of
// the workgroup share them.
template <bool BLOCKS>
__global__ __launch_bounds__(kJoinWaves * kWave) void embedding_join_kernel(GradArgs a)
{
    __shared__ float part[kJoinWaves][kJoinCols];
    __shared__ int64_t last_of[kJoinWaves];         // the last chunk of a run with many heads; 0: there is none
    const int64_t at = workgroup(), slab = at % a.slabs, chunk0 = at / a.slabs * kJoinWaves;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int32_t col = (int32_t)slab * kJoinCols + lane * 4;
    const int left = a.dim - col;
    const float *heads = a.parts + col;
    // of the heads begin .. last every step-th from the first-th on
    auto sum_heads = [&](int64_t begin, int64_t last, int first, int step, float (&sum)[4]) {
        const int64_t block = (begin + kBlockChunks - 1) / kBlockChunks, blocks = (last + 1) / kBlockChunks;
        if (!BLOCKS || block >= blocks) {
            add_rows(heads, 2 * a.pitch, begin + first, last, step, sum);
            return;
        }
        add_rows(heads, 2 * a.pitch, begin + first, block * kBlockChunks - 1, step, sum);
        add_rows(a.block_parts + col, a.pitch, block + first, blocks - 1, step, sum);
        add_rows(heads, 2 * a.pitch, blocks * kBlockChunks + first, last, step, sum);
    };
    auto store = [&](int32_t id, float (&v)[4]) {
        if (col >= a.written) return;
        float *to = a.dtable + id * a.ldd + col;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = k < left ? v[k] * a.scale : 0.0f;
            if (a.accumulate && k < left) v[k] += to[k];
        }
        store_piece<float, 4>(to, a.accumulate ? left : a.written - col, v);
    };
    {
        const int64_t chunk = chunk0 + wave, end = (chunk + 1) * a.chunk;       // end of the chunk's places
        int64_t last = 0;
        if (end < a.n_ids) {
            const int32_t id = a.sorted[end - 1], behind = a.sorted[end], begins = a.sorted[chunk * a.chunk], before = chunk > 0 ? a.sorted[chunk * a.chunk - 1] : 0;
            const bool own = behind == id && id >= 0 && id < a.n_entries && !(chunk > 0 && begins == id && before == id);      // a run that begins here and goes on
            if (own) {
                last = chunk;                       // of the chunks that begin with the id
                for (;;) {
                    const int64_t place = (last + 1 + lane) * a.chunk;
                    const uint64_t with = __ballot(place < a.n_ids && a.sorted[min(place, a.n_ids - 1)] == id);
                    const int n = with == ~(uint64_t)0 ? kWave : __builtin_ctzll(~with);
                    last += n;
                    if (n < kWave) break;
                }
                if (last - chunk <= kFewHeads) {
                    float v[4] = {};
                    if (left > 0) {
                        load_elements<float, 4>(heads + (chunk * 2 + 1) * a.pitch, v);
                        sum_heads(chunk + 1, last, 0, 1, v);
                    }
                    store(id, v);
                    last = 0;
                }
            }
        }
        if (lane == 0) last_of[wave] = last;
    }
    __syncthreads();
    for (int w = 0; w < kJoinWaves; ++w) {
        const int64_t chunk = chunk0 + w, last = last_of[w];
        if (last == 0) continue;
        float sum[4] = {};
        if (left > 0) sum_heads(chunk + 1, last, wave, kJoinWaves, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k) part[wave][k * kWave + lane] = sum[k];
        __syncthreads();
        if (wave == w) {
            float v[4] = {};
            if (left > 0) load_elements<float, 4>(heads + (chunk * 2 + 1) * a.pitch, v);
#pragma unroll
            for (int i = 0; i < kJoinWaves; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += part[i][k * kWave + lane];
            store(a.sorted[(chunk + 1) * a.chunk - 1], v);
        }
        __syncthreads();
    }
}

// Entries of a wave that clears: 20 000 x 301 with 9001 ids 23 us with 64, 16 with 16; 456 000 x 64 with 306 000 ids 48 with 64, 54 with 16.
constexpr int32_t kFewClear = 16;

// Where long chunks would leave SIMDs without a wave, short ones.
int32_t grad_chunk(int64_t n_ids, int32_t dim) { return (n_ids + kLongChunk - 1) / kLongChunk * (((int64_t)dim + 255) / 256) < 4096 ? kShortChunk : kLongChunk; }
int64_t grad_chunks(int64_t n_ids, int32_t dim) { return (n_ids + grad_chunk(n_ids, dim) - 1) / grad_chunk(n_ids, dim); }
int64_t grad_pitch(int32_t dim) { return ((int64_t)dim + 7) / 8 * 8; }
// Blocks of chunks: the workspace has room for them from 2048 chunks on.
int64_t grad_blocks(int64_t n_ids, int32_t dim) { return grad_chunks(n_ids, dim) < 2048 ? 0 : grad_chunks(n_ids, dim) / kBlockChunks; }

// Ids for each entry from which on the blocks have a launch of their own: the places of a block.  Without and with, fp32: 65 536 ids of 10 entries x 256 53 and 37 us, 131 072 of 40 x 1024
// 113 and 111; of 256 x 1024 110 and 113, of 50 000 x 1024 147 and 153.  A large table with one very frequent id has none, since the host does not know the ids, and waits for the workgroups that add its
// heads: where one of 50 000 entries has half of the ids, 131 072 ids x 1024 take 166 (151 without it), 306 000 x 256 147 (87), 306 000 x 64 106 (41).  An id that stands for no entry is better outside the table.
constexpr int64_t kManyPlaces = kBlockChunks * kLongChunk;

template <typename T, int LANES>
void launch_runs(GradArgs &a, hipStream_t st)
{
    constexpr int V = 4, kGroups = kBlock / LANES;
    a.slabs = (a.written + LANES * V - 1) / (LANES * V);
    a.run_blocks = (a.chunks * a.slabs + kGroups - 1) / kGroups;
    const int64_t clear = a.accumulate ? 0 : ((a.n_entries + a.clear - 1) / a.clear + kWavesPerBlock - 1) / kWavesPerBlock;
    const dim3 grid = grid_of(a.run_blocks + clear, kBlock);
    if (a.chunk == kShortChunk)               embedding_runs_kernel<T, LANES, V, kShortChunk, false><<<grid, kBlock, 0, st>>>(a);
    else if (passes_caches(a.span, sizeof(T))) embedding_runs_kernel<T, LANES, V, kLongChunk, true><<<grid, kBlock, 0, st>>>(a);
    else                                      embedding_runs_kernel<T, LANES, V, kLongChunk, false><<<grid, kBlock, 0, st>>>(a);
}

template <typename T>
hipError_t launch_gradient(GradArgs a, hipStream_t st)
{
    const int64_t vectors = ((int64_t)a.written + 3) / 4;
    if (vectors <= 8)       launch_runs<T, 8>(a, st);
    else if (vectors <= 16) launch_runs<T, 16>(a, st);
    else if (vectors <= 32) launch_runs<T, 32>(a, st);
    else                    launch_runs<T, 64>(a, st);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.chunks < 2) return err;
    a.slabs = (a.written + kJoinCols - 1) / kJoinCols;
    if (a.block_parts) {
        embedding_blocks_kernel<<<grid_of(a.chunks / kBlockChunks * a.slabs, kJoinWaves * kWave), kJoinWaves * kWave, 0, st>>>(a);
        err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    const dim3 grid = grid_of((a.chunks - 1 + kJoinWaves - 1) / kJoinWaves * a.slabs, kJoinWaves * kWave);
    if (a.block_parts) embedding_join_kernel<true><<<grid, kJoinWaves * kWave, 0, st>>>(a);
    else               embedding_join_kernel<false><<<grid, kJoinWaves * kWave, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace
}  // namespace adaqp

using namespace adaqp;

extern "C" int adaqp_embedding_forward(const void *table_dev, int64_t ldt, int64_t n_entries, int32_t dim, int32_t table_type, const int32_t *ids_dev, int64_t n_ids,
                                       float scale, void *out_dev, int64_t ldo, int32_t type, void *stream)
{
    if (n_entries < 0 || n_ids < 0 || dim <= 0 || !valid_type(table_type) || !valid_type(type) || !(scale - scale == 0.0f)) return ADAQP_EINVAL;
    if (n_entries >= kMostIds || n_ids >= kMostIds || dim > kMostDim) return ADAQP_ESIZE;
    if (n_ids == 0) return ADAQP_OK;
    if (!ids_dev || !aligned_to(ids_dev, 4)) return ADAQP_EINVAL;
    if (n_entries > 0) ADAQP_TRY(check_rows(table_dev, ldt, dim, table_type));
    ADAQP_TRY(check_rows(out_dev, ldo, dim, type));
    if (!countable(n_entries, ldt) || !countable(n_ids, ldo)) return ADAQP_ESIZE;
    LookArgs a{};
    a.table = table_dev; a.ids = ids_dev; a.out = out_dev; a.ldt = ldt; a.ldo = ldo; a.n_entries = n_entries; a.dim = dim; a.scale = scale;
    a.span = matrix_span(n_entries, ldt, dim);
    a.written = (int32_t)columns_to_write(out_dev, ldo, dim, element_bytes(type));
    const int64_t each = ((int64_t)a.written + 7) / 8;
    if (n_ids > kMostWorkgroups * kBlock / each) return ADAQP_ESIZE;
    a.pieces = (uint64_t)(n_ids * each);
    a.pieces_of_row = divider(each, (int64_t)a.pieces);
    const dim3 grid = grid_of((int64_t)((a.pieces + 2 * kBlock - 1) / (2 * kBlock)), kBlock);
    const hipStream_t st = (hipStream_t)stream;
    auto go = [&](auto e, auto t) {
        if (passes_caches(n_ids * ldo, element_bytes(type))) lookup_kernel<decltype(e), decltype(t), true><<<grid, kBlock, 0, st>>>(a);
        else                                                 lookup_kernel<decltype(e), decltype(t), false><<<grid, kBlock, 0, st>>>(a);
    };
    if (table_type == ADAQP_F32 && type == ADAQP_F32) go(0.0f, 0.0f);
    else if (table_type == ADAQP_F32)                 go(0.0f, (__bf16)0.0f);
    else if (type == ADAQP_F32)                       go((__bf16)0.0f, 0.0f);
    else                                              go((__bf16)0.0f, (__bf16)0.0f);
    ADAQP_HIP_TRY(hipGetLastError());
    return ADAQP_OK;
}

extern "C" int adaqp_embedding_sort_workspace_bytes(int64_t n_ids, int64_t n_entries, int64_t *bytes_out)
{
    if (!bytes_out || n_ids < 0 || n_entries < 0) return ADAQP_EINVAL;
    if (n_entries >= kMostIds || n_ids >= kMostIds) return ADAQP_ESIZE;
    *bytes_out = sort_shape(n_ids, n_entries).bytes;
    return ADAQP_OK;
}

extern "C" int adaqp_embedding_sort(const int32_t *ids_dev, int64_t n_ids, int64_t n_entries, int32_t *sorted_dev, int32_t *order_dev,
                                    void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (n_ids < 0 || n_entries < 0) return ADAQP_EINVAL;
    if (n_entries >= kMostIds || n_ids >= kMostIds) return ADAQP_ESIZE;
    if (n_ids == 0) return ADAQP_OK;
    if (!ids_dev || !sorted_dev || !order_dev || !aligned_to(ids_dev, 4) || !aligned_to(sorted_dev, 4) || !aligned_to(order_dev, 4)) return ADAQP_EINVAL;
    if (sorted_dev == ids_dev || order_dev == ids_dev || sorted_dev == order_dev) return ADAQP_EINVAL;
    const SortShape s = sort_shape(n_ids, n_entries);
    if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
    if (workspace_bytes < s.bytes) return ADAQP_ESIZE;
    uint8_t *work = (uint8_t *)workspace_dev;
    const hipStream_t st = (hipStream_t)stream;
    if (n_ids <= kFewIds) {
        sort_few_kernel<<<dim3((uint32_t)((n_ids + kCountItems - 1) / kCountItems)), kCountThreads, 0, st>>>(ids_dev, (int32_t)n_ids, (uint32_t)n_entries, sorted_dev, order_dev);
        ADAQP_HIP_TRY(hipGetLastError());
        return ADAQP_OK;
    }
    const bool few = s.blocks <= kFewSortBlocks;
    SortPass p{};
    p.ids = ids_dev;
    p.n = n_ids;
    p.n_entries = n_entries;
    p.counts = (uint32_t *)(work + 2 * s.bytes_keys);
    p.blocks = (int32_t)s.blocks;
    p.bits = s.bits_of_pass;
    if (!few) p.totals = p.counts + (s.blocks << s.bits_of_pass);
    for (int i = 0; i < s.passes; ++i) {
        const bool to_outputs = (s.passes - 1 - i) % 2 == 0;
        p.keys_out = to_outputs ? sorted_dev : (int32_t *)work;
        p.places_out = to_outputs ? order_dev : (int32_t *)(work + s.bytes_keys);
        p.shift = i * s.bits_of_pass;
        sort_count_kernel<<<dim3((uint32_t)s.blocks), kSortThreads, 0, st>>>(p);
        if (!few) sort_scan_kernel<<<dim3(((1u << p.bits) + kWave - 1) / kWave), kScanThreads, 0, st>>>(p);
        sort_deal_kernel<<<dim3((uint32_t)s.blocks), kSortThreads, 0, st>>>(p);
        ADAQP_HIP_TRY(hipGetLastError());
        p.ids = nullptr;
        p.keys = (const uint32_t *)p.keys_out;
        p.places = p.places_out;
    }
    return ADAQP_OK;
}

extern "C" int adaqp_embedding_backward_workspace_bytes(int64_t n_ids, int32_t dim, int64_t *bytes_out)
{
    if (!bytes_out || n_ids < 0 || dim <= 0) return ADAQP_EINVAL;
    if (n_ids >= kMostIds || dim > kMostDim) return ADAQP_ESIZE;
    *bytes_out = n_ids > grad_chunk(n_ids, dim) ? ((grad_chunks(n_ids, dim) * 2 + grad_blocks(n_ids, dim)) * grad_pitch(dim) * 4 + 255) / 256 * 256 : 0;
    return ADAQP_OK;
}

extern "C" int adaqp_embedding_backward(const void *dy_dev, int64_t lddy, int64_t n_ids, int32_t dim, int32_t type, const int32_t *sorted_dev, const int32_t *order_dev,
                                        int64_t n_entries, float scale, int32_t accumulate, float *dtable_dev, int64_t ldd,
                                        void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (n_entries < 0 || n_ids < 0 || dim <= 0 || !valid_type(type) || !(scale - scale == 0.0f) || (accumulate != 0 && accumulate != 1)) return ADAQP_EINVAL;
    if (n_entries >= kMostIds || n_ids >= kMostIds || dim > kMostDim) return ADAQP_ESIZE;
    if (n_entries == 0 || (n_ids == 0 && accumulate)) return ADAQP_OK;
    ADAQP_TRY(check_rows(dtable_dev, ldd, dim, ADAQP_F32));
    int64_t need;
    ADAQP_TRY(adaqp_embedding_backward_workspace_bytes(n_ids, dim, &need));
    if (n_ids > 0) {
        ADAQP_TRY(check_rows(dy_dev, lddy, dim, type));
        if (!sorted_dev || !order_dev || !aligned_to(sorted_dev, 4) || !aligned_to(order_dev, 4)) return ADAQP_EINVAL;
        if (need > 0) {
            if (!workspace_dev || !aligned_to(workspace_dev, 256)) return ADAQP_EINVAL;
            if (workspace_bytes < need) return ADAQP_ESIZE;
        }
    }
    if (!countable(n_entries, ldd) || !countable(n_ids, lddy)) return ADAQP_ESIZE;
    GradArgs a{};
    a.dy = dy_dev; a.sorted = sorted_dev; a.order = order_dev; a.dtable = dtable_dev; a.parts = (float *)workspace_dev;
    a.lddy = lddy; a.ldd = ldd; a.n_ids = n_ids; a.n_entries = n_entries; a.dim = dim; a.scale = scale; a.accumulate = accumulate;
    a.span = matrix_span(n_ids, lddy, dim);
    a.chunk = grad_chunk(n_ids, dim);
    a.chunks = grad_chunks(n_ids, dim);
    a.pitch = grad_pitch(dim);
    const int64_t blocks = grad_blocks(n_ids, dim);
    a.block_parts = blocks > 0 && n_ids / n_entries >= kManyPlaces ? a.parts + a.chunks * 2 * a.pitch : nullptr;
    a.clear = dim >= 128 ? kFewClear : kWave;
    a.written = accumulate ? dim : (int32_t)columns_to_write(dtable_dev, ldd, dim, 4);
    if ((a.chunks + 1) * (((int64_t)a.written + kWave - 1) / kWave + 1) + a.n_entries / kFewClear >= kMostWorkgroups) return ADAQP_ESIZE;
    if (type == ADAQP_F32) ADAQP_HIP_TRY(launch_gradient<float>(a, (hipStream_t)stream));
    else                   ADAQP_HIP_TRY(launch_gradient<__bf16>(a, (hipStream_t)stream));
    return ADAQP_OK;
}
