// Embedding (adaqp_train.h): rows of a table by their ids, a stable sort of ids, and the table's gradient along the sorted ids.
//
// Lookup: a lane has pieces of 8 columns of the output's rows; a wave's lanes read neighbouring pieces of the same table row or of a few.
//
// Sort: least significant digit first, at most kMostDigitBits bits a pass, as many passes as the table's size needs.  A pass counts each digit in blocks of kSortItems ids and then
// deals the ids out: a wave takes 64 ids at a time and finds the lanes with its digit by a ballot for each bit, so that equal digits keep their order.  No atomics but
// the counts', which are whole numbers.
//
// Gradient: the sorted places are cut into chunks of kChunk.  A group of lanes walks a chunk, adds the rows of equal ids in registers and stores the sum of every run that lies in
// its chunk; of the runs that go on it leaves the parts (the first run's as the chunk's head, the last one's as its tail), and a second kernel adds a tail and the heads
// behind it.  Entries without a row are found by a search of the sorted ids, 64 a wave, and set to zero beside it in the same launch.
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

template <typename E, typename T>
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
        if (first + e * kBlock < a.pieces) store_piece<T, 8>((T *)a.out + row[e] * a.ldo + col[e], a.written - col[e], x[e]);
}

// ---- sort --------------------------------------------------------------------------------------------------------------------------------

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / kWave, kSortEach = 8, kSortItems = kSortThreads * kSortEach;
constexpr int kMostDigitBits = 9, kMostDigits = 1 << kMostDigitBits;
static_assert(kMostDigits == kSortThreads, "a thread has a digit");
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
    count[threadIdx.x] = 0;
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

// The sum over the threads before this one, of a workgroup of kSortThreads.
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
    for (int w = 0; w < kSortWaves; ++w) before += w < wave ? lds[w] : 0;
    return before + sum - v;
}

__global__ __launch_bounds__(kSortThreads) void sort_deal_kernel(SortPass p)
{
    __shared__ uint32_t count[kSortWaves][kMostDigits];        // of a wave's own ids; then where they go
    __shared__ uint32_t scan[kSortWaves];
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
    // this thread's digit: how many of it lie in the blocks before, and in all
    uint32_t before = 0, total = 0;
    if (threadIdx.x <= mask) {
        const uint32_t *of_digit = p.counts + threadIdx.x;
        if (p.totals) {
            before = of_digit[(int64_t)blockIdx.x * (mask + 1)];
            total = p.totals[threadIdx.x];
        } else {
#pragma unroll 16
            for (int32_t b = 0; b < p.blocks; ++b) {
                const uint32_t c = of_digit[(int64_t)b * (mask + 1)];
                before += b < (int32_t)blockIdx.x ? c : 0;
                total += c;
            }
        }
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) count[w][threadIdx.x] = 0;
    before += sum_before(total, scan);               // its barrier is behind the counts' clearing
#pragma unroll
    for (int e = 0; e < kSortEach; ++e) {
        const bool there = begin + e * kWave + lane < p.n;
        const uint32_t digit = key[e] >> p.shift & mask;
        uint64_t same = __ballot(there);
        for (int b = 0; b < p.bits; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        const uint64_t lower = same & (((uint64_t)1 << lane) - 1);
        const uint32_t so_far = count[wave][digit];
        rank[e] = so_far + (uint32_t)__popcll(lower);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (there && lower == 0) count[wave][digit] = so_far + (uint32_t)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
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

constexpr int kChunk = 32;

struct GradArgs {
    const void *dy;
    const int32_t *sorted, *order;
    float *dtable, *parts;                          // [chunks][head, tail][pitch]
    int64_t lddy, ldd, span, n_ids, n_entries, chunks, pitch;
    int64_t run_blocks;                             // workgroups that walk chunks; those behind them set entries to zero
    int32_t dim, written;                           // columns of dy; of dtable's rows that are written
    int32_t slabs;
    float scale;
    int accumulate;
};

// Of LANES lanes with V columns each, the runs of a chunk.
template <typename T, int LANES, int V>
__device__ __forceinline__ void walk_chunk(const GradArgs &a, int64_t chunk, int32_t col)
{
    constexpr int kAtOnce = 8;
    const int64_t begin = chunk * kChunk, end = min(begin + kChunk, a.n_ids);
    const bool from_before = begin > 0 && a.sorted[begin - 1] == a.sorted[begin];
    const int left = a.dim - col, left_written = a.written - col;
    float *head = a.parts + chunk * 2 * a.pitch + col;
    float sum[V];
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] = 0.0f;
    int32_t now = a.sorted[begin];
    bool first = from_before;                       // the run goes on from the chunk before
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
    for (int64_t at = begin; at < end; at += kAtOnce) {
        int32_t id[kAtOnce];
        int64_t place[kAtOnce];
        float v[kAtOnce][V];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t p = min(at + u, end - 1);
            id[u] = a.sorted[p];
            place[u] = a.order[p];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const bool there = at + u < end && place[u] >= 0 && place[u] < a.n_ids && left > 0 && id[u] < a.n_entries;
            if (there) load_piece<T, V>((const T *)a.dy, place[u] * a.lddy + col, left, a.span, v[u]);
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
    leave(end < a.n_ids && a.sorted[end] == now);
}

// Zeros in the entries of a wave's 64 that no id names.
__device__ __forceinline__ void clear_entries(const GradArgs &a, int64_t tile)
{
    const int lane = threadIdx.x % kWave;
    const int64_t entry0 = tile * kWave, entry = entry0 + lane;
    if (entry0 >= a.n_entries) return;
    int64_t lo = 0, hi = a.n_ids;                   // the first place of an id that is not below entry
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (a.sorted[mid] < entry) lo = mid + 1;
        else                       hi = mid;
    }
    uint64_t absent = __ballot(entry < a.n_entries && !(lo < a.n_ids && a.sorted[lo] == entry));
    const float zeros[4] = {};
    while (absent) {
        const int64_t at = entry0 + __builtin_ctzll(absent);
        absent &= absent - 1;
        for (int32_t col = lane * 4; col < a.written; col += kWave * 4) store_piece<float, 4>(a.dtable + at * a.ldd + col, a.written - col, zeros);
    }
}

template <typename T, int LANES, int V>
__global__ __launch_bounds__(kBlock) void embedding_runs_kernel(GradArgs a)
{
    const int64_t at = workgroup();
    if (at >= a.run_blocks) {
        if (!a.accumulate) clear_entries(a, (at - a.run_blocks) * kWavesPerBlock + threadIdx.x / kWave);
        return;
    }
    constexpr int kGroups = kBlock / LANES;
    const int64_t slab = at % a.slabs, chunk = at / a.slabs * kGroups + threadIdx.x / LANES;
    const int32_t col = (int32_t)(slab * LANES + threadIdx.x % LANES) * V;
    if (chunk < a.chunks && col < a.written) walk_chunk<T, LANES, V>(a, chunk, col);
}

// Of each run that begins in a chunk and goes on behind it: the chunk's tail and the heads of the chunks that it covers.  Four waves share the heads.
constexpr int kJoinCols = kWave * 4;

__global__ __launch_bounds__(kBlock) void embedding_join_kernel(GradArgs a)
{
    __shared__ float part[kWavesPerBlock][kJoinCols];
    const int64_t at = workgroup(), slab = at % a.slabs, chunk = at / a.slabs;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t end = (chunk + 1) * kChunk;       // of the chunk's places
    if (end >= a.n_ids) return;
    const int32_t id = a.sorted[end - 1];
    if (a.sorted[end] != id) return;
    if (id < 0 || id >= a.n_entries) return;
    if (a.sorted[chunk * kChunk] == id && chunk > 0 && a.sorted[chunk * kChunk - 1] == id) return;         // began before this chunk
    // chunks that begin with the id
    int64_t last = chunk;
    for (;;) {
        const int64_t place = (last + 1 + lane) * kChunk;
        const uint64_t with = __ballot(place < a.n_ids && a.sorted[min(place, a.n_ids - 1)] == id);
        const int n = with == ~(uint64_t)0 ? kWave : __builtin_ctzll(~with);
        last += n;
        if (n < kWave) break;
    }
    const int32_t col = (int32_t)slab * kJoinCols + lane * 4;
    const int left = a.dim - col;
    const float *heads = a.parts + col;
    constexpr int kAtOnce = 8;
    float sum[4] = {};
    if (left > 0)
        for (int64_t c = chunk + 1 + wave; c <= last; c += kWavesPerBlock * kAtOnce) {
            float v[kAtOnce][4];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                load_elements<float, 4>(heads + min(c + u * kWavesPerBlock, last) * 2 * a.pitch, v[u]);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[u][k] = c + u * kWavesPerBlock <= last ? v[u][k] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += v[u][k];
        }
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][k * kWave + lane] = sum[k];
    __syncthreads();
    if (wave != 0 || col >= a.written) return;
    float v[4] = {};
    if (left > 0) {
        load_elements<float, 4>(heads + (chunk * 2 + 1) * a.pitch, v);
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += part[w][k * kWave + lane];
    }
    float *to = a.dtable + id * a.ldd + col;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[k] = k < left ? v[k] * a.scale : 0.0f;
        if (a.accumulate && k < left) v[k] += to[k];
    }
    store_piece<float, 4>(to, a.accumulate ? left : a.written - col, v);
}

int64_t grad_chunks(int64_t n_ids) { return (n_ids + kChunk - 1) / kChunk; }
int64_t grad_pitch(int32_t dim) { return ((int64_t)dim + 7) / 8 * 8; }

template <typename T, int LANES>
void launch_runs(GradArgs &a, hipStream_t st)
{
    constexpr int V = 16 / sizeof(T), kGroups = kBlock / LANES;
    a.slabs = (a.written + LANES * V - 1) / (LANES * V);
    a.run_blocks = (a.chunks + kGroups - 1) / kGroups * a.slabs;
    const int64_t clear = a.accumulate ? 0 : ((a.n_entries + kWave - 1) / kWave + kWavesPerBlock - 1) / kWavesPerBlock;
    embedding_runs_kernel<T, LANES, V><<<grid_of(a.run_blocks + clear, kBlock), kBlock, 0, st>>>(a);
}

template <typename T>
hipError_t launch_gradient(GradArgs a, hipStream_t st)
{
    const int64_t vectors = ((int64_t)a.written * (int64_t)sizeof(T) + 15) / 16;
    if (vectors <= 8)       launch_runs<T, 8>(a, st);
    else if (vectors <= 16) launch_runs<T, 16>(a, st);
    else if (vectors <= 32) launch_runs<T, 32>(a, st);
    else                    launch_runs<T, 64>(a, st);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.chunks < 2) return err;
    a.slabs = (a.written + kJoinCols - 1) / kJoinCols;
    embedding_join_kernel<<<grid_of((a.chunks - 1) * a.slabs, kBlock), kBlock, 0, st>>>(a);
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
    if (table_type == ADAQP_F32 && type == ADAQP_F32) lookup_kernel<float, float><<<grid, kBlock, 0, st>>>(a);
    else if (table_type == ADAQP_F32)                 lookup_kernel<float, __bf16><<<grid, kBlock, 0, st>>>(a);
    else if (type == ADAQP_F32)                       lookup_kernel<__bf16, float><<<grid, kBlock, 0, st>>>(a);
    else                                              lookup_kernel<__bf16, __bf16><<<grid, kBlock, 0, st>>>(a);
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
    *bytes_out = n_ids > kChunk ? (grad_chunks(n_ids) * 2 * grad_pitch(dim) * 4 + 255) / 256 * 256 : 0;
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
    a.chunks = grad_chunks(n_ids);
    a.pitch = grad_pitch(dim);
    a.written = accumulate ? dim : (int32_t)columns_to_write(dtable_dev, ldd, dim, 4);
    if ((a.chunks + 1) * (((int64_t)a.written + kWave - 1) / kWave + 1) + a.n_entries / kWave >= kMostWorkgroups) return ADAQP_ESIZE;
    if (type == ADAQP_F32) ADAQP_HIP_TRY(launch_gradient<float>(a, (hipStream_t)stream));
    else                   ADAQP_HIP_TRY(launch_gradient<__bf16>(a, (hipStream_t)stream));
    return ADAQP_OK;
}
