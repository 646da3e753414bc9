// Tiles of a matrix in the LDS for the matrix cores: of each row one 128-byte line, loaded from memory without passing registers.
// The eight 16-byte parts of a line lie at (part ^ row / 2 mod 8).  Two rows fill the 64 banks, so of lanes that read the same part of 16 rows at a time
// none meet (with row mod 8 in the place of row / 2, rows that are 8 apart did: 44 % of the LDS's cycles in a product of 8192 x 8192 x 4096).
//
// The loads are written as instructions: with the builtin the compiler has every read of the LDS wait for all loads that are under way, also those into
// another buffer.  A wave counts its own loads instead (arrived) before the barrier.  A load of 64 times 16 bytes keeps the CU's path to the caches busy for 16
// cycles, and waves that find it busy stand still: loads are issued one by one between products, not in a row.
#pragma once

#include "elements.hpp"

namespace adaqp {

constexpr int kLine = 128;

__device__ __forceinline__ uint32_t lds_offset(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// Of each lane the 16 or 4 bytes at base + offset, to lds + lane * that; base and lds are the wave's.  (Nothing else in these kernels uses m0.)
__device__ __forceinline__ void load_to_lds_16(const void *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds) : "memory");
}
__device__ __forceinline__ void load_to_lds_4(const void *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(offset), "s"(base), "s"(lds) : "memory");
}

// All but the newest OUTSTANDING loads of every wave of the workgroup are in the LDS, and no wave reads the LDS any more.
template <int OUTSTANDING>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(OUTSTANDING) : "memory");
}

// The same for a wave with a part of the LDS of its own: its loads are there; what it read there is in registers.
template <int OUTSTANDING>
__device__ __forceinline__ void own_arrived()
{
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(OUTSTANDING) : "memory");
}
__device__ __forceinline__ void own_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Which 16 bytes of a line this lane loads with the i-th load of a wave: 8 rows each, the first a multiple of 16.
__device__ __forceinline__ uint32_t part_of_lane(int i) { return threadIdx.x % 8 ^ (i % 2 * 4 + threadIdx.x % kWave / 16); }

// The places of a wave's loads of a tile of ROWS rows, one of four waves' that load it together, relative to the tile's first row.  Rows behind the matrix's last take that one's place: what is
// computed from them is not stored.  256 rows of a pitch of 2^24 bytes still fit.
template <int ROWS>
struct TileLoads {
    static constexpr int kLoads = ROWS / (8 * kWavesPerBlock);          // 8 rows of 8 parts each
    static_assert(ROWS % (16 * kWavesPerBlock) == 0, "a wave's rows begin at a multiple of 16");
    uint32_t offset[kLoads];

    __device__ __forceinline__ TileLoads(int64_t row0, int64_t n_rows, int64_t pitch)
    {
        const int wave = threadIdx.x % kBlock / kWave, lane = threadIdx.x % kWave;
        const uint32_t last = (uint32_t)min((int64_t)ROWS, n_rows - row0) - 1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t row = wave * (ROWS / kWavesPerBlock) + i * 8 + lane / 8;
            offset[i] = min(row, last) * (uint32_t)pitch + part_of_lane(i) * 16;
        }
    }

    // Where the wave's loads into a buffer go.
    __device__ __forceinline__ static uint32_t place(const uint8_t *lds)
    {
        return __builtin_amdgcn_readfirstlane(lds_offset(lds) + threadIdx.x % kBlock / kWave * (ROWS / kWavesPerBlock) * kLine);
    }

    // Load i of one line of each row; `from` is that line of the tile's first row.  With `half` the second half of the lines does not exist, and the first is
    // loaded in its place.
    template <bool MAY_BE_HALF>
    __device__ __forceinline__ void load(int i, const uint8_t *from, uint32_t to, bool half = false) const
    {
        const uint32_t back = MAY_BE_HALF && half ? part_of_lane(i) / 4 * (kLine / 2) : 0;
        load_to_lds_16(from, offset[i] - back, to + i * 8 * kLine);
    }
};

// Which tile a workgroup takes.  Workgroups are dealt to the eight XCDs in turn; an XCD gets neighbouring tiles, so that operands are read into its L2 once
// and the ends of neighbouring tiles' rows meet there.  Within that, kRowGroup tile rows are walked together, column by column: what runs at a time is
// about square and needs the fewest rows of both operands.  `parts`: cuts of k; the tiles of one part are neighbours.  part < 0: none, the grid is a
// multiple of eight.
constexpr int kRowGroup = 8;

struct TilePlace { int64_t part, row, col; };

inline int64_t tile_blocks(int64_t n_tiles, int64_t parts) { return (n_tiles * parts + 7) / 8 * 8; }

__device__ __forceinline__ TilePlace tile_place(uint32_t block, uint32_t blocks, uint32_t tiles_r, uint32_t tiles_c, uint32_t parts)
{
    const uint32_t tiles = tiles_r * tiles_c, at = xcd_neighbour(block, blocks);
    const uint32_t part = at / tiles, tile = at % tiles;
    const uint32_t group = tile / (kRowGroup * tiles_c), in_group = tile % (kRowGroup * tiles_c);
    const uint32_t rows = min((uint32_t)kRowGroup, tiles_r - group * kRowGroup);
    return TilePlace{part < parts ? (int64_t)part : -1, group * kRowGroup + in_group % rows, in_group / rows};
}

__device__ __forceinline__ const uint8_t *line_part(const uint8_t *lds, int row, int part) { return lds + row * kLine + (part ^ row / 2 % 8) * 16; }

}  // namespace adaqp
