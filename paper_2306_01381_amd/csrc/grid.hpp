// Grids of many workgroups (host and device; needs no HIP header on the host).
#pragma once

#include <stdint.h>

namespace adaqp {

// A launch has fewer than 2^32 threads in each dimension.  Workgroups beyond that go on in the second: workgroup (i, j) is number j * x + i.  The last row may have more of
// them than were asked for; they have nothing to do.  x is a multiple of eight where there are several rows, so that a number modulo eight still says its XCD.
struct GridSize { uint32_t x, y; };

constexpr int64_t kMostWorkgroups = (int64_t)1 << 31;        // of a launch

inline GridSize grid_size(int64_t workgroups, int32_t threads)
{
    const int64_t most = ((int64_t)1 << 31) / threads;       // threads: a power of two up to 1024
    if (workgroups <= most) return GridSize{(uint32_t)workgroups, 1};
    return GridSize{(uint32_t)most, (uint32_t)((workgroups + most - 1) / most)};
}

}  // namespace adaqp
