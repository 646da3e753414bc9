// Grids of many workgroups (host and device; needs no HIP header on the host).
#pragma once

#include <stdint.h>

namespace adaqp {

// A launch has fewer than 2^32 threads in each dimension.  Workgroups beyond that go on in the second: number y * x_count + x, some more than were asked for, which
// a kernel has to do nothing in.  Numbers stay neighbours of their XCD's: x is a multiple of eight wherever there is a second row of them.
struct GridSize { uint32_t x, y; };

constexpr int64_t kMostWorkgroups = (int64_t)1 << 31;        // of a launch

inline GridSize grid_size(int64_t workgroups, int32_t threads)
{
    const int64_t most = ((int64_t)1 << 31) / threads;       // threads: a power of two up to 1024
    if (workgroups <= most) return GridSize{(uint32_t)workgroups, 1};
    return GridSize{(uint32_t)most, (uint32_t)((workgroups + most - 1) / most)};
}

}  // namespace adaqp
