// What the products share (project.hip, project_fp8.hip).
#pragma once
#include "dsla_internal.h"

namespace dsla {

template <int N>
__device__ __forceinline__ void wait_loads()   // at most N of this wavefront's loads are still in flight
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Tile order: the 8 XCDs each take a contiguous run of the linear tile order (workgroup ids go round-robin over the
// XCDs, each XCD has its own L2), and the linear order runs in groups of GM row tiles: inside a group the row tile
// runs fastest, then the column tile, so the tiles in flight at one time (a few dozen per XCD) share GM panels of x
// and a handful of panels of W instead of one panel of W and dozens of x.  M = 16384, K = 4096, N = 20480 with GM = 4, 6, 8,
// 16: 1.98, 1.99, 2.09, 2.24 ms.  Each group reads all of W, so a last group of one or two row tiles after a single full
// one is worth avoiding (group_rows()): M = 1060, K = 11008, N = 20480 in 4 + 1 and 5 row tiles 562 and 509 us.
// False: no tile for this workgroup.
__device__ __forceinline__ bool tile_of(uint32_t workgroup, int tiles_m, int tiles_n, int GM, long long per_xcd, int &tm, int &tn)
{
    const long long ntiles = static_cast<long long>(tiles_m) * tiles_n;
    const long long lin = static_cast<long long>(workgroup % 8) * per_xcd + workgroup / 8;
    if (lin >= ntiles) return false;
    const long long per_group = static_cast<long long>(GM) * tiles_n;
    const int first_m = static_cast<int>(lin / per_group) * GM;
    const int gsz = tiles_m - first_m < GM ? tiles_m - first_m : GM;
    const int in_group = static_cast<int>(lin % per_group);
    tn = in_group / gsz;
    tm = first_m + in_group % gsz;
    return true;
}

}  // namespace dsla
