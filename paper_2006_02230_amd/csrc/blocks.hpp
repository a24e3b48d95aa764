// Grids of any number of workgroups.  A launch holds fewer than 2^32 threads along one axis of its grid; past that only what is left over
// 2^32 runs, without an error (2^32 itself is one).  So more workgroups than that lie along x and z, and block_number() is the workgroup's
// number among them.  The last row of z may go past the last one.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace polydl {

constexpr int64_t kBlocksAlong = 1 << 20;
constexpr int64_t kMaxBlocks = 0x7ff00000;      // for kernels that keep the number in an int, the numbers past the last one among them

inline dim3 many_blocks(int64_t blocks, int threads, unsigned across = 1)
{
    if (blocks * threads <= 0xffffffffll) return dim3((unsigned)blocks, across);
    return dim3((unsigned)kBlocksAlong, across, (unsigned)((blocks + kBlocksAlong - 1) / kBlocksAlong));
}
__device__ __forceinline__ unsigned block_number() { return blockIdx.x + blockIdx.z * (unsigned)kBlocksAlong; }

}  // namespace polydl
