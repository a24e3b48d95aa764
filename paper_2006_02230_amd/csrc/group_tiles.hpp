// Which tile of which group a workgroup works on: rows sorted by group, offsets in device memory.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "lanes.hpp"

namespace polydl {

// Rows [lo, hi) of group e; E names the slots behind the last group.  Whatever the offsets hold, the rows are inside [0, M).
struct GroupRows { int lo, hi; };
__device__ __forceinline__ GroupRows group_rows(const int32_t *offsets, int e, int E, int M)
{
    if (!offsets) return {e < E ? 0 : M, M};                 // one group of all rows
    const int lo = min(max(offsets[e], 0), M);
    const int hi = e < E ? min(max(offsets[e + 1], lo), M) : M;
    return {lo, hi};
}

// Consecutive workgroups go to the eight dies in turn: die x takes the x-th eighth of the tiles, so that the tiles that
// share operands share an L2.
__device__ __forceinline__ int die_order(int id, int total)
{
    const int q = total >> 3, r = total & 7, x = id & 7;
    return x * q + min(x, r) + (id >> 3);
}

// The tile of workgroup `id` among the tiles of `height` rows of all groups times `col_tiles`: false where there is none.
// Four column tiles at a time, down the rows.
struct GroupTile { int e, lo, hi, m, n; };
__device__ __forceinline__ bool find_tile(const int32_t *offsets, int E, int M, int height, int col_tiles, int id, GroupTile *t)
{
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const GroupRows g = group_rows(offsets, min(e0 + lane, E), E, M);
        total += lane_of(wave_prefix(e0 + lane <= E ? (g.hi - g.lo + height - 1) / height : 0), 63);
    }
    total *= col_tiles;
    if (id >= total) return false;
    id = die_order(id, total);
    int before = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const GroupRows g = group_rows(offsets, min(e0 + lane, E), E, M);
        const int tiles = e0 + lane <= E ? (g.hi - g.lo + height - 1) / height : 0;
        const int upto = wave_prefix(tiles) * col_tiles;
        const unsigned long long past = __ballot(id < before + upto);
        if (past) {
            const int l = __builtin_ctzll(past), rows = lane_of(tiles, l);
            const int at = id - before - (lane_of(upto, l) - rows * col_tiles);
            const int band = at / max(rows * 4, 1), n0 = band * 4, width = max(min(4, col_tiles - n0), 1), in = at - band * rows * 4;
            t->e = e0 + l;
            t->lo = lane_of(g.lo, l);
            t->hi = lane_of(g.hi, l);
            t->m = in / width;
            t->n = n0 + in - t->m * width;
            // offsets that are none (groups that overlap many times) may make the sums above wrap around
            return (unsigned)t->m < (unsigned)rows && (unsigned)t->n < (unsigned)col_tiles;
        }
        before += lane_of(upto, 63);
    }
    return false;
}

}  // namespace polydl
