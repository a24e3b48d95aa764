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

// The group that comes turn-th by length, the longest first, the lower first among equal ones; of at most kSorted groups (more even out by themselves).
constexpr int kSorted = 32;
__device__ __forceinline__ int by_length(const int32_t *offsets, int turn, int E, int M)
{
    const int lane = threadIdx.x & 63;
    const GroupRows g = group_rows(offsets, min(lane, E), E, M);
    const int length = lane < E ? g.hi - g.lo : -1;
    int before = lane < E ? 0 : -1;
    for (int i = 0; i < E; ++i) {
        const int other = lane_of(length, i);
        before += other > length || (other == length && i < lane);
    }
    return __builtin_ctzll(__ballot(lane < E && before == turn));
}

// Consecutive workgroups go to the eight dies in turn: die x takes the x-th eighth of the tiles, so that the tiles that
// share operands share an L2.
__device__ __forceinline__ int die_order(int id, int total)
{
    const int q = total >> 3, r = total & 7, x = id & 7;
    return x * q + min(x, r) + (id >> 3);
}

// The tiles of `height` rows of all groups times `col_tiles`, four column tiles at a time down the rows.  The first 64 groups'
// counts stay in a wave's registers, the others are read again for every tile.
struct GroupTile { int e, lo, hi, m, n; };
struct GroupTiles {
    const int32_t *offsets;
    int E, M, height, col_tiles;
    int total;
    GroupRows first;               // of group `lane`
    int first_upto;                // row tiles of the groups up to it

    __device__ __forceinline__ int count(int e, const GroupRows &g) const { return e <= E ? (g.hi - g.lo + height - 1) / height : 0; }
    __device__ __forceinline__ GroupRows rows(int e) const { return group_rows(offsets, min(e, E), E, M); }

    __device__ __forceinline__ void init(const int32_t *offsets_, int E_, int M_, int height_, int col_tiles_)
    {
        offsets = offsets_; E = E_; M = M_; height = height_; col_tiles = col_tiles_;
        const int lane = threadIdx.x & 63;
        first = rows(lane);
        first_upto = wave_prefix(count(lane, first));
        total = lane_of(first_upto, 63);
        for (int e0 = 64; e0 <= E; e0 += 64) total += lane_of(wave_prefix(count(e0 + lane, rows(e0 + lane))), 63);
        total *= col_tiles;
    }
    // the id-th tile; false where there is none
    __device__ __forceinline__ bool find(int id, GroupTile *t) const
    {
        if (id >= total) return false;
        const int lane = threadIdx.x & 63;
        id = die_order(id, total);
        int before = 0;
        for (int e0 = 0; e0 <= E; e0 += 64) {
            const GroupRows g = e0 ? rows(e0 + lane) : first;
            const int tiles = count(e0 + lane, g), upto = (e0 ? wave_prefix(tiles) : first_upto) * col_tiles;
            const unsigned long long past = __ballot(id < before + upto);
            if (past) {
                const int l = __builtin_ctzll(past), high = lane_of(tiles, l);
                const int at = id - before - (lane_of(upto, l) - high * col_tiles);
                const int band = wave_value(at / max(high * 4, 1)), n0 = band * 4, width = max(min(4, col_tiles - n0), 1), in = at - band * high * 4;
                t->e = wave_value(e0 + l);
                t->lo = lane_of(g.lo, l);
                t->hi = lane_of(g.hi, l);
                t->m = wave_value(in / width);
                t->n = wave_value(n0 + in - t->m * width);
                // offsets that are none (groups that overlap many times) may make the sums above wrap around
                return (unsigned)t->m < (unsigned)high && (unsigned)t->n < (unsigned)col_tiles;
            }
            before += lane_of(upto, 63);
        }
        return false;
    }
};

}  // namespace polydl
