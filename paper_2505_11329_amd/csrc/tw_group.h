// Rows in groups, one for each expert: where the tiles of a grouped product lie. The offsets stay on the device, so every
// wave finds its tile by itself.
#pragma once

#include <stdint.h>

#include "tw_scan.h"

namespace tw {

// The groups' first rows, n_groups + 1 of them. They are taken as they should be, whatever they are: inside the tensor
// and ascending, so that no two groups share a row and the tiles are no more than the launch has counted on.
struct Groups {
    const int32_t *offsets;
    int n_groups;
    int rows;
};

// 64 groups, one to a lane: their first rows and those behind them. `carry` is where the first of them begins, and then where
// the last of them ends.
struct GroupRows {
    int begin, end;
};
__device__ __forceinline__ GroupRows group_rows(const Groups &g, int first, int lane, int *carry)
{
    const int e = first + lane;
    const int mine = e < g.n_groups ? min(max(g.offsets[e + 1], 0), g.rows) : 0;
    const int end = max(max_upto(mine), *carry);
    int begin = __builtin_amdgcn_update_dpp(0, end, 0x138, 0xf, 0xf, false);  // wave_shr 1: the lane before
    if (lane == 0) begin = *carry;
    *carry = __builtin_amdgcn_readlane(end, 63);
    return {begin, end};
}
__device__ __forceinline__ int first_group_row(const Groups &g)
{
    return min(max(__builtin_amdgcn_readfirstlane(g.offsets[0]), 0), g.rows);
}

// Tile `index` of a list of all groups' tiles, group after group: rows of `tile_rows` times `tiles_n` columns of them. All of it
// is the same in every lane.
struct GroupTile {
    int group;        // -1: there is no such tile
    int tile;         // within the group's tiles
    int begin, rows;  // the group's
    int total;        // tiles of all groups up to this one's, of all where there is no such tile
};
// ... of 64 groups from `first` on, whose tiles follow `before` others; -1 where it is none of theirs
__device__ __forceinline__ GroupTile find_among(const GroupRows &r, int first, uint32_t tile_rows, int tiles_n, int before, int index)
{
    const int tiles = static_cast<int>((static_cast<uint32_t>(r.end - r.begin) + tile_rows - 1) / tile_rows) * tiles_n;
    const int upto = before + sum_upto(tiles);
    const uint64_t past = __ballot(upto > index);
    if (!past) return {-1, 0, 0, 0, __builtin_amdgcn_readlane(upto, 63)};
    const int l = __builtin_ctzll(past);
    const int begin = __builtin_amdgcn_readlane(r.begin, l), last = __builtin_amdgcn_readlane(upto, l);
    return {first + l, index - (last - __builtin_amdgcn_readlane(tiles, l)), begin, __builtin_amdgcn_readlane(r.end, l) - begin, last};
}
__device__ __forceinline__ GroupTile find_group_tile(const Groups &g, uint32_t tile_rows, int tiles_n, int index)
{
    const int lane = threadIdx.x & 63;
    int carry = first_group_row(g);
    GroupTile t = {-1, 0, 0, 0, 0};
    for (int first = 0; first < g.n_groups && t.group < 0; first += 64)
        t = find_among(group_rows(g, first, lane, &carry), first, tile_rows, tiles_n, t.total, index);
    return t;
}

// The same with the first 64 groups, which most lists do not exceed, kept in registers, so that a wave goes to memory once before its first
// load (4 rows of 4 experts [2048 x 1024]: 7.0 to 6.6 us; 96 of 8 [4096 x 3584]: 36.9 to 35.3).
struct KeptGroups {
    Groups g;
    GroupRows rows;
    int total;  // all groups' tiles
};
__device__ __forceinline__ KeptGroups keep_groups(const Groups &g, uint32_t tile_rows, int tiles_n)
{
    int carry = first_group_row(g);
    KeptGroups k = {g, group_rows(g, 0, threadIdx.x & 63, &carry), 0};
    k.total = g.n_groups > 64 ? find_group_tile(g, tile_rows, tiles_n, INT32_MAX).total
                              : find_among(k.rows, 0, tile_rows, tiles_n, 0, INT32_MAX).total;
    return k;
}
__device__ __forceinline__ GroupTile find_group_tile(const KeptGroups &k, uint32_t tile_rows, int tiles_n, int index)
{
    return k.g.n_groups > 64 ? find_group_tile(k.g, tile_rows, tiles_n, index) : find_among(k.rows, 0, tile_rows, tiles_n, 0, index);
}

// What a kernel of single products takes besides for products by group: B has a weight for each, `b_bytes` apart.
struct GroupedB {
    Groups groups;
    int64_t b_bytes;
};
__device__ __forceinline__ GroupedB group_argument() { return {}; }
__device__ __forceinline__ GroupedB group_argument(const GroupedB &g) { return g; }

// All groups' tiles.
__device__ __forceinline__ int count_group_tiles(const Groups &g, uint32_t tile_rows, int tiles_n)
{
    return find_group_tile(g, tile_rows, tiles_n, INT32_MAX).total;
}

}  // namespace tw
