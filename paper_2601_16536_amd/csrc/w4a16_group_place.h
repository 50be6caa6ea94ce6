// Which rows of which group a workgroup of the products of rows in groups has.
//
// Row tiles are numbered group by group; how many there are only the device knows, so the launch has as many workgroups as there could be, and those past the last tile have none.
// XCD x (workgroup mod 8) takes the x-th eighth of the (row tile, column tile) pairs that there are, in order: neighbours read the same rows and weights through one L2.
// Offsets that descend are wrong but may not lead outside of the arguments.  Each group's rows are kept within 0 .. count, so 1026 groups may have all 2^30 rows each: their tiles are counted in 64 bits.
#pragma once
#include <cstdint>
#include "w4a16_place.h"

namespace w4a16 {

typedef long long TileCount;

__host__ __device__ inline int clamp_to(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// The rows of group g; E: those behind the last group, E + 1: those ahead of the first.
__host__ __device__ inline void group_range(const int32_t *offsets, int E, int count, int g, int *begin, int *end)
{
    const int b = g <= E ? clamp_to(offsets[g], 0, count) : 0;
    *begin = b;
    *end = g == E ? count : clamp_to(offsets[g < E ? g + 1 : 0], b, count);
}

struct GroupTiling {
    const int32_t *offsets;
    int E, groups, count, tile_rows, cols;  // groups: E, or with the rows that no group has E + 2; cols: column tiles
};
struct RowTile {
    int group, row0, end;  // rows row0 .. min(end, row0 + tile) - 1
    int col;               // column tile
};
constexpr int kBlockRows = 4;

// The tiles of the groups that thread tid of `threads` counts.
__host__ __device__ inline TileCount tiles_of_thread(const GroupTiling &g, int tid, int threads)
{
    const int per = (g.groups + threads - 1) / threads;
    TileCount tiles = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < g.groups) {
            int b, e;
            group_range(g.offsets, g.E, g.count, tid * per + i, &b, &e);
            tiles += (e - b + g.tile_rows - 1) / g.tile_rows;
        }
    return tiles;
}

// The (row tile, column tile) pair of a workgroup; false: it has none.
__host__ __device__ inline bool pair_of_block(TileCount total, int cols, unsigned block, TileCount *pair)
{
    const TileCount pairs = total * cols, eighth = (pairs + kPlaceXcds - 1) / kPlaceXcds, in = block / kPlaceXcds;
    *pair = (TileCount)(block % kPlaceXcds) * eighth + in;
    return in < eighth && *pair < pairs;
}

// Where that is, if it is among the thread's tiles, which begin with number `at`.  In a group, kBlockRows row tiles at a time, column by column.
__host__ __device__ inline bool tile_of_thread(const GroupTiling &g, int tid, int threads, TileCount at, TileCount tiles, TileCount pair, RowTile *found)
{
    const TileCount tile = pair / g.cols;
    if (tile < at || tile >= at + tiles) return false;
    const int per = (g.groups + threads - 1) / threads;
    for (int i = 0; i < per && tid * per + i < g.groups; ++i) {
        int b, e;
        group_range(g.offsets, g.E, g.count, tid * per + i, &b, &e);
        const int n = (e - b + g.tile_rows - 1) / g.tile_rows;
        if (tile < at + n) {
            const TileCount in_group = pair - at * g.cols, in_block = (TileCount)kBlockRows * g.cols;
            const int block = (int)(in_group / in_block), high = n - block * kBlockRows < kBlockRows ? n - block * kBlockRows : kBlockRows;
            const int rest = (int)(in_group - block * in_block);
            *found = {tid * per + i, b + (block * kBlockRows + rest % high) * g.tile_rows, e, rest / high};
            return true;
        }
        at += n;
    }
    return false;
}

// At most so many row tiles.
inline long long most_row_tiles(long long groups, long long count, int tile_rows)
{
    if (groups > count) groups = count;
    return (count + groups * (tile_rows - 1)) / tile_rows;
}

}  // namespace w4a16
