// How a call over a paged cache is cut into workgroups (host code, no HIP).
#pragma once
#include <algorithm>

namespace ead {

constexpr int kPagedKeyTile = 32;          // keys a wave takes at a time
constexpr int kPagedMaxSplits = 64;

// Blocks of 16 rows that a wave's registers hold at most: float queries and outputs of 128 dimensions take twice as many
constexpr int paged_max_blocks(bool f32, int head_dim) { return f32 && head_dim == 128 ? 2 : 4; }

// A call of k_paged_attn: blocks of 16 rows a workgroup takes, tiles of rows per KV head, ranges of keys per tile
struct PagedPlan {
    int nb, row_tiles, splits, split_tiles;
    long units;                            // (sequence, KV head, tile of rows)
};

inline PagedPlan paged_plan(int batch, int n_kv, int group, int max_q, int max_kv, int window, int sinks, int cus, int nb_max) {
    PagedPlan p;
    const long rows = (long)max_q * group;
    p.nb = rows <= 16 ? 1 : rows <= 32 ? 2 : nb_max;
    const int tile_rows = 16 * p.nb;
    p.row_tiles = (int)std::max(1l, (rows + tile_rows - 1) / tile_rows);
    p.units = (long)batch * n_kv * p.row_tiles;
    // key tiles that a tile of rows sees at most
    long keys = std::max(1, max_kv);
    if (window > 0) {
        const long seen = (long)window + (tile_rows - 1) / group + 1 + 2 * kPagedKeyTile + (sinks > 0 ? (long)sinks + kPagedKeyTile : 0);
        keys = std::min(keys, seen);
    }
    const long tiles = (keys + kPagedKeyTile - 1) / kPagedKeyTile;
    // Ranges of keys where there are too few tiles of rows for four workgroups a compute unit, none shorter than a tile for each of
    // a workgroup's four waves
    const long want = std::max(1l, (4l * cus + p.units - 1) / p.units);
    const long splits = std::max(1l, std::min({want, tiles / 4, (long)kPagedMaxSplits}));
    p.split_tiles = (int)(((tiles + splits - 1) / splits + 3) / 4 * 4);
    p.splits = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
    return p;
}

// Workspace: a ticket per unit (to a multiple of 64), then every range's maxima and sums, then its outputs
inline unsigned long long paged_bytes(const PagedPlan &p, int head_dim) {
    if (p.splits == 1) return 0;
    const unsigned long long rows = (unsigned long long)p.units * p.splits * 16 * p.nb;
    return ((unsigned long long)p.units + 63) / 64 * 256 + rows * 8 + rows * head_dim * 4;
}

}  // namespace ead
