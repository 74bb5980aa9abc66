// How a call over a paged cache is cut into workgroups (host code, no HIP).
#pragma once
#include <algorithm>

namespace ead {

constexpr int kPagedMaxSplits = 64;

// Blocks of 16 rows that a wave's registers hold at most: float queries and outputs of 128 dimensions take twice as many
constexpr int paged_max_blocks(bool f32, int head_dim) { return f32 && head_dim == 128 ? 2 : 4; }

// Rows per KV head (new tokens times query heads per KV head) of a sequence up to which k_paged_attn takes it
constexpr int kPagedFewRows = 64;

// Keys a row sees at most up to which k_paged_chunk takes two bf16 terms of every probability (its comment has both sides)
constexpr int kPagedTwoTerms = 4096;

// Ranges of keys of k_paged_chunk: their maxima and sums are joined in the LDS of two key tiles
constexpr int paged_many_splits(int head_dim) { return head_dim / 2; }

// A launch: rows a workgroup takes, tiles of rows per KV head, ranges of keys per tile
struct PagedPlan {
    int tile_rows, row_tiles, splits, split_tiles;
    long units;                            // (sequence, KV head, tile of rows)
};

// keys that a tile of rows sees at most
inline long paged_keys(int tile_rows, int key_tile, int group, int max_kv, int window, int sinks) {
    const long keys = std::max(1, max_kv);
    if (window <= 0) return keys;
    return std::min(keys, (long)window + (tile_rows - 1) / group + 1 + 2 * key_tile + (sinks > 0 ? (long)sinks + key_tile : 0));
}

inline PagedPlan paged_cut(int tile_rows, int key_tile, long rows, int batch, int n_kv, int group, int max_kv, int window, int sinks, long want_groups, int min_tiles, int max_splits) {
    PagedPlan p;
    p.tile_rows = tile_rows;
    p.row_tiles = (int)std::max(1l, (rows + tile_rows - 1) / tile_rows);
    p.units = (long)batch * n_kv * p.row_tiles;
    const long tiles = (paged_keys(tile_rows, key_tile, group, max_kv, window, sinks) + key_tile - 1) / key_tile;
    const long want = std::max(1l, (want_groups + p.units - 1) / p.units);
    const long splits = std::max(1l, std::min({want, tiles / min_tiles, (long)max_splits}));
    p.split_tiles = (int)((tiles + splits - 1) / splits + min_tiles - 1) / min_tiles * min_tiles;
    p.splits = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
    return p;
}

// k_paged_attn: ranges of keys where there are too few tiles of rows for four workgroups a compute unit, none shorter than a tile for each
// of a workgroup's four waves
inline PagedPlan paged_few(int batch, int n_kv, int group, long rows, int max_kv, int window, int sinks, int cus, int nb_max) {
    const int nb = rows <= 16 ? 1 : rows <= 32 ? 2 : nb_max;
    return paged_cut(16 * nb, 32, rows, batch, n_kv, group, max_kv, window, sinks, 4l * cus, 4, kPagedMaxSplits);
}

// k_paged_chunk: two workgroups fit a compute unit
inline PagedPlan paged_many(int batch, int n_kv, int group, long rows, int max_kv, int window, int sinks, int cus, int head_dim) {
    return paged_cut(128, 64, rows, batch, n_kv, group, max_kv, window, sinks, 2l * cus, 4, paged_many_splits(head_dim));
}

// Workspace of a launch: a ticket per unit (to a multiple of 64), then every range's maxima and sums, then its outputs
inline unsigned long long paged_bytes(const PagedPlan &p, int head_dim) {
    if (p.splits == 1) return 0;
    const unsigned long long rows = (unsigned long long)p.units * p.splits * p.tile_rows;
    return ((unsigned long long)p.units + 63) / 64 * 256 + rows * 8 + rows * head_dim * 4;
}

}  // namespace ead
