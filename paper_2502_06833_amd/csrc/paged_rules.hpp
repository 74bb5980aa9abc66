// How a call over a paged cache is cut into workgroups (host code, no HIP).
#pragma once
#include <algorithm>

namespace ead {

// Whether a write or a read moves more than stays in the second-level caches (32 MB) for who comes next
inline bool paged_copy_streams(long rows, int n_kv, int head_dim, int bytes) { return 2.0 * rows * n_kv * head_dim * bytes > 64e6; }

// Blocks of 16 rows that a wave's registers hold at most
constexpr int paged_max_blocks(int head_dim) { return head_dim == 128 ? 2 : 4; }

// Rows per KV head (new tokens times query heads per KV head) of a sequence up to which k_paged_attn takes it
constexpr int paged_few_rows(int head_dim) { return head_dim == 128 ? 32 : 64; }

// Ranges of keys of k_paged_chunk at most: their maxima and sums are joined in the LDS of a key tile
constexpr int paged_many_splits(int head_dim) { return head_dim / 4; }

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

// A launch of k_paged_attn: blocks of 16 rows to a workgroup, tiles of rows per KV head, pairs it cuts into shares (0: a workgroup to a unit),
// workgroups, and the parts of units that there may be
struct PagedShares {
    int nb, row_tiles, pairs, min_share;
    long units, groups, parts;
};
constexpr long kPagedMaxPairs = 1024;      // pairs a wave adds up before it starts; with more there are enough units for every compute unit
// Groups (128 keys) a workgroup starts for at least
constexpr int kPagedMinShare = 2;
// Units of up to this many groups go to a workgroup each: cutting them saves less time than adding up the shares and joining the parts takes
// (4 sequences of 400 8-bit keys: 10.8 us whole, 11.6 in shares; of 700: 14.7 and 12.2).  Where every KV head has several tiles of rows a join has more to read, and a
// unit is cut only if it is longer than kPagedWholeTiles and the units do not fill the device (float prompts of 3 x 500: 18.3 whole, 21.5 in shares; 4 x 2000: 141 and 211).
constexpr long kPagedWholeGroups = 3, kPagedWholeTiles = 8;

// `capacity`: positions a row of the page table reaches, whatever max_kv says; `resident`: workgroups of the kernel the device holds at once
inline PagedShares paged_few(int batch, int n_kv, long rows, int nb, int group, int max_kv, long capacity, int window, int sinks, long resident,
                             long whole_groups = kPagedWholeGroups, long whole_tiles = kPagedWholeTiles) {
    PagedShares p;
    p.nb = nb;
    p.row_tiles = (int)std::max(1l, (rows + 16 * nb - 1) / (16 * nb));
    const long pairs = (long)batch * p.row_tiles;
    p.units = pairs * n_kv;
    const long each = (paged_keys(16 * nb, 32, group, max_kv, window, sinks) + 127) / 128;
    const bool whole = each <= whole_groups || (p.row_tiles > 1 && (each <= whole_tiles || (whole_tiles && p.units >= resident)));
    p.pairs = !whole && pairs <= kPagedMaxPairs && p.units * ((capacity + 127) / 128) < 1l << 30 ? (int)pairs : 0;
    p.min_share = kPagedMinShare;
    p.groups = p.pairs ? std::max(1l, std::min(resident, (p.units * each + p.min_share - 1) / p.min_share)) : p.units;
    p.parts = p.pairs ? 2 * p.groups : 0;
    return p;
}

// Operations of a call at the most
inline double paged_work(int batch, int n_kv, int head_dim, int group, long rows, int max_kv, int window, int sinks) {
    return 4.0 * head_dim * n_kv * rows * batch * (double)paged_keys(16, 32, group, max_kv, window, sinks);
}
// Calls of up to this much work are latency: k_paged_attn takes them alone, however many rows their sequences have (a second launch and k_paged_chunk's longer start
// cost more than its products save; 32 heads, 64 rows after 1000 keys, 1.1e9: 24 us against 36; 256 rows after 2000, 9.4e9: 43 and 47; 8 prompts of 256,
// 8.6e9: 92 and 24)
constexpr double kPagedSmallWork = 4e9;
// Blocks of 16 rows to a workgroup.  One where the work is small and K and V come from the second-level caches when other blocks read them again: more workgroups
// share the work (8 sequences of 32 rows after 2000 keys 27 us with one block, 31 with two; 32 of them 71 and 52).  Float products take eight times
// as long, and the measured bounds are lower (prompts of 3 x 500: 20 / 19 / 21 us with 1 / 2 / 4 blocks; 8 x 500 after 500: 67 / 57 / 51).
inline int paged_blocks(bool f32, long rows, int nb_max, double work, double kv_bytes) {
    if (rows <= 16) return 1;
    if (work <= (f32 ? kPagedSmallWork / 8 : kPagedSmallWork) && kv_bytes <= 64e6) return 1;
    if (rows <= 32 || (f32 && work <= kPagedSmallWork / 2)) return 2;
    return nb_max;
}

// A ticket has a cache line of its own (256 arrivals at 8 tickets side by side made a call of 16 us 2 us longer)
constexpr int kPagedTicketInts = 32;
// Workspace of a launch: a ticket per unit, then every part's maxima and sums, then its outputs
inline unsigned long long paged_workspace(long units, long parts, int tile_rows, int head_dim) {
    if (parts == 0) return 0;
    const unsigned long long rows = (unsigned long long)parts * tile_rows;
    return (unsigned long long)units * kPagedTicketInts * 4 + rows * 8 + rows * head_dim * 4;
}

// k_paged_chunk: two workgroups fit a compute unit
inline PagedPlan paged_many(int batch, int n_kv, int group, long rows, int max_kv, int window, int sinks, int cus, int head_dim) {
    return paged_cut(128, 64, rows, batch, n_kv, group, max_kv, window, sinks, 2l * cus, 4, paged_many_splits(head_dim));
}

}  // namespace ead
