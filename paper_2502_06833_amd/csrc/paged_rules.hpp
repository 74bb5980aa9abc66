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

// ---- rotation ----
// Heads of a row that a group of lanes takes: one, or of many bf16 rows four, which share sines and cosines and are requested together.  Such calls move 67 MB and more, none of
// which stays in the second-level caches (32 MB), so their accesses are non-temporal.  Inputs from memory, 32 and 8 heads, four against one: heads of 128, 816 rows 8.7 and 9.3 us, 3272
// rows (the bound) 18.5 and 26.9, 26208 rows 114 and 173; of 64, 6552 rows (the bound) 21.8 and 27.2.  Where a call just before left its inputs in the last-level cache the two cross
// about the bound (heads of 64, 6552 rows: 22.7 and 21.2; of 128, 2048: 10.8 and 14.6).  One is the faster where vectors are short or wide: heads of 32, 32768 rows of 16, 35 and 27 us; float32,
// 8 requests of 32 bytes to a lane: heads of 128, 6552 rows 62.5 and 60.0, prompts to 8 bits 115 and 101; heads of 32 49 and 35.
constexpr int kRotateEach = 4;
constexpr bool rotate_shares(int bytes, int head_dim) { return bytes == 2 && head_dim >= 64; }
inline bool rotate_wide(long rows, long heads, int head_dim, int bytes) { return rotate_shares(bytes, head_dim) && rows * heads * (head_dim / 16) > 4l * 256 * 1024; }
inline long rotate_units(long q, long k, long v, int each) { return (q + each - 1) / each + (k + each - 1) / each + (v + each - 1) / each; }

// ---- weighing ----
// Sequences of up to this many rows per KV head (new tokens times query heads per KV head) keep their queries in registers while keys stream past (k_weigh_few); with more
// the keys stay and the rows stream (k_weigh_many).  Float queries take twice the registers.  Few against many, 8 KV heads: heads of 128, one sequence of 8192 bf16 keys, 16 rows 5.3 and
// 7.6 us, 32 6.6 and 7.5, 64 10.2 and 10.0; sixteen of 4096 26 and 32, 29.5 and 28.9, 41 and 34; of 8-bit ones 16 and 30, 20 and 28, 37 and 33; heads of 64, bf16, 14 and 20, 16 and 19, 28
// and 24.  So 64 rows are past the crossing where there are many keys, and on it for one sequence.
constexpr int weigh_few_rows(bool f32, int head_dim) { return f32 && head_dim == 128 ? 32 : 64; }
// Workgroups of k_weigh for a KV head of a sequence: 16 keys each, and past 2^24 positions again 2^24 further on (a launch counts its threads in 32 bits: from 2^28 positions on
// one workgroup to every 16 keys would not fit)
inline unsigned weigh_simple_groups(int held) { return (unsigned)std::min((held + 15l) / 16, 1l << 20); }
// Tiles of 32 keys to a wave of k_weigh_few: eight at most, since sequences are of different lengths (64 of 1024 to 16384 8-bit keys: 102, 74, 68, 70, 80 and 98 us with at most 1, 2, 4, 8,
// 16 and 32; 64 of 4096: 73, 52, 48, 49, 49 and 49; 16 of 8192 bf16 keys: 62, 47, and 42 from 4 on)
inline int weigh_tiles(long units, int held, int cus) {
    const long groups = units * std::max(1, (held + 127) / 128);
    return (int)std::max(1l, std::min(8l, (groups + 8l * cus - 1) / (8l * cus)));
}
// Ranges of rows of k_weigh_many, and the keys that a range's sums are kept for.  With 1, 3, 6, 12 and 24 workgroups for every compute unit (bf16, 32 and 8 heads): 2048 rows of 8193 keys 304,
// 194, 181, 168 and 156 us; 512 rows of 8193 118, 80, 64, 61 and 61; 2048 of 2048 118, 70, 47, 50 and 50; four times 1024 of 4096 272, 285, 243, 221 and 211.  (24 would hold twice the sums.)
struct WeighPlan { int splits, part_keys; };
inline WeighPlan weigh_many(int batch, int n_kv, long rows, int held, int cus) {
    WeighPlan p;
    p.part_keys = std::max(1, (held + 255) / 256) * 256;
    const long units = (long)batch * n_kv * (p.part_keys / 256), tiles = (rows + 31) / 32;
    p.splits = (int)std::max(1l, std::min((12l * cus + units - 1) / units, tiles / 8));
    return p;
}

// ---- eviction ----
constexpr int kEvictMost = 1 << 20;        // positions of a sequence at most
// LDS of a workgroup that chooses: a bit for every position that the host vouched for, and as many scores' ranks as there is room for
constexpr int kEvictLds = 144 << 10, kEvictPlainLds = 52 << 10;      // all that a compute unit has beside the bins; what needs no asking for
inline int evict_words(int held) { return (held + 63) / 64; }
inline int evict_cached(int held, int room) { return std::min((std::max(held, 1) + 3) / 4 * 4, (room - evict_words(held) * 8) / 16 * 4); }
inline unsigned long long evict_moves_at(unsigned long long units) { return (units * 4 + 15) / 16 * 16; }
struct EvictPlan {
    int threads;                           // of a workgroup that chooses
    int columns;                           // pieces of a vector that workgroups of their own move
    int shares;                            // workgroups that share a sequence's and head's free places (whole vectors, in a launch of their own); 0: the same ones
    int shift_threads;                     // of a workgroup that moves the last positions down
};
inline EvictPlan evict_plan(int batch, int n_kv, int held, int keep, int recent, int vec_bytes, int cus) {
    EvictPlan p;
    const long units = (long)batch * n_kv, moves = std::max(0, std::min(held - keep, keep - recent));
    // Whole evictions with 256, 512 and 1024 threads, 8 heads: 64 sequences of 700 positions 38.7, 37.3 and 45.9 us, of 2176 48, 46 and 54, of 4000 54, 50 and 59, of 8000 67, 58 and 66;
    // three of 2176 17.8, 15.3 and 16.1, of 8000 30, 22 and 21, of 16000 69, 51 and 46, of 28000 111, 79 and 69.  1024 are the faster ones where few sequences are long; `held` is the
    // caller's bound, so one that is far above the lengths takes them too (64 of 700 under a bound of 16384: 45.3, with 512 37.4).
    p.threads = held > 4096 ? 1024 : held > 1024 ? 512 : 256;
    p.columns = 1;
    while (vec_bytes / p.columns > 64 && 2 * units * p.columns < 2l * cus) p.columns *= 2;
    p.shares = moves > 512 ? (int)std::max(1l, std::min(moves / 64, 8l * cus / (2 * units))) : 0;
    p.shift_threads = 2 * units * p.columns <= 2l * cus ? 1024 : 256;
    return p;
}

// ---- log probabilities ----
// Workgroups of four waves that a row of logits goes to, and sets of `set` vectors to each (a row that does not start on a 16-byte boundary has up to one vector more)
struct LogprobPlan { int parts, part_sets; };
// Workgroups for every compute unit.  1, 2, 4 and 8: 64 rows of 151936 with twenty alternatives 18.3, 17.0, 16.4 and 20.4 us, without 12.6, 11.6, 11.3 and 12.8; 512 of 128256 without 32.7, 31.4,
// 30.3 and 32.7; 300 of 50257 with five 20.4, 20.3, 22.5 and 23.1; fewer or shorter rows are cut into as many parts as they have either way.
constexpr long kLogprobTarget = 4;
constexpr int kLogprobTickets = 1024;      // rows that may be cut: with more there is a workgroup for every compute unit anyway
inline LogprobPlan logprob_plan(long rows, int vocab, int set, int cus) {
    const long sets = ((vocab + 14) / 8 + set - 1) / set, most = (sets + 3) / 4;
    const long want = rows > kLogprobTickets ? 1 : std::max(1l, std::min(most, kLogprobTarget * cus / std::max(1l, rows)));
    LogprobPlan p;
    p.part_sets = (int)((sets + 4 * want - 1) / (4 * want)) * 4;
    p.parts = (int)((sets + p.part_sets - 1) / p.part_sets);
    return p;
}

}  // namespace ead
