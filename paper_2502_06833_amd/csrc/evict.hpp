// A paged cache's sequences cut to a number of positions: which stay (by weight), and the moves that close the gaps.
#pragma once
#include "paged.hpp"

namespace ead {

struct PagedEvict {
    PagedArgs a;
    const float *scores;            // [page][KV head][slot]: what is chosen by
    float *weights;                 // the same layout: moves with the positions
    int *kept;                      // [sequence][KV head][keep]
    int *counts;                    // [sequence][KV head]: moves into free places
    int2 *moves;                    // [sequence][KV head][keep - recent - sinks]: (to, from)
    int keep, sinks, recent, held;  // held: positions of a sequence that the host vouched for; longer ones are left as they are
    int cached;                     // scores that the workgroup's LDS holds, a multiple of 4
    int columns, column_bytes;      // k_evict_move: pieces of a vector, each a workgroup's
    int steps, shares;              // what it does, and the workgroups that share the free places
};

// Order of scores as whole numbers, the largest largest: -0 as 0, NaN below everything
__device__ __forceinline__ uint32_t evict_rank(float f) {
    if (f != f) return 0u;
    const uint32_t u = __float_as_uint(f + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kEvictThreads = 1024, kEvictBins = 2048;
constexpr int kEvictAhead = 4;               // scores, or vectors, that a lane has on their way

constexpr uint32_t kEvictNothing = 0x80000000u;      // the rank of 0: holes

// Sum of `mine` over the waves before this one, and over all (s: 17 ints of LDS).  Called by the whole workgroup with the same value in all lanes of a wave.
__device__ __forceinline__ int2 evict_before(int mine, int *s) {
    const int wave = (int)threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[wave] = mine;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        before += w < wave ? s[w] : 0;
        all += s[w];
    }
    return make_int2(before, all);
}

// A lane's sum with all lanes' before it
__device__ __forceinline__ int evict_upto(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(v, o, kWave);
        v += lane >= o ? t : 0;
    }
    return v;
}

// One workgroup to a (sequence, KV head).  The threshold comes from histograms of the scores' ranks, 11, 11 and 10 bits at a time from the top; of those that equal it
// the lowest positions stay.  Free places below the cut and chosen positions past it, both in ascending order, make the moves.  Latency, for the most part: scores come
// four in a row and kEvictAhead of those at a time, and are read again from LDS; which positions stay is noted 64 to a word, so that ranks are looked at once for the
// threshold's every pass and once for that, after which the chosen positions past the cut are listed in their place.  A pass ends the search where its bin holds no
// more than are needed (mostly the second).  64 sequences of 2049 to 2176 positions, 8 heads: 16.5 us, one workgroup's latency; three of 24001 to 32768: 40 us, of which in a
// workgroup 4.5 for the scores, 9.5 for the passes, 4 for the words, 12 for the moves.
template <bool CACHED>
__device__ __forceinline__ void evict_choose(const PagedEvict &c, const PagedSeq &s, size_t unit, int h, uint32_t *lds, int *bins, int *part, int *found) {
    uint64_t *stays = (uint64_t *)(lds + c.cached);
    const int tid = (int)threadIdx.x, threads = (int)blockDim.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = threads / 64;
    const int cut = c.keep - c.recent, middle = s.kv - c.recent;             // middle: end of those that are asked
    int *kept = c.kept + unit * c.keep;
    const int mask = (1 << c.a.page_shift) - 1;
    auto load4 = [&](int i, int page) { return *(gptr<f32x4e_t>)(c.scores + paged_vec(c.a, max(page, 0), h, i & mask)); };      // four slots of a page: i is a multiple of 4
    const int here = min(middle, c.cached);
    for (int i0 = tid * 4; i0 < here; i0 += threads * 4 * kEvictAhead) {
        int page[kEvictAhead];
        f32x4e_t f[kEvictAhead];
        auto at = [&](int e) { return min(i0 + e * threads * 4, (here - 1) & ~3); };
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) page[e] = paged_page(c.a, s, at(e));
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) f[e] = load4(at(e), page[e]);
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e)
            if (i0 + e * threads * 4 < here)
                *(u32x4_t *)(lds + i0 + e * threads * 4) = page[e] < 0 ? u32x4_t{kEvictNothing, kEvictNothing, kEvictNothing, kEvictNothing}
                                                                       : u32x4_t{evict_rank(f[e].x), evict_rank(f[e].y), evict_rank(f[e].z), evict_rank(f[e].w)};
    }
    __syncthreads();
    auto rank = [&](int i) {
        if (CACHED || i < c.cached) return lds[i];
        const int page = paged_page(c.a, s, i);
        return page < 0 ? kEvictNothing : evict_rank(c.scores[paged_vec(c.a, page, h, i & mask)]);
    };
    // ---- the threshold: the (cut - sinks)-th largest
    int need = cut - c.sinks;                             // still to be found among those that share the bits so far
    const bool none = need == 0;                          // no place for any of them
    uint32_t prefix = 0;
    int shift = 32, alike = 0;                            // alike: those that share them
    for (int pass = 0; pass < 3 && !none && alike != need; ++pass) {
        const int bits = pass < 2 ? 11 : 10, low = shift - bits;
        for (int i = tid; i < kEvictBins; i += threads) bins[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int i = c.sinks + tid; i < middle; i += threads) {
            const uint32_t r = rank(i);
            if (pass == 0 || r >> shift == prefix) atomicAdd(&bins[(r >> low) & ((1u << bits) - 1)], 1);
        }
        __syncthreads();
        // every thread adds up some bins, the largest first; the one within whose bins the count is reached says which it is
        const int own = (1 << bits) / threads, top = (1 << bits) - 1 - tid * own;
        int sum = 0;
        for (int e = 0; e < own; ++e) sum += bins[top - e];
        const int in_wave = evict_upto(sum, lane), upto = in_wave + evict_before(__builtin_amdgcn_readlane(in_wave, 63), part).x;
        if (upto >= need && upto - sum < need) {
            int left = need - (upto - sum), e = 0;
            while (bins[top - e] < left) left -= bins[top - e++];
            found[0] = top - e;
            found[1] = left;
            found[2] = bins[top - e];
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)found[0];
        need = found[1];
        alike = found[2];
        shift = low;
    }
    // ---- a bit for every position that is asked: whether it stays.  A contiguous piece for each wave, 64 positions to a word
    const int words = (middle - c.sinks + 63) / 64, piece = (words + waves - 1) / waves;
    const int from = wave * piece, to = min(from + piece, words);
    // (words are a wave's, kept in scalar registers: as every lane's own their 64-bit operations were most of the time)
    auto scalar_word = [](uint64_t v) { return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    auto below = [](uint64_t v) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(v >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)v, 0u)); };       // bits before this lane's
    const bool ties = !none && alike != need;             // all bits have been looked at, and some of the equal ones go
    int before = 0;
    if (ties) {
        int equal = 0;
        for (int w = from; w < to; ++w) {
            const int i = c.sinks + w * 64 + lane;
            equal += __popcll(__ballot(i < middle && rank(i) == prefix));
        }
        before = evict_before(equal, part).x;
    }
#pragma unroll 4
    for (int w = from; w < to; ++w) {
        const int i = c.sinks + w * 64 + lane;
        const uint32_t r = i < middle ? rank(i) : 0u;
        uint64_t stay = __ballot(i < middle && !none && r >> shift >= prefix);
        if (ties) {
            const uint64_t same = __ballot(i < middle && r == prefix);
            stay &= ~__ballot((same >> lane & 1) && before + below(same) >= need);
            before += __popcll(same);
        }
        if (lane == 0) stays[w] = stay;
    }
    __syncthreads();                                      // ranks are not read after this
    // ---- the moves: free places lie below the cut, chosen positions that have to go there at or past it.  Words go round the waves, `group` neighbours at a time, with
    // the numbers of free places and of late positions before them; one compute unit's issue rate is what bounds this, so that a word is to take few instructions.
    auto bits_of = [&](int w, uint64_t stay, uint64_t &free, uint64_t &late) {
        const int i0 = c.sinks + w * 64;
        const uint64_t low = i0 >= cut ? 0 : i0 + 64 <= cut ? ~0ull : (1ull << (cut - i0)) - 1, in = middle - i0 >= 64 ? ~0ull : (1ull << (middle - i0)) - 1;
        free = ~stay & low & in;
        late = stay & ~low;
    };
    constexpr int kGroups = kEvictBins / 2;
    const int group = (words + kGroups - 1) / kGroups, groups = (words + group - 1) / group;
    int *free_before = bins, *late_before = bins + kGroups;
    const int mine = (kGroups + threads - 1) / threads;  // groups of a thread, side by side
    int n_free = 0, n_late = 0;
    for (int g = tid * mine; g < min((tid + 1) * mine, groups); ++g) {
        free_before[g] = n_free;
        late_before[g] = n_late;
        for (int w = g * group; w < min((g + 1) * group, words); ++w) {
            uint64_t free, late;
            bits_of(w, stays[w], free, late);
            n_free += __popcll(free);
            n_late += __popcll(late);
        }
    }
    const int free_upto = evict_upto(n_free, lane), late_upto = evict_upto(n_late, lane);
    const int free_first = free_upto - n_free + evict_before(__builtin_amdgcn_readlane(free_upto, 63), part).x;
    const int2 of_late = evict_before(__builtin_amdgcn_readlane(late_upto, 63), part);
    const int count = of_late.y;                          // as many as free places: the chosen are as many as the places
    for (int g = tid * mine; g < min((tid + 1) * mine, groups); ++g) {
        free_before[g] += free_first;
        late_before[g] += late_upto - n_late + of_late.x;
    }
    __syncthreads();
    const bool listed = count <= c.cached;                // in place of the ranks
    int2 *moves = c.moves + unit * (size_t)max(cut - c.sinks, 0);
    const int cut_word = (cut - c.sinks) / 64;           // the one word that may have both
    for (int g = cut_word / group + (wave + waves - cut_word / group % waves) % waves; g < groups; g += waves) {
        int l = __builtin_amdgcn_readfirstlane(late_before[g]);
        for (int w = g * group; w < min((g + 1) * group, words); ++w) {
            uint64_t free, late;
            bits_of(w, scalar_word(stays[w]), free, late);
            const unsigned at = (unsigned)(l + below(late)), i = (unsigned)(c.sinks + w * 64 + lane);
            if (listed) { if (__builtin_amdgcn_inverse_ballot_w64(late)) lds[at] = i; }
            else if (__builtin_amdgcn_inverse_ballot_w64(late)) moves[at].y = (int)i;
            l += __popcll(late);
        }
    }
    __syncthreads();                                      // also the moves are this workgroup's own: what its waves have written is there for all of it
    for (int g = wave; g <= min(cut_word / group, groups - 1); g += waves) {
        int f = __builtin_amdgcn_readfirstlane(free_before[g]);
        for (int w = g * group; w < min((g + 1) * group, words); ++w) {
            uint64_t free, late;
            bits_of(w, scalar_word(stays[w]), free, late);
            const unsigned at = (unsigned)(f + below(free)), i = (unsigned)(c.sinks + w * 64 + lane);
            if (__builtin_amdgcn_inverse_ballot_w64(free)) {
                const int of = listed ? (int)lds[at] : moves[at].y;
                moves[at] = make_int2((int)i, of);
                kept[i] = of;
            }
            f += __popcll(free);
        }
    }
    if (tid == 0) c.counts[unit] = count;
}

__global__ __launch_bounds__(kEvictThreads) void k_evict_choose(PagedEvict c) {
    extern __shared__ __align__(16) uint32_t lds[];       // ranks of the first c.cached positions (written four at a time), then a bit for every position, 64 to a word
    __shared__ int bins[kEvictBins];
    __shared__ int part[17], found[3];
    const int h = (int)blockIdx.x, b = (int)blockIdx.y;
    const PagedSeq s = paged_seq(c.a, b);
    const size_t unit = (size_t)b * c.a.n_kv + h;
    int *kept = c.kept + unit * c.keep;
    const int n = s.kv, cut = c.keep - c.recent;
    for (int i = (int)threadIdx.x; i < c.keep; i += (int)blockDim.x) kept[i] = n <= c.keep ? (i < n ? i : -1) : n > c.held ? -1 : i < cut ? i : n - c.keep + i;
    if (n <= c.keep || n > c.held) {
        if (threadIdx.x == 0) c.counts[unit] = 0;
        return;
    }
    __syncthreads();                                      // (some places are written once more, by other threads)
    if (n - c.recent <= c.cached) evict_choose<true>(c, s, unit, h, lds, bins, part, found);
    else evict_choose<false>(c, s, unit, h, lds, bins, part, found);
}

// One workgroup moves one piece of the vectors of a (sequence, KV head); pieces do not touch each other, so the order within one is all that matters.  First the free
// places are filled, from positions past the cut that nothing is written to meanwhile; then the last positions move down in ascending order, a block of them read before
// it is written.  Where there may be many free places several workgroups share them, in a launch of their own (kEvictFill, then kEvictShift).  Holes give zeros and take
// nothing.  64 sequences, 8 heads of 128 8-bit elements, some 60 places and 256 last positions each: 18 us (5 TB/s); three sequences of some 28000 bf16 positions, 6500 places each:
// 38 us for the places (4.3 TB/s), 9 for the 1023 last positions, in pieces of 64 bytes.
enum { kEvictFill = 1, kEvictShift = 2 };
template <typename T>
__device__ __forceinline__ void evict_piece(const PagedEvict &c, const PagedSeq &s, int h, size_t unit, int share, char *pool, int vec_bytes, int at, int lanes) {
    const int mask = (1 << c.a.page_shift) - 1, per = (int)blockDim.x / lanes, lane = (int)threadIdx.x % lanes, first = (int)threadIdx.x / lanes;
    auto place = [&](int page, int pos) { return (T *)(pool + paged_vec(c.a, max(page, 0), h, pos & mask) * vec_bytes + at) + lane; };
    const int cut = c.keep - c.recent;
    if (c.steps & kEvictFill) {
        const int count = c.counts[unit];
        const int2 *moves = c.moves + unit * (size_t)max(cut - c.sinks, 0);
        for (int i0 = share * per * kEvictAhead; i0 < count; i0 += c.shares * per * kEvictAhead) {
            int2 m[kEvictAhead];
            int from[kEvictAhead], to[kEvictAhead];
            T v[kEvictAhead];
#pragma unroll
            for (int e = 0; e < kEvictAhead; ++e) m[e] = moves[min(i0 + e * per + first, count - 1)];
#pragma unroll
            for (int e = 0; e < kEvictAhead; ++e) { from[e] = paged_page(c.a, s, m[e].y); to[e] = paged_page(c.a, s, m[e].x); }
#pragma unroll
            for (int e = 0; e < kEvictAhead; ++e) v[e] = *place(from[e], m[e].y);
#pragma unroll
            for (int e = 0; e < kEvictAhead; ++e)
                if (i0 + e * per + first < count && to[e] >= 0) *place(to[e], m[e].x) = from[e] >= 0 ? v[e] : T{};
        }
    }
    if (!(c.steps & kEvictShift)) return;
    const int down = s.kv - c.keep;
    for (int i0 = cut; i0 < c.keep; i0 += per * kEvictAhead) {
        int from[kEvictAhead], to[kEvictAhead];
        T v[kEvictAhead];
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) {
            const int i = min(i0 + e * per + first, c.keep - 1);
            from[e] = paged_page(c.a, s, i + down);
            to[e] = paged_page(c.a, s, i);
        }
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) v[e] = *place(from[e], min(i0 + e * per + first, c.keep - 1) + down);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) {
            const int i = i0 + e * per + first;
            if (i < c.keep && to[e] >= 0) *place(to[e], i) = from[e] >= 0 ? v[e] : T{};
        }
    }
}

__global__ __launch_bounds__(1024) void k_evict_move(PagedEvict c) {
    // part: pieces of K, of V, then exponents of K and V, weights
    const int h = (int)blockIdx.x % c.a.n_kv, share = (int)blockIdx.x / c.a.n_kv, part = (int)blockIdx.y, b = (int)blockIdx.z;
    const PagedSeq s = paged_seq(c.a, b);
    if (s.kv <= c.keep || s.kv > c.held) return;
    const size_t unit = (size_t)b * c.a.n_kv + h;
    if (part < 2 * c.columns) {
        char *pool = (char *)(part < c.columns ? c.a.k : c.a.v);
        evict_piece<u32x4_t>(c, s, h, unit, share, pool, c.columns * c.column_bytes, (part % c.columns) * c.column_bytes, c.column_bytes / 16);
    } else if (c.a.ks && part < 2 * c.columns + 2) evict_piece<uint8_t>(c, s, h, unit, share, (char *)(part == 2 * c.columns ? c.a.ks : c.a.vs), 1, 0, 1);
    else evict_piece<float>(c, s, h, unit, share, (char *)c.weights, 4, 0, 1);
}

}  // namespace ead
