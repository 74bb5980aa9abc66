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
    int keep, sinks, recent;
    int cached;                     // scores that the workgroup's LDS holds
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

// One workgroup to a (sequence, KV head).  The threshold comes from histograms of the scores' ranks, 11, 11 and 10 bits at a time from the top; of those that equal it
// the lowest positions stay.  Free places below the cut and chosen positions past it, both in ascending order, make the moves.
__global__ __launch_bounds__(kEvictThreads) void k_evict_choose(PagedEvict c) {
    extern __shared__ uint32_t lds[];                     // ranks of the first c.cached positions
    __shared__ int bins[kEvictBins];
    __shared__ int part[17], found[2];
    const int tid = (int)threadIdx.x, threads = (int)blockDim.x, lane = tid & 63, wave = tid >> 6, waves = threads / 64;
    const int h = (int)blockIdx.x, b = (int)blockIdx.y;
    const PagedSeq s = paged_seq(c.a, b);
    const size_t unit = (size_t)b * c.a.n_kv + h;
    int *kept = c.kept + unit * c.keep;
    const int n = s.kv, cut = c.keep - c.recent, middle = n - c.recent;      // middle: end of those that are asked
    for (int i = tid; i < c.keep; i += threads) kept[i] = n <= c.keep ? (i < n ? i : -1) : i < cut ? i : n - c.keep + i;
    if (n <= c.keep) {
        if (tid == 0) c.counts[unit] = 0;
        return;
    }
    const int mask = (1 << c.a.page_shift) - 1;
    auto load = [&](int i) {
        const int page = paged_page(c.a, s, i);
        return page < 0 ? kEvictNothing : evict_rank(c.scores[paged_vec(c.a, page, h, i & mask)]);
    };
    const int here = min(middle, c.cached);
    for (int i0 = tid; i0 < here; i0 += threads * kEvictAhead) {
        int page[kEvictAhead];
        float f[kEvictAhead];
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) page[e] = paged_page(c.a, s, min(i0 + e * threads, here - 1));
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e) f[e] = c.scores[paged_vec(c.a, max(page[e], 0), h, min(i0 + e * threads, here - 1) & mask)];
#pragma unroll
        for (int e = 0; e < kEvictAhead; ++e)
            if (i0 + e * threads < here) lds[i0 + e * threads] = page[e] < 0 ? kEvictNothing : evict_rank(f[e]);
    }
    __syncthreads();
    auto rank = [&](int i) { return i < c.cached ? lds[i] : load(i); };
    // ---- the threshold: the (cut - sinks)-th largest
    int need = cut - c.sinks;                             // still to be found among those that share the bits so far
    uint32_t prefix = 0;
    int shift = 32;
    if (need > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass < 2 ? 11 : 10, low = shift - bits;
            for (int i = tid; i < kEvictBins; i += threads) bins[i] = 0;
            __syncthreads();
            for (int i = c.sinks + tid; i < middle; i += threads) {
                const uint32_t r = rank(i);
                if (pass == 0 || r >> shift == prefix) atomicAdd(&bins[(r >> low) & ((1u << bits) - 1)], 1);
            }
            __syncthreads();
            // every thread adds up some bins, the largest first; the one within whose bins the count is reached says which it is
            const int own = (1 << bits) / threads, top = (1 << bits) - 1 - tid * own;
            int sum = 0;
            for (int e = 0; e < own; ++e) sum += bins[top - e];
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int t = __shfl_up(upto, o, kWave);
                upto += lane >= o ? t : 0;
            }
            upto += evict_before(__builtin_amdgcn_readlane(upto, 63), part).x;
            if (upto >= need && upto - sum < need) {
                int left = need - (upto - sum), e = 0;
                while (bins[top - e] < left) left -= bins[top - e++];
                found[0] = top - e;
                found[1] = left;
            }
            __syncthreads();
            prefix = prefix << bits | (uint32_t)found[0];
            need = found[1];
            shift = low;
        }
    }
    // ---- a contiguous piece for each wave, in steps of 64 positions
    const int asked = middle - c.sinks, piece = ((asked + waves * 64 - 1) / (waves * 64)) * 64;
    const int from = c.sinks + wave * piece, to = min(from + piece, middle);
    const uint64_t below = (1ull << lane) - 1;
    const bool none = cut == c.sinks;                     // no place for any of them
    int equal = 0;
    for (int i = from + lane; i - lane < to; i += 64) equal += __popcll(__ballot(i < to && !none && rank(i) == prefix));
    const int equal_before = evict_before(equal, part).x;
    auto walk = [&](auto take) {
        int ties = equal_before;
        for (int i = from + lane; i - lane < to; i += 64) {
            const uint32_t r = i < to ? rank(i) : 0u;
            const uint64_t same = __ballot(i < to && !none && r == prefix);
            const bool stays = i < to && !none && (r > prefix || (r == prefix && ties + __popcll(same & below) < need));
            ties += __popcll(same);
            take(i, __ballot(i < to && i < cut && !stays), __ballot(i < to && i >= cut && stays));
        }
    };
    int n_free = 0, n_late = 0;
    walk([&](int, uint64_t free, uint64_t late) { n_free += __popcll(free); n_late += __popcll(late); });
    const int2 free_at = evict_before(n_free, part), late_at = evict_before(n_late, part);
    int f = free_at.x, l = late_at.x;
    int2 *moves = c.moves + unit * (size_t)max(cut - c.sinks, 0);
    walk([&](int i, uint64_t free, uint64_t late) {
        if (free >> lane & 1) moves[f + __popcll(free & below)].x = i;
        if (late >> lane & 1) moves[l + __popcll(late & below)].y = i;
        f += __popcll(free);
        l += __popcll(late);
    });
    __syncthreads();                                      // the moves are this workgroup's own: what its waves have written is there for all of it
    const int count = free_at.y;                          // as many free places as late ones: the chosen are as many as the places
    for (int i = tid; i < count; i += threads) kept[moves[i].x] = moves[i].y;
    if (tid == 0) c.counts[unit] = count;
}

// One workgroup moves one piece of the vectors of a (sequence, KV head); pieces do not touch each other, so the order within one is all that matters.  First the free
// places are filled, from positions past the cut that nothing is written to meanwhile; then the last positions move down in ascending order, a block of them read before
// it is written.  Where there may be many free places several workgroups share them, in a launch of their own (kEvictFill, then kEvictShift).  Holes give zeros and take
// nothing.
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

__global__ __launch_bounds__(256) void k_evict_move(PagedEvict c) {
    // part: pieces of K, of V, then exponents of K and V, weights
    const int h = (int)blockIdx.x % c.a.n_kv, share = (int)blockIdx.x / c.a.n_kv, part = (int)blockIdx.y, b = (int)blockIdx.z;
    const PagedSeq s = paged_seq(c.a, b);
    if (s.kv <= c.keep) return;
    const size_t unit = (size_t)b * c.a.n_kv + h;
    if (part < 2 * c.columns) {
        char *pool = (char *)(part < c.columns ? c.a.k : c.a.v);
        evict_piece<u32x4_t>(c, s, h, unit, share, pool, c.columns * c.column_bytes, (part % c.columns) * c.column_bytes, c.column_bytes / 16);
    } else if (c.a.ks && part < 2 * c.columns + 2) evict_piece<uint8_t>(c, s, h, unit, share, (char *)(part == 2 * c.columns ? c.a.ks : c.a.vs), 1, 0, 1);
    else evict_piece<float>(c, s, h, unit, share, (char *)c.weights, 4, 0, 1);
}

}  // namespace ead
