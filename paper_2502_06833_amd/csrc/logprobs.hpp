// Log probabilities of given tokens and of the most likely ones, ranks and entropies, from logits in memory.
#pragma once
#include <type_traits>

#include "common.hpp"

namespace ead {

constexpr int kTopMost = 32;                  // alternatives of a row at most
constexpr int kSetVecs = 4;                   // vectors of 8 logits that a lane holds of a set
constexpr int kSet = 64 * kSetVecs;           // vectors of a set: what a wave takes at a time
constexpr int kLpTicketInts = 32;             // a row's ticket has a cache line of its own
constexpr int kLpSlots = 20;                  // groups of sets whose largest logits a wave remembers, lane by lane

struct LpPartial { float m, Z, S; int above; };
struct LogprobArgs {
    const void *logits;
    long stride;                              // elements from row to row
    int rows, V;
    const int *tokens;                        // null: none
    int top, unit, parts, part_sets;          // a row goes to `parts` workgroups, part_sets sets to each
    float *logprob, *H;
    int *rank, *top_tokens;
    float *top_logprobs;
    int *tickets;                             // parts > 1: [row], zero between launches
    LpPartial *stats;                         // [row][part]
    float *list_value;                        // [row][place][part]: neighbours are of one place, so that the bound of the join is a good one
    int *list_token;
};

// Sums refer to a maximum m: Z = sum 2^d, S = sum 2^d d with d = l log2(e) - m log2(e), one fused operation whose second term is rounded once for all logits: what that
// leaves (lp_rest) is in every d and cancels in what comes out (log2 Z less that rest, log2 Z - S / Z).  Past 2^16, where it would be more than 1/256 and at last overflow 2^d, the difference
// is taken first.
constexpr float kLpLog2e = 1.4426950408889634f, kLpLn2 = 0.6931471805599453f;
__device__ __forceinline__ bool lp_large(float m) { return __builtin_fabsf(m) > 65536.f && m != -INFINITY; }
__device__ __forceinline__ float lp_ref(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float lp_bits(float l, float m) {
    const float ref = lp_ref(m);
    return lp_large(m) ? (l - ref) * kLpLog2e : __builtin_fmaf(l, kLpLog2e, -(ref * kLpLog2e));
}
__device__ __forceinline__ float lp_rest(float m) { return lp_large(m) ? 0.f : __builtin_fmaf(m, kLpLog2e, -(m * kLpLog2e)); }

__device__ __forceinline__ float lp_largest(const float (&f)[8]) {
    return fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
}

struct LpRun {
    float m, Z, S;
    int above;
    __device__ __forceinline__ void init() { m = -INFINITY; Z = 0.f; S = 0.f; above = 0; }
    // the same sums relative to a maximum that is no smaller
    __device__ __forceinline__ void move(float to) {
#pragma clang fp contract(off)                                 // both products rounded, as in d
        if (to == m) return;
        if (m == -INFINITY) { m = to; return; }               // nothing was added yet
        float by;                                              // d of a logit, new minus old
        if (lp_large(m) || lp_large(to)) by = (m - to) * kLpLog2e + (lp_rest(to) - lp_rest(m));
        else by = m * kLpLog2e - to * kLpLog2e;
        by = fmaxf(by, -200.f);
        const float f = __builtin_amdgcn_exp2f(by);
        S = f * (S + by * Z);
        Z *= f;
        m = to;
    }
    __device__ __forceinline__ void add(LpRun o) {
        const float to = fmaxf(m, o.m);
        move(to);
        o.move(to);
        Z += o.Z; S += o.S; above += o.above;
    }
};

// The k largest logits seen so far, sorted: lane i has the i-th, (-inf, kNoIndex) where there is none.  Equal ones: the lower token first.
struct LpList {
    float v;
    int t;
    __device__ __forceinline__ void init() { v = -INFINITY; t = kNoIndex; }
    __device__ __forceinline__ void insert(float cv, int ct, int lane) {
        const int at = __popcll(__ballot(v > cv || (v == cv && t < ct)));
        const float pv = __uint_as_float((uint32_t)__shfl_up((int)__float_as_uint(v), 1, kWave));
        const int pt = __shfl_up(t, 1, kWave);
        v = lane < at ? v : lane == at ? cv : pv;
        t = lane < at ? t : lane == at ? ct : pt;
    }
    __device__ __forceinline__ float last(int k) const { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), k - 1)); }
    __device__ __forceinline__ int last_token(int k) const { return __builtin_amdgcn_readlane(t, k - 1); }
    // one candidate to a lane
    __device__ __forceinline__ void offer(float cv, int ct, bool is, int k, int lane) {
        const float kv = last(k);
        const int kt = last_token(k);
        for (uint64_t hit = __ballot(is && (cv > kv || (cv == kv && ct < kt))); hit; hit &= hit - 1) {
            const int l = __builtin_ctzll(hit);
            insert(__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(cv), l)), __builtin_amdgcn_readlane(ct, l), lane);
        }
    }
};

// Order of floats as whole numbers, and back
__device__ __forceinline__ uint32_t lp_rank(float f) { const uint32_t u = __float_as_uint(f); return u & 0x80000000u ? ~u : u | 0x80000000u; }
__device__ __forceinline__ float lp_value(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r & 0x7FFFFFFFu : ~r); }

// A row's logits as vectors of 8 from a 16-byte boundary on: logit i is element i + shift.  Vectors that reach past the row's ends are read element by element, -inf
// where there is no logit, which adds nothing to any result.
template <typename T>
struct LpRow {
    const T *base, *row;
    int shift, V, vecs, whole0, whole1;       // vectors whole0 .. whole1 - 1 are whole
    __device__ __forceinline__ LpRow(const LogprobArgs &a, int r) {
        row = (const T *)a.logits + (size_t)r * a.stride;
        V = a.V;
        shift = (int)(((uintptr_t)row & 15) / sizeof(T));
        base = row - shift;
        vecs = (V + shift + 7) >> 3;
        whole0 = shift ? 1 : 0;
        whole1 = (V + shift) >> 3;
    }
    __device__ __forceinline__ void load(Vec8<T> (&s)[kSetVecs], int set, int lane) const {
        const int v0 = set * kSet;
        if (v0 >= whole0 && v0 + kSet <= whole1) {
#pragma unroll
            for (int i = 0; i < kSetVecs; ++i) s[i].load_stream(base + (size_t)(v0 + i * 64 + lane) * 8);
            return;
        }
#pragma unroll
        for (int i = 0; i < kSetVecs; ++i) load_one(s[i], v0 + i * 64 + lane);
    }
    // any vector
    __device__ __forceinline__ void load_one(Vec8<T> &s, int v) const {
        if (v >= whole0 && v < whole1) { s.load(base + (size_t)v * 8); return; }
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = v * 8 + e - shift;
            f[e] = j >= 0 && j < V ? to_f32(row[j]) : -INFINITY;
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s.raw[e] = __float_as_uint(f[2 * e]) >> 16 | (__float_as_uint(f[2 * e + 1]) & 0xFFFF0000u);
        } else {
            s.lo = f32x4e_t{f[0], f[1], f[2], f[3]};
            s.hi = f32x4e_t{f[4], f[5], f[6], f[7]};
        }
    }
};

// ---- the most likely tokens ----------------------------------------------------------------------
// While the sums are taken each lane only notes the largest logit of every group of its sets.  The k-th largest of 128 disjoint parts' largest logits (two waves' lanes
// together, lane by lane) is a bound from below for the k-th largest logit, and few more than k logits reach it (37 expected where k is 32): the groups that do are read
// again, what reaches the bound is collected, and each collected logit's place is the number of those before it.  Where more than 64 reach it (many equal logits) the row
// is gone through once more with a list that is kept sorted (LpList).
// The k-th largest of 128 values, two to a lane, -inf where fewer are above that.  HALF: of bf16 values, whose lower halves are 0 (or all ones below 0, which a bound need
// not have)
template <bool HALF> __device__ __forceinline__ float lp_kth(float v, float w, int k) {
    const uint32_t kv = lp_rank(v), kw = lp_rank(w);
    uint32_t t = 0;
    for (int bit = 31; bit >= (HALF ? 16 : 0); --bit) {
        const uint32_t tried = t | 1u << bit;
        if (__popcll(__ballot(kv >= tried)) + __popcll(__ballot(kw >= tried)) >= k) t = tried;
    }
    const float f = lp_value(t);
    return f == f ? f : -INFINITY;
}
// A wave's collected logits: the n-th to its n-th place; 64 at most are kept, and counted on
struct LpCollect {
    float v[64];
    int t[64];
};
__device__ __forceinline__ void lp_collect(LpCollect &c, int &n, float v, int t, bool is, int lane) {
    const uint64_t hit = __ballot(is);
    if (!hit) return;
    const int at = n + __popcll(hit & ((1ull << lane) - 1));
    if (is && at < 64) { c.v[at] = v; c.t[at] = t; }
    n += __popcll(hit);
}
// The place of a lane's logit among the first n lanes' (64 for the others): larger ones first, of equal ones the lower token
__device__ __forceinline__ int lp_place(float v, int t, int n, int lane) {
    const uint64_t key = (uint64_t)lp_rank(v + 0.f) << 32 | (uint32_t)~t;
    int place = 0;
    for (int j = 0; j < n; ++j) {
        const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)key, j);
        place += other > key;
    }
    return lane < n ? place : 64;
}

// One pass over a row: four waves take sets of 64 x 4 vectors in turn, one in hand and the next on its way; sums, the count of larger logits (scalar: a comparison
// and a population count) and the largest are each lane's own until the end.  Rows that would leave compute units idle are cut into parts, and the last to arrive joins
// them in their order (logprob_plan).  About 11 vector-issue slots a logit, exponential included: 2048 rows of 128256 bf16 logits 97 us (5.4 TB/s), 1023 of 50257 float32
// 42.6 us (4.8 TB/s, every wave's start and end in it).  Small calls are latency: one row of 128256 with five alternatives 9.4 us, 64 rows of 151936 with twenty 16.2 us,
// of which in the last workgroup 5 for the sums, 1.1 for the bound, 2 for the collection, 1.5 for the places, 1.1 for the ticket, 3.2 for the join; without alternatives 6.8
// and 10.8.  (Lists that every wave kept sorted while it read took 10.9 and 43 us.)  All logits equal: 54 us for the 64 rows.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprobs(LogprobArgs a) {
    __shared__ float s_m[4], s_Z[4], s_S[4];
    __shared__ int s_above[4], s_last;
    __shared__ float s_best[TOP ? 4 : 1][TOP ? kLpSlots : 1][64], s_lv[TOP ? 4 : 1][kTopMost];
    __shared__ float s_lane[TOP ? 4 : 1][64];
    __shared__ int s_group[TOP ? 4 : 1][64], s_lt[TOP ? 4 : 1][kTopMost];
    __shared__ LpCollect s_c[TOP ? 4 : 1];
    __shared__ int s_n[4];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int r = (int)blockIdx.x / a.parts, part = (int)blockIdx.x % a.parts;
    const LpRow<T> row(a, r);
    const int begin = part * a.part_sets + wave, end = min((row.vecs + kSet - 1) / kSet, (part + 1) * a.part_sets);
    const int sets = begin < end ? (end - begin + 3) / 4 : 0, each = (sets + kLpSlots - 1) / kLpSlots;       // this wave's: begin, begin + 4, ...; of a group

    Vec8<T> A[kSetVecs], B[kSetVecs];
    if (sets > 0) row.load(A, begin, lane);
    if (sets > 1) row.load(B, begin + 4, lane);
    const int token = a.tokens ? __builtin_amdgcn_readfirstlane(a.tokens[r]) : -1;
    const bool given = token >= 0 && token < a.V;
    const float mine = given ? to_f32(row.row[token]) : INFINITY;
    LpRun run;
    run.init();
    int above = 0, of_group = 0, slot = 0;
    float best = -INFINITY;
    float topA[kSetVecs], topB[kSetVecs];                      // the largest logits of the vectors in A and B
    auto take = [&](const Vec8<T> (&s)[kSetVecs], float (&tops)[kSetVecs]) {
        float f[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kSetVecs; ++i) {
            s[i].unpack(f);
            tops[i] = lp_largest(f);
            top = fmaxf(top, tops[i]);
        }
        const float m = fmaxf(run.m, top);
        run.move(m);
        const float off = -(lp_ref(m) * kLpLog2e);
        auto add = [&](auto large_c) {
#pragma unroll
            for (int i = 0; i < kSetVecs; ++i) {
                s[i].unpack(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = decltype(large_c)::value ? lp_bits(f[e], m) : __builtin_fmaf(f[e], kLpLog2e, off);
                    const float x = __builtin_amdgcn_exp2f(d);     // NaN stays one, in Z; -inf is 0, and adds 0 * -200 to S
                    run.Z += x;
                    run.S = __builtin_fmaf(x, fmaxf(d, -200.f), run.S);
                    above += __popcll(__ballot(f[e] > mine));
                }
            }
        };
        if (__any(lp_large(m))) add(std::true_type{});
        else add(std::false_type{});
        if constexpr (TOP) {
            best = fmaxf(best, top);
            if (++of_group == each) {
                s_best[wave][slot++][lane] = best;
                best = -INFINITY;
                of_group = 0;
            }
        }
    };
    for (int set = begin; set < end; set += 8) {               // one in hand, the next on its way
        take(A, topA);
        if (set + 8 < end) row.load(A, set + 8, lane);
        if (set + 4 < end) take(B, topB);
        if (set + 12 < end) row.load(B, set + 12, lane);
    }
    if (TOP && of_group) s_best[wave][slot++][lane] = best;

    // ---- the workgroup's: waves in order, lanes in the order of the exchange
    const float lane_best = run.m, wm = wave_max(run.m);
    run.move(wm);
    run.Z = wave_sum(run.Z);
    run.S = wave_sum(run.S);
    if (lane == 0) { s_m[wave] = wm; s_Z[wave] = run.Z; s_S[wave] = run.S; s_above[wave] = above; }
    LpList list;
    list.init();
    int place = 64, top_t = kNoIndex, collected = 0;                          // wave 0: this lane's token and its place among the most likely, once they are known
    float top_v = -INFINITY;
    if constexpr (TOP) {
        s_lane[wave][lane] = lane_best;
        __syncthreads();
        const float bound = lp_kth<sizeof(T) == 2>(fmaxf(s_lane[0][lane], s_lane[1][lane]), fmaxf(s_lane[2][lane], s_lane[3][lane]), a.top);
        const float least = fmaxf(bound, -3.402823466e38f);   // what is -inf is no candidate
        int found = 0;
        auto collect = [&](const Vec8<T> (&s)[kSetVecs], const float (&tops)[kSetVecs], int first_vec) {
#pragma unroll
            for (int i = 0; i < kSetVecs; ++i) {
                if (!__any(tops[i] >= least)) continue;
                float f[8];
                s[i].unpack(f);
                const int first = (first_vec + i * 64) * 8 - row.shift;
#pragma unroll
                for (int e = 0; e < 8; ++e) lp_collect(s_c[wave], found, f[e], first + e, f[e] >= least, lane);
            }
        };
        // this wave's groups that reach the bound; two sets are still in registers
        int n = 0;
        if (sets <= 2) {
            slot = 0;
            if (sets > 0) collect(A, topA, begin * kSet + lane);
            if (sets > 1) collect(B, topB, (begin + 4) * kSet + lane);
        }
        for (int i = 0; i < slot; ++i) {
            const float b = s_best[wave][i][lane];
            const uint64_t hit = __ballot(b >= least);
            if (!hit) continue;
            const int at = n + __popcll(hit & ((1ull << lane) - 1));
            if ((hit >> lane & 1) && at < 64) s_group[wave][at] = i * 64 + lane;
            n += __popcll(hit);
        }
        if (n > 64) found = 65;
        if (n <= 64 && n > 0) {
            const int id = lane < n ? s_group[wave][lane] : 0;
            for (int j = 0; j < each; ++j) {
                const int at = (id >> 6) * each + j;           // the wave's set
                const bool in = lane < n && at < sets;
                Vec8<T> s[kSetVecs];
                float tops[kSetVecs];
#pragma unroll
                for (int i = 0; i < kSetVecs; ++i) {
                    s[i].zero();
                    if (in) row.load_one(s[i], (begin + 4 * at) * kSet + i * 64 + (id & 63));
                }
#pragma unroll
                for (int i = 0; i < kSetVecs; ++i) {
                    float f[8];
                    s[i].unpack(f);
                    tops[i] = in ? lp_largest(f) : -INFINITY;
                }
                if (least > 0.f || __all(in)) collect(s, tops, (begin + 4 * at) * kSet + (id & 63));
                else                                           // (the zeros of lanes that have no group would count)
#pragma unroll
                    for (int i = 0; i < kSetVecs; ++i) {
                        float f[8];
                        s[i].unpack(f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) lp_collect(s_c[wave], found, f[e], ((begin + 4 * at) * kSet + (id & 63) + i * 64) * 8 - row.shift + e, in && f[e] >= least, lane);
                    }
            }
        }
        if (lane == 0) s_n[wave] = found;
        __syncthreads();
        collected = s_n[0] + s_n[1] + s_n[2] + s_n[3];
        if (collected > 64) {                                  // this wave's sets once more, with a sorted list
            for (int at = begin; at < end; at += 4) {
                row.load(A, at, lane);
#pragma unroll
                for (int i = 0; i < kSetVecs; ++i) {
                    float f[8];
                    A[i].unpack(f);
                    const float top = lp_largest(f);
                    if (!__any(top > list.last(a.top) && top >= bound)) continue;
                    const int first = (at * kSet + i * 64 + lane) * 8 - row.shift;
#pragma unroll 1
                    for (int e = 0; e < 8; ++e) {
                        float v = f[0];
#pragma unroll
                        for (int j = 1; j < 8; ++j) v = e == j ? f[j] : v;
                        list.offer(v, first + e, v > -INFINITY && v >= bound, a.top, lane);
                    }
                }
            }
            if (lane < kTopMost) { s_lv[wave][lane] = list.v; s_lt[wave][lane] = list.t; }
        }
    }
    __syncthreads();
    auto join_sums = [&] {
        run.m = s_m[0]; run.Z = s_Z[0]; run.S = s_S[0]; run.above = s_above[0];
        for (int w = 1; w < 4; ++w) { LpRun o; o.m = s_m[w]; o.Z = s_Z[w]; o.S = s_S[w]; o.above = s_above[w]; run.add(o); }
    };
    auto join_lists = [&] {                                    // by wave 0
        if constexpr (TOP) {
            if (collected <= 64) {
                int w = 0, at = lane;
                while (w < 3 && at >= s_n[w]) at -= s_n[w++];
                if (lane < collected) { top_v = s_c[w].v[at]; top_t = s_c[w].t[at]; }
                place = lp_place(top_v, top_t, collected, lane);
                return;
            }
            list.v = lane < kTopMost ? s_lv[0][lane] : -INFINITY;
            list.t = lane < kTopMost ? s_lt[0][lane] : kNoIndex;
            for (int w = 1; w < 4; ++w) {
                const bool is = lane < a.top;
                list.offer(is ? s_lv[w][lane] : 0.f, is ? s_lt[w][lane] : 0, is, a.top, lane);
            }
            top_v = list.v; top_t = list.t; place = list.t == kNoIndex ? 64 : lane;
        }
    };
    if (a.parts > 1) {
        const size_t at = (size_t)r * a.parts + part;
        // wave 0 has the list, wave 1 the sums meanwhile (and without a list both)
        if (wave == (TOP ? 1 : 0)) {
            join_sums();
            if (lane == 0) {
                LpPartial *p = a.stats + at;
                st_coherent(&p->m, run.m); st_coherent(&p->Z, run.Z); st_coherent(&p->S, run.S); st_coherent(&p->above, run.above);
            }
            wait_stores();
        }
        if constexpr (TOP) {
            if (wave == 0) {
                join_lists();
                const int have = __popcll(__ballot(place < a.top));
                const size_t to = (size_t)r * a.parts * a.top + part;
                if (place < a.top) { st_coherent(a.list_value + to + place * a.parts, top_v); st_coherent(a.list_token + to + place * a.parts, top_t); }
                if (lane >= have && lane < a.top) { st_coherent(a.list_value + to + lane * a.parts, -INFINITY); st_coherent(a.list_token + to + lane * a.parts, kNoIndex); }
                wait_stores();
            }
            __syncthreads();
        }
        if (wave == 0) {
            if (lane == 0) {
                int *ticket = a.tickets + (size_t)r * kLpTicketInts;
                const bool last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts - 1;
                if (last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = last;
            }
        }
        __syncthreads();
        if (!s_last || wave) return;
        // the last to arrive joins the parts in their order, whoever it is
        const size_t first = (size_t)r * a.parts;
        const int total = a.parts * a.top;
        const float *values = a.list_value + first * a.top;
        const int *tokens = a.list_token + first * a.top;
        constexpr int kHeld = TOP ? 6 : 0;                     // candidates that a lane asks for at once
        float held_v[kHeld + 1];
        int held_t[kHeld + 1];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            const bool in = j * 64 + lane < total;
            held_v[j] = in ? ld_coherent(values + j * 64 + lane) : -INFINITY;
            held_t[j] = in ? ld_coherent(tokens + j * 64 + lane) : kNoIndex;
        }
        run.init();
        for (int p = lane; p < a.parts; p += 64) {
            const LpPartial *q = a.stats + first + p;
            LpRun o;
            o.m = ld_coherent(&q->m); o.Z = ld_coherent(&q->Z); o.S = ld_coherent(&q->S); o.above = ld_coherent(&q->above);
            run.add(o);
        }
        if constexpr (TOP) {
            float most = -INFINITY, most_too = -INFINITY;
#pragma unroll
            for (int j = 0; j < kHeld; ++j) (j & 1 ? most_too : most) = fmaxf(j & 1 ? most_too : most, held_v[j]);
            for (int i = kHeld * 64 + lane; i < total; i += 64) most = fmaxf(most, ld_coherent(values + i));
            const float bound = lp_kth<sizeof(T) == 2>(most, most_too, a.top);
            int n = 0;
#pragma unroll
            for (int j = 0; j < kHeld; ++j) lp_collect(s_c[0], n, held_v[j], held_t[j], held_v[j] >= bound && held_v[j] > -INFINITY, lane);
            for (int i = kHeld * 64; i < total; i += 64) {
                const bool in = i + lane < total;
                const float v = in ? ld_coherent(values + i + lane) : -INFINITY;
                lp_collect(s_c[0], n, v, in ? ld_coherent(tokens + i + lane) : 0, v >= bound && v > -INFINITY, lane);
            }
            __builtin_amdgcn_wave_barrier();                   // LDS serves a wave's accesses in order: what its lanes wrote is there for all of them
            if (n <= 64) {
                if (lane < n) { top_v = s_c[0].v[lane]; top_t = s_c[0].t[lane]; }
                else { top_v = -INFINITY; top_t = kNoIndex; }
                place = lp_place(top_v, top_t, n, lane);
            } else {
                list.init();
                for (int i = 0; i < total; i += 64) {
                    const bool in = i + lane < total;
                    list.offer(in ? ld_coherent(values + i + lane) : -INFINITY, in ? ld_coherent(tokens + i + lane) : kNoIndex, in, a.top, lane);
                }
                top_v = list.v; top_t = list.t; place = list.t == kNoIndex ? 64 : lane;
            }
        }
        const float pm = wave_max(run.m);
        run.move(pm);
        run.Z = wave_sum(run.Z);
        run.S = wave_sum(run.S);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) run.above += __shfl_xor(run.above, o, kWave);
    } else {
        if (wave) return;
        join_sums();
        join_lists();
    }
    // nothing above -inf, or something that is no number: no distribution
    const bool some = run.Z > 0.f && run.Z < INFINITY;
    const float log2z = some ? log2f(run.Z) : __builtin_nanf(""), lnz = (log2z - lp_rest(lp_ref(run.m))) * kLpLn2;
    if (lane == 0) {
        // (where one token is certain, roundings leave a few 1e-9 of either sign)
        const float h = (log2z - run.S / run.Z) * (a.unit ? 1.f : kLpLn2);
        if (a.H) a.H[r] = h < 0.f ? 0.f : h;
        const float lp = (mine - run.m) - lnz;
        if (a.logprob) a.logprob[r] = !given || lp > 0.f ? 0.f : lp;
        if (a.rank) a.rank[r] = given ? run.above + 1 : 0;
    }
    if constexpr (TOP) {
        // rows with fewer logits above -inf than were asked for: the lowest other tokens
        const int have = __popcll(__ballot(place < a.top));
        int t = 0;
        for (int i = have; i < a.top; ++i) {
            while (__any(place < a.top && top_t == t)) ++t;
            const uint64_t idle = __ballot(place >= a.top);
            if (lane == __builtin_ctzll(idle)) { place = i; top_t = t; top_v = -INFINITY; }
        }
        if (place < a.top) {
            const float lp = (top_v - run.m) - lnz;
            a.top_tokens[(size_t)r * a.top + place] = top_t;
            a.top_logprobs[(size_t)r * a.top + place] = lp > 0.f ? 0.f : lp;
        }
    }
}

}  // namespace ead
