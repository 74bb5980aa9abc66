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
    float *list_value;                        // [row][part][top]
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
// While the sums are taken each lane only notes the largest logit of every group of its sets.  The k-th largest of 64 disjoint parts' largest logits (the four waves' lanes,
// lane by lane) is a bound from below for the k-th largest logit, and hardly more than k logits reach it: the groups that do are read again, what reaches the bound is
// collected, and each collected logit's place is the number of those before it.  Where more than 64 reach it (many equal logits) the row is gone through once more with
// a list that is kept sorted (LpList).
struct LpCollect {
    float bound;
    int count, groups[4];                     // collected; groups of a wave
    float v[64];
    int t[64];
};

// The k-th largest of 64 lanes' values, -inf where fewer are above that
template <bool HALF> __device__ __forceinline__ float lp_kth(float v, int k) {
    const uint32_t key = lp_rank(v);
    uint32_t t = 0;
    for (int bit = 31; bit >= (HALF ? 16 : 0); --bit)                     // bf16 values: the lower halves are 0 (or all ones below 0, which the bound need not have)
        if (__popcll(__ballot(key >= (t | 1u << bit))) >= k) t |= 1u << bit;
    const float f = lp_value(t);
    return f == f ? f : -INFINITY;
}
__device__ __forceinline__ void lp_collect(LpCollect &c, float v, int t, bool is, int lane) {
    const uint64_t hit = __ballot(is);
    if (!hit) return;
    int at = 0;
    if (lane == __builtin_ctzll(hit)) at = atomicAdd(&c.count, __popcll(hit));
    at = __shfl(at, __builtin_ctzll(hit), kWave) + __popcll(hit & ((1ull << lane) - 1));
    if (is && at < 64) { c.v[at] = v; c.t[at] = t; }
}
// Lane i's collected logit and its place among them (64 and more: there is none)
__device__ __forceinline__ int lp_place(const LpCollect &c, int n, int lane, float &v, int &t) {
    v = lane < n ? c.v[lane] : -INFINITY;
    t = lane < n ? c.t[lane] : kNoIndex;
    int place = 0;
    for (int j = 0; j < n; ++j) {
        const float ov = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), j));
        const int ot = __builtin_amdgcn_readlane(t, j);
        place += ov > v || (ov == v && ot < t);
    }
    return lane < n ? place : 64;
}

template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprobs(LogprobArgs a) {
    __shared__ float s_m[4], s_Z[4], s_S[4];
    __shared__ int s_above[4], s_last;
    __shared__ float s_best[TOP ? 4 : 1][TOP ? kLpSlots : 1][64], s_lv[TOP ? 4 : 1][kTopMost];
    __shared__ int s_group[TOP ? 4 : 1][64], s_lt[TOP ? 4 : 1][kTopMost];
    __shared__ LpCollect s_c;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int r = (int)blockIdx.x / a.parts, part = (int)blockIdx.x % a.parts;
    const LpRow<T> row(a, r);
    const int token = a.tokens ? __builtin_amdgcn_readfirstlane(a.tokens[r]) : -1;
    const bool given = token >= 0 && token < a.V;
    const float mine = given ? to_f32(row.row[token]) : INFINITY;
    const int begin = part * a.part_sets + wave, end = min((row.vecs + kSet - 1) / kSet, (part + 1) * a.part_sets);
    const int sets = begin < end ? (end - begin + 3) / 4 : 0, each = (sets + kLpSlots - 1) / kLpSlots;       // this wave's: begin, begin + 4, ...; of a group

    LpRun run;
    run.init();
    int above = 0, of_group = 0, slot = 0;
    float best = -INFINITY;
    auto take = [&](const Vec8<T> (&s)[kSetVecs]) {
        float f[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kSetVecs; ++i) {
            s[i].unpack(f);
            top = fmaxf(top, fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7]))));
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
    Vec8<T> A[kSetVecs], B[kSetVecs];
    int set = begin;
    if (set < end) row.load(A, set, lane);
    while (set < end) {
        const int next = set + 4;
        if (next < end) row.load(B, next, lane);
        take(A);
        if (next >= end) break;
        set = next + 4;
        if (set < end) row.load(A, set, lane);
        take(B);
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
    int place = 64, top_t = kNoIndex;                          // wave 0: this lane's token and its place among the most likely, once they are known
    float top_v = -INFINITY;
    if constexpr (TOP) {
        float *lanes = &s_lv[0][0];                            // (64 of its 128 places at a time: the waves' lanes' largest, joined by the first)
        static_assert(4 * kTopMost >= 64, "");
        if (threadIdx.x == 0) s_c.count = 0;
        if (threadIdx.x < 64) lanes[lane] = lane_best;
        __syncthreads();
        for (int w = 1; w < 4; ++w) {
            if (wave == w) lanes[lane] = fmaxf(lanes[lane], lane_best);
            __syncthreads();
        }
        const float bound = lp_kth<sizeof(T) == 2>(lanes[lane], a.top);
        // this wave's groups that reach the bound
        int n = 0;
        for (int i = 0; i < slot; ++i) {
            const float b = s_best[wave][i][lane];
            const uint64_t hit = __ballot(b >= bound && b > -INFINITY);
            if (!hit) continue;
            const int at = n + __popcll(hit & ((1ull << lane) - 1));
            if ((hit >> lane & 1) && at < 64) s_group[wave][at] = i * 64 + lane;
            n += __popcll(hit);
        }
        if (n > 64 && lane == 0) atomicAdd(&s_c.count, 1 << 20);
        if (n <= 64 && n > 0) {
            const int id = lane < n ? s_group[wave][lane] : 0;
            for (int j = 0; j < each; ++j) {
                const int at = (id >> 6) * each + j;           // the wave's set
                Vec8<T> s[kSetVecs];
#pragma unroll
                for (int i = 0; i < kSetVecs; ++i) {
                    s[i].zero();
                    if (lane < n && at < sets) row.load_one(s[i], (begin + 4 * at) * kSet + i * 64 + (id & 63));
                }
#pragma unroll
                for (int i = 0; i < kSetVecs; ++i) {
                    float f[8];
                    s[i].unpack(f);
                    const float top = fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
                    const bool in = lane < n && at < sets;
                    if (!__any(in && top >= bound)) continue;
                    const int first = ((begin + 4 * at) * kSet + i * 64 + (id & 63)) * 8 - row.shift;
#pragma unroll
                    for (int e = 0; e < 8; ++e) lp_collect(s_c, f[e], first + e, in && f[e] >= bound && f[e] > -INFINITY, lane);
                }
            }
        }
        __syncthreads();
        if (s_c.count > 64) {                                  // this wave's sets once more, with a sorted list
            for (int at = begin; at < end; at += 4) {
                row.load(A, at, lane);
#pragma unroll
                for (int i = 0; i < kSetVecs; ++i) {
                    float f[8];
                    A[i].unpack(f);
                    const float top = fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
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
    auto join_waves = [&] {                                    // by wave 0
        run.m = s_m[0]; run.Z = s_Z[0]; run.S = s_S[0]; run.above = s_above[0];
        for (int w = 1; w < 4; ++w) { LpRun o; o.m = s_m[w]; o.Z = s_Z[w]; o.S = s_S[w]; o.above = s_above[w]; run.add(o); }
        if constexpr (TOP) {
            if (s_c.count <= 64) { place = lp_place(s_c, s_c.count, lane, top_v, top_t); return; }
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
        if (wave == 0) {
            join_waves();
            if (lane == 0) {
                LpPartial *p = a.stats + at;
                st_coherent(&p->m, run.m); st_coherent(&p->Z, run.Z); st_coherent(&p->S, run.S); st_coherent(&p->above, run.above);
            }
            if constexpr (TOP) {
                const int have = __popcll(__ballot(place < a.top));
                if (place < a.top) { st_coherent(a.list_value + at * a.top + place, top_v); st_coherent(a.list_token + at * a.top + place, top_t); }
                if (lane >= have && lane < a.top) { st_coherent(a.list_value + at * a.top + lane, -INFINITY); st_coherent(a.list_token + at * a.top + lane, kNoIndex); }
            }
            wait_stores();
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
        run.init();
        for (int p = lane; p < a.parts; p += 64) {
            const LpPartial *q = a.stats + first + p;
            LpRun o;
            o.m = ld_coherent(&q->m); o.Z = ld_coherent(&q->Z); o.S = ld_coherent(&q->S); o.above = ld_coherent(&q->above);
            run.add(o);
        }
        if constexpr (TOP) {
            const int total = a.parts * a.top;
            const float *values = a.list_value + first * a.top;
            const int *tokens = a.list_token + first * a.top;
            float most = -INFINITY;
            for (int i = lane; i < total; i += 64) most = fmaxf(most, ld_coherent(values + i));
            const float bound = lp_kth<sizeof(T) == 2>(most, a.top);
            s_c.count = 0;
            __builtin_amdgcn_wave_barrier();
            for (int i = 0; i < total; i += 64) {
                const bool in = i + lane < total;
                const float v = in ? ld_coherent(values + i + lane) : -INFINITY;
                lp_collect(s_c, v, in ? ld_coherent(tokens + i + lane) : 0, v >= bound && v > -INFINITY, lane);
            }
            __builtin_amdgcn_wave_barrier();
            const int n = s_c.count;
            if (n <= 64) place = lp_place(s_c, n, lane, top_v, top_t);
            else {
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
        join_waves();
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
