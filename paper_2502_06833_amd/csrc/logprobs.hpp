// Log probabilities of given tokens and of the most likely ones, ranks and entropies, from logits in memory.
#pragma once
#include <type_traits>

#include "common.hpp"

namespace ead {

constexpr int kTopMost = 32;                  // alternatives of a row at most
constexpr int kSetVecs = 4;                   // vectors of 8 logits that a lane holds of a set
constexpr int kSet = 64 * kSetVecs;           // vectors of a set: what a wave takes at a time
constexpr int kLpTicketInts = 32;             // a row's ticket has a cache line of its own

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
        for (int i = 0; i < kSetVecs; ++i) {
            const int v = v0 + i * 64 + lane;
            if (v >= whole0 && v < whole1) { s[i].load_stream(base + (size_t)v * 8); continue; }
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = v * 8 + e - shift;
                f[e] = j >= 0 && j < V ? to_f32(row[j]) : -INFINITY;
            }
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i].raw[e] = __float_as_uint(f[2 * e]) >> 16 | (__float_as_uint(f[2 * e + 1]) & 0xFFFF0000u);
            } else {
                s[i].lo = f32x4e_t{f[0], f[1], f[2], f[3]};
                s[i].hi = f32x4e_t{f[4], f[5], f[6], f[7]};
            }
        }
    }
};

template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprobs(LogprobArgs a) {
    __shared__ float s_m[4], s_Z[4], s_S[4], s_lv[4][kTopMost];
    __shared__ int s_above[4], s_lt[4][kTopMost], s_last;
    __shared__ __align__(16) Vec8<T> s_vec[4][64];
    __shared__ int s_at[4][64];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int r = (int)blockIdx.x / a.parts, part = (int)blockIdx.x % a.parts;
    const LpRow<T> row(a, r);
    const int token = a.tokens ? __builtin_amdgcn_readfirstlane(a.tokens[r]) : -1;
    const bool given = token >= 0 && token < a.V;
    const float mine = given ? to_f32(row.row[token]) : INFINITY;
    const int end = min((row.vecs + kSet - 1) / kSet, (part + 1) * a.part_sets);

    LpRun run;
    run.init();
    LpList list;
    list.init();
    int above = 0;
    auto take = [&](const Vec8<T> (&s)[kSetVecs], int set) {
        float top[kSetVecs], f[8], m = run.m;
#pragma unroll
        for (int i = 0; i < kSetVecs; ++i) {
            s[i].unpack(f);
            top[i] = fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
            m = fmaxf(m, top[i]);
        }
        run.move(m);
        const float ref = lp_ref(m), off = -(ref * kLpLog2e);
        const bool large = __any(lp_large(m));
#pragma unroll
        for (int i = 0; i < kSetVecs; ++i) {
            s[i].unpack(f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = large ? lp_bits(f[e], m) : __builtin_fmaf(f[e], kLpLog2e, off);
                const float x = __builtin_amdgcn_exp2f(d);         // NaN stays one, in Z; -inf is 0, and adds 0 * -200 to S
                run.Z += x;
                run.S = __builtin_fmaf(x, fmaxf(d, -200.f), run.S);
                above += __popcll(__ballot(f[e] > mine));
            }
        }
        if constexpr (TOP) {
            const float best = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            float kth = list.last(a.top), least = -INFINITY;
            const uint64_t lanes = __ballot(best > kth);
            if (!lanes) return;
            if (__popcll(lanes) > a.top) {
                // of so many lanes' largest the k-th largest is a bound for the set's own k-th
                const uint32_t key = lp_rank(best);
                uint32_t t = 0;
                for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 0); --bit)
                    if (__popcll(__ballot(key >= (t | 1u << bit))) >= a.top) t |= 1u << bit;
                least = lp_value(t);
            }
#pragma unroll
            for (int i = 0; i < kSetVecs; ++i) {
                const bool has = top[i] > kth && top[i] >= least;
                const uint64_t hit = __ballot(has);
                if (!hit) continue;
                if (has) {
                    const int at = __popcll(hit & ((1ull << lane) - 1));
                    s_vec[wave][at] = s[i];
                    s_at[wave][at] = (set * kSet + i * 64 + lane) * 8 - row.shift;
                }
                __builtin_amdgcn_wave_barrier();               // LDS serves a wave's accesses in order: what its lanes wrote is there for all of them
                const int n = __popcll(hit);
                for (int j = 0; j < n; j += 8) {
                    const int at = j + (lane >> 3);
                    const bool is = at < n;
                    float g[8];
                    s_vec[wave][is ? at : 0].unpack(g);
                    float v = g[0];
#pragma unroll
                    for (int e = 1; e < 8; ++e) v = (lane & 7) == e ? g[e] : v;
                    list.offer(v, s_at[wave][is ? at : 0] + (lane & 7), is && v > -INFINITY && v >= least, a.top, lane);
                }
                __builtin_amdgcn_wave_barrier();
                kth = list.last(a.top);
            }
        }
    };
    Vec8<T> A[kSetVecs], B[kSetVecs];
    int set = part * a.part_sets + wave;
    if (set < end) row.load(A, set, lane);
    while (set < end) {
        const int next = set + 4;
        if (next < end) row.load(B, next, lane);
        take(A, set);
        if (next >= end) break;
        set = next + 4;
        if (set < end) row.load(A, set, lane);
        take(B, next);
    }

    // ---- the workgroup's: waves in order, lanes in the order of the exchange
    const float wm = wave_max(run.m);
    run.move(wm);
    run.Z = wave_sum(run.Z);
    run.S = wave_sum(run.S);
    if (lane == 0) { s_m[wave] = wm; s_Z[wave] = run.Z; s_S[wave] = run.S; s_above[wave] = above; }
    if (TOP && lane < kTopMost) { s_lv[wave][lane] = list.v; s_lt[wave][lane] = list.t; }
    __syncthreads();
    auto join_waves = [&] {                                    // by wave 0
        run.m = s_m[0]; run.Z = s_Z[0]; run.S = s_S[0]; run.above = s_above[0];
        for (int w = 1; w < 4; ++w) { LpRun o; o.m = s_m[w]; o.Z = s_Z[w]; o.S = s_S[w]; o.above = s_above[w]; run.add(o); }
        if (TOP) {
            list.v = lane < kTopMost ? s_lv[0][lane] : -INFINITY;
            list.t = lane < kTopMost ? s_lt[0][lane] : kNoIndex;
            for (int w = 1; w < 4; ++w) {
                const bool is = lane < a.top;
                list.offer(is ? s_lv[w][lane] : 0.f, is ? s_lt[w][lane] : 0, is, a.top, lane);
            }
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
            if (TOP && lane < a.top) { st_coherent(a.list_value + at * a.top + lane, list.v); st_coherent(a.list_token + at * a.top + lane, list.t); }
            wait_stores();
            if (lane == 0) {
                int *ticket = a.tickets + (size_t)r * kLpTicketInts;
                const bool last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts - 1;
                if (last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = last;
            }
        }
        __syncthreads();
        if (!s_last) return;
        // the last to arrive joins the parts in their order, whoever it is
        const size_t first = (size_t)r * a.parts;
        run.init();
        for (int p = wave * 64 + lane; p < a.parts; p += 256) {
            const LpPartial *q = a.stats + first + p;
            LpRun o;
            o.m = ld_coherent(&q->m); o.Z = ld_coherent(&q->Z); o.S = ld_coherent(&q->S); o.above = ld_coherent(&q->above);
            run.add(o);
        }
        const float pm = wave_max(run.m);
        run.move(pm);
        run.Z = wave_sum(run.Z);
        run.S = wave_sum(run.S);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) run.above += __shfl_xor(run.above, o, kWave);
        if (TOP) {
            list.init();
            const int total = a.parts * a.top;
            for (int i = wave * 64; i < total; i += 256) {
                const bool is = i + lane < total;
                const float v = is ? ld_coherent(a.list_value + first * a.top + i + lane) : 0.f;
                const int t = is ? ld_coherent(a.list_token + first * a.top + i + lane) : 0;
                list.offer(v, t, is, a.top, lane);
            }
        }
        __syncthreads();
        if (lane == 0) { s_m[wave] = pm; s_Z[wave] = run.Z; s_S[wave] = run.S; s_above[wave] = run.above; }
        if (TOP && lane < kTopMost) { s_lv[wave][lane] = list.v; s_lt[wave][lane] = list.t; }
        __syncthreads();
    }
    if (wave) return;
    join_waves();
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
    if (TOP) {
        // rows with fewer logits above -inf than were asked for: the lowest other tokens
        const int have = __popcll(__ballot(lane < a.top && list.t != kNoIndex));
        int t = 0;
        for (int i = have; i < a.top; ++i) {
            while (__any(lane < a.top && list.t == t)) ++t;
            if (lane == i) list.t = t;
        }
        if (lane < a.top) {
            a.top_tokens[(size_t)r * a.top + lane] = list.t;
            const float lp = (list.v - run.m) - lnz;
            a.top_logprobs[(size_t)r * a.top + lane] = lp > 0.f ? 0.f : lp;
        }
    }
}

}  // namespace ead
