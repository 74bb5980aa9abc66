// How much of the rows' attention every cached position gets, added to what it had: the weights that a cache is cut by.
#pragma once
#include "paged.hpp"

namespace ead {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

struct PagedWeigh {
    PagedArgs a;
    RowsArg q;
    const float *lse;               // [row][query head]
    float *weights;                 // [page][KV head][slot]
    int n_heads, group;             // group: query heads per KV head
    float c2;                       // scale * log2(e)
    int window, sinks;
    int tiles;                      // k_weigh_few: tiles of 32 keys to a wave, 32 at most (their pages lie in its lanes)
    int splits, part_keys;          // k_weigh_many: ranges of rows; keys of a range's sums
    float *part;                    // [range][sequence][KV head][key]
};
__device__ __forceinline__ bool weigh_sees(const PagedWeigh &c, int pos, int key) {
    return key <= pos && (!c.window || pos - key < c.window || key < c.sinks);
}

// Whether any row sees a key.  What a window has passed is not written at all: its weight stays as it is, and its page may be another sequence's by now, with an owner of its own
__device__ __forceinline__ bool weigh_seen(const PagedWeigh &c, const PagedSeq &s, int key) {
    return !c.window || key < c.sinks || max(s.first, 0) - key < c.window;
}

// A workgroup takes 16 keys, its waves every fourth block of 16 rows (a row: a token and a head of the group): S = Q K^T with the rows as the M of the product and the keys as its N, so
// that lane (n, g) = (lane & 15, lane >> 4) gets key n's scores of rows 4 g .. 4 g + 3 and adds their exponentials up by itself; the four g, and then the waves in their order, are added at the end.
// Every position has one owner: no atomics, and the sums' order is fixed.  Serves what the two kernels below do not: many rows of float32 models, and many whose queries do
// not start on 16-byte boundaries.  Latency: every block's queries are waited for (three float prompts of 500, 8 heads of 32: 18 us; 40 with a wave to 16 keys and all rows).
template <typename CT, int HD>
__global__ __launch_bounds__(256) void k_weigh(PagedWeigh c) {
    constexpr bool F32 = sizeof(CT) == 4;
    constexpr int KE = F32 ? 4 : 8, KL = HD / 4 / KE;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4, h = (int)blockIdx.y;
    __shared__ float sums[4][16];
    const PagedSeq s = paged_seq(c.a, blockIdx.z);
    const int rows = s.n_rows * c.group;
    if (rows == 0) return;
    const int step = (int)gridDim.x * 16;
    for (int base = (int)blockIdx.x * 16; base < s.kv; base = s.kv - base > step ? base + step : s.kv) {       // (a sum past 2^31 would start over)
        const int page = __builtin_amdgcn_readfirstlane(paged_page(c.a, s, base));
        if (page < 0) continue;
        const int key = base + n;
        const size_t vec = paged_vec(c.a, page, h, key & ((1 << c.a.page_shift) - 1));
        uint32_t k[KL][4];
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            const int d = (4 * i + g) * KE;
            if constexpr (sizeof(CT) == 1) {
                const u32x2_t w = *(gptr<u32x2_t>)((const uint8_t *)c.a.k + vec * HD + d);
                const float f = exp2_of(c.a.ks[vec]);
                k[i][0] = fp8_bf16x2<false>(w.x, f); k[i][1] = fp8_bf16x2<true>(w.x, f);
                k[i][2] = fp8_bf16x2<false>(w.y, f); k[i][3] = fp8_bf16x2<true>(w.y, f);
            } else {
                Raw<16> x; x.load((const CT *)c.a.k + vec * HD + d);
                for (int e = 0; e < 4; ++e) k[i][e] = x.w[e];
            }
        }
        float sum = 0.f;
        for (int r0 = wave * 16; r0 < rows; r0 += 64) {
            // rows before the first that reaches these keys see none of them, and with a window neither do those past its end
            const int p_hi = s.first + min(r0 + 15, rows - 1) / c.group, p_lo = s.first + r0 / c.group;
            if (p_hi < base || (c.window && p_lo - (base + 15) >= c.window && base >= c.sinks)) continue;
            const int r = r0 + n, tok = r / c.group, qh = h * c.group + r % c.group;
            const size_t at = (size_t)(s.row0 + tok) * c.q.row_stride + (size_t)qh * c.q.head_stride;
            f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const int d = (4 * i + g) * KE;
                u32x4_t q = {0u, 0u, 0u, 0u};
                if (r < rows) {
                    if constexpr (F32) {
                        const float *p = (const float *)c.q.p + at + d;
                        if (c.q.vec) q = *(gptr<u32x4_t>)p;
                        else for (int e = 0; e < 4; ++e) q[e] = __float_as_uint(p[e]);
                    } else {
                        const bf16_t *p = (const bf16_t *)c.q.p + at + d;
                        if (c.q.vec) q = *(gptr<u32x4_t>)p;
                        else for (int e = 0; e < 4; ++e) q[e] = (uint32_t)p[2 * e].u | (uint32_t)p[2 * e + 1].u << 16;
                    }
                }
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[e]), __uint_as_float(k[i][e]), sc, 0, 0, 0);
                } else {
                    sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q), __builtin_bit_cast(bf16x8_t, u32x4_t{k[i][0], k[i][1], k[i][2], k[i][3]}), sc, 0, 0, 0);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int rr = r0 + 4 * g + e, t = rr / c.group;
                if (rr < rows && weigh_sees(c, s.first + t, key)) {
                    const float z = c.lse[(size_t)(s.row0 + t) * c.n_heads + h * c.group + rr % c.group];
                    if (z != -INFINITY) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], c.c2, -1.4426950408889634f * z));
                }
            }
        }
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        if (g == 0) sums[wave][n] = sum;
        __syncthreads();
        if (wave == 0 && g == 0 && key < s.kv && weigh_seen(c, s, key)) {
            float *w = c.weights + vec;
            *w = (key < s.first ? *w : 0.f) + (((sums[0][n] + sums[1][n]) + sums[2][n]) + sums[3][n]);
        }
        __syncthreads();
    }
}

// The same for sequences whose rows fit NB blocks of 16 (decode steps, catch-ups): bound by the reading of K, so K comes as whole lines, through a ring of tiles of 32 keys in
// LDS that is the wave's own (no barrier), with the exponents and with the weights as they were; the rows' queries stay in registers.  No joins: a position's weight is one wave's.
// All tiles of a sequence are gone through, with a window too.  Few instructions a tile and four workgroups to a compute unit are what it takes to keep requests on their way: 64
// sequences of 1024 to 16384 8-bit keys, 40 query heads, 113 us (5.35 TB/s; 141 with two workgroups and rings of 16 KB, 267 with loads in the products' operand layout and no ring); one sequence of 8191 bf16 keys, 32 heads, 5.5 us.
template <typename CT, int HD, int NB>
struct WeighWave {
    static constexpr bool F32 = sizeof(CT) == 4, F8 = sizeof(CT) == 1;
    static constexpr int kRow = HD * (int)sizeof(CT), kKeys = 32 * kRow;      // bytes of a key, of a tile's keys
    static constexpr int kReq = 16 * kRow / 1024 > 0 ? 16 * kRow / 1024 : 1;  // requests for 16 keys (8-bit HD 32: for 32)
    static constexpr bool kShort = 16 * kRow < 1024;
    static constexpr int kTile = kKeys + 256 + (F8 ? 256 : 0), kRequests = (kShort ? 1 : 2 * kReq) + 1 + (F8 ? 1 : 0);
    static constexpr int kRing = kKeys >= 4096 ? 2 : 8192 / kKeys;             // tiles
    static constexpr int KE = F32 ? 4 : F8 ? (HD >= 64 ? 16 : 8) : 8;         // neighbouring elements of K in one read
    static constexpr int KL = HD / 4 / KE;                                    // reads per key
    static constexpr int QW = F32 ? HD / 4 : HD / 8;                          // words of Q per lane
    static constexpr int kBlocks = 4 * kRing * kTile <= 40960 && NB < 4 ? 4 : 2;   // workgroups to a compute unit
};
// 4 bytes per lane from base + voff (base the same in all lanes) to LDS at lds + 4 lane
__device__ __forceinline__ void request_words_from(const void *base, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory");
}

template <typename CT, int HD, int NB>
__global__ __launch_bounds__(256, (WeighWave<CT, HD, NB>::kBlocks)) void k_weigh_few(PagedWeigh c) {
    using W = WeighWave<CT, HD, NB>;
    constexpr int kRow = W::kRow;
    __shared__ __align__(1024) char lds[4 * W::kRing * W::kTile];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4, h = (int)blockIdx.x % c.a.n_kv;
    const PagedSeq s = paged_seq(c.a, blockIdx.y);
    const int rows = min(s.n_rows * c.group, NB * 16);
    const int key0 = ((int)blockIdx.x / c.a.n_kv * c.tiles * 4 + wave) * 32;       // this wave's tiles: every fourth from here
    const int count = min((s.kv - key0 + 127) / 128, c.tiles);
    if (rows <= 0 || count <= 0) return;
    const int page_mask = (1 << c.a.page_shift) - 1;
    int pages = -1;                                          // lane 2 i + half: keys 16 half .. of tile i
    {
        const int pos = key0 + (lane >> 1) * 128 + (lane & 1) * 16;
        if ((lane >> 1) < count && pos < s.kv) pages = paged_page(c.a, s, pos);
    }
    // element KE (4 i + g) + .. of a row's queries belongs to K's read i: the contraction's order is free as long as both have the same
    uint32_t q[NB][W::QW];
    float nl[NB][4];                                         // -lse in bits of this lane's rows, far below anything where one pays nothing or there is none
    const int p_lo = s.first, p_hi = s.first + (rows - 1) / c.group;
    bool odd = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int i = 0; i < W::QW; ++i) q[b][i] = 0u;
        // (past the last row: that one again, which adds nothing that it does not)
        const int r = min(b * 16 + n, rows - 1), tok = r / c.group, qh = h * c.group + r % c.group;
        {
            const size_t at = (size_t)(s.row0 + tok) * c.q.row_stride + (size_t)qh * c.q.head_stride;
#pragma unroll
            for (int i = 0; i < W::KL; ++i) {
                const int d = (4 * i + g) * W::KE;
                if constexpr (W::F32) {
                    const float *p = (const float *)c.q.p + at + d;
                    if (c.q.vec) { Raw<16> x; x.load(p); for (int e = 0; e < 4; ++e) q[b][i * 4 + e] = x.w[e]; }
                    else for (int e = 0; e < 4; ++e) q[b][i * 4 + e] = __float_as_uint(p[e]);
                } else {
                    const bf16_t *p = (const bf16_t *)c.q.p + at + d;
                    if (c.q.vec) { Raw<W::KE * 2> x; x.load(p); for (int e = 0; e < W::KE / 2; ++e) q[b][i * (W::KE / 2) + e] = x.w[e]; }
                    else for (int e = 0; e < W::KE / 2; ++e) q[b][i * (W::KE / 2) + e] = (uint32_t)p[2 * e].u | (uint32_t)p[2 * e + 1].u << 16;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int rr = b * 16 + 4 * g + e;
            float z = -INFINITY;
            if (rr < rows) z = c.lse[(size_t)(s.row0 + rr / c.group) * c.n_heads + h * c.group + rr % c.group];
            odd |= rr < rows && z == -INFINITY;
            nl[b][e] = z == -INFINITY ? -1e30f : -1.4426950408889634f * z;
        }
    }
    odd = __any(odd);
    uint32_t from[W::kReq], k_at[W::KL];
#pragma unroll
    for (int e = 0; e < W::kReq; ++e) {                      // where this lane's piece of a request lies among 16 keys
        const int at = e * 1024 + lane * 16, key = at / kRow, piece = at % kRow >> 4;
        from[e] = (W::kShort ? key & 15 : key) * kRow + ((piece ^ lds_swizzle<kRow>(key)) << 4);
    }
    const uint32_t ring = lds_address(lds) + wave * W::kRing * W::kTile;
#pragma unroll
    for (int i = 0; i < W::KL; ++i) {
        const int byte = (4 * i + g) * W::KE * (int)sizeof(CT);
        k_at[i] = n * kRow + (((byte >> 4) ^ lds_swizzle<kRow>(n)) << 4) + (byte & 15);
    }
    // Requests a tile.  Every address is inside the pools: halves without a page read page 0, and nothing is kept of them
    auto request = [&](int i) {
        const int base = key0 + i * 128;
        const int page0 = max(__builtin_amdgcn_readlane(pages, 2 * i), 0), page1 = max(__builtin_amdgcn_readlane(pages, 2 * i + 1), 0);
        const size_t vec0 = scalar(paged_vec(c.a, page0, h, base & page_mask)), vec1 = scalar(paged_vec(c.a, page1, h, (base + 16) & page_mask));
        const uint32_t to = __builtin_amdgcn_readfirstlane(ring + i % W::kRing * W::kTile);
        if constexpr (W::kShort) {
            request_pieces((const char *)c.a.k + (lane < 32 ? vec0 : vec1) * kRow + from[0], to);
        } else {
#pragma unroll
            for (int e = 0; e < W::kReq; ++e) request_tile<true>((const bf16_t *)((const char *)c.a.k + vec0 * kRow), from[e], to + e * 1024);
#pragma unroll
            for (int e = 0; e < W::kReq; ++e) request_tile<true>((const bf16_t *)((const char *)c.a.k + vec1 * kRow), from[e], to + (W::kReq + e) * 1024);
        }
        // weights, in lanes 0 .. 31, and exponents, four to a word, in lanes 0 .. 7; the others repeat them
        if (vec1 == vec0 + 16) {
            request_words_from(c.weights + vec0, 4 * (lane & 31), to + W::kKeys);
            if constexpr (W::F8) request_words_from(c.a.ks + vec0, 4 * (lane & 7), to + W::kKeys + 256);
        } else {
            request_words(c.weights + (lane & 16 ? vec1 : vec0) + n, to + W::kKeys);
            if constexpr (W::F8) request_words(c.a.ks + (lane & 4 ? vec1 : vec0) + 4 * (lane & 3), to + W::kKeys + 256);
        }
    };
    auto take = [&](int i, auto edge_c) {
        constexpr bool EDGE = decltype(edge_c)::value;
        const int base = key0 + i * 128;
        const uint32_t at = ring + i % W::kRing * W::kTile;
        float sum[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t keys = at + half * 16 * kRow;
            f32x4_t sc[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) sc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            float f = 0.f;
            if constexpr (W::F8) f = exp2_of((int)lds_read<uint8_t>(at + W::kKeys + 256 + half * 16 + n));
#pragma unroll
            for (int j = 0; j < W::KL; ++j) {
                if constexpr (W::F32) {
                    const f32x4e_t k = lds_read<f32x4e_t>(keys + k_at[j]);
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[b][j * 4 + e]), k[e], sc[b], 0, 0, 0);
                } else {
                    uint32_t w[W::KE / 2];
                    if constexpr (!W::F8) { const u32x4_t x = lds_read<u32x4_t>(keys + k_at[j]); w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; }
                    else if constexpr (W::KE == 16) {
                        const u32x4_t x = lds_read<u32x4_t>(keys + k_at[j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) { w[2 * e] = fp8_bf16x2<false>(x[e], f); w[2 * e + 1] = fp8_bf16x2<true>(x[e], f); }
                    } else {
                        const u32x2_t x = lds_read<u32x2_t>(keys + k_at[j]);
                        w[0] = fp8_bf16x2<false>(x.x, f); w[1] = fp8_bf16x2<true>(x.x, f); w[2] = fp8_bf16x2<false>(x.y, f); w[3] = fp8_bf16x2<true>(x.y, f);
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int x = 0; x < W::KE / 8; ++x) {
                            const uint32_t *p = q[b] + j * (W::KE / 2) + 4 * x;
                            sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, u32x4_t{p[0], p[1], p[2], p[3]}),
                                                                            __builtin_bit_cast(bf16x8_t, u32x4_t{w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]}), sc[b], 0, 0, 0);
                        }
                }
            }
            float t = 0.f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int rr = b * 16 + 4 * g + e;
                    float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][e], c.c2, nl[b][e]));
                    if constexpr (EDGE) x = rr < rows && nl[b][e] != -1e30f && weigh_sees(c, s.first + rr / c.group, base + 16 * half + n) ? x : 0.f;
                    t += x;
                }
            sum[half] = t;
        }
        // both halves' four sums a key at once: the first half's come to lanes 0 .. 15 and 16 .. 31, the second's to the others
        const auto over = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[0]), __float_as_uint(sum[1]), false, false);
        const uint32_t two = __float_as_uint(__uint_as_float(over[0]) + __uint_as_float(over[1]));
        const auto row = __builtin_amdgcn_permlane16_swap(two, two, false, false);
        const float paid = __uint_as_float(row[0]) + __uint_as_float(row[1]);
        const int key = base + 16 * (lane >> 5) + n, page = __builtin_amdgcn_readlane(pages, 2 * i), page_too = __builtin_amdgcn_readlane(pages, 2 * i + 1);
        const int mine = lane & 32 ? page_too : page;
        const float old = lds_read<float>(at + W::kKeys + 64 * (lane >> 5) + 4 * n);
        if (!(lane & 16) && mine >= 0 && key < s.kv && (!EDGE || weigh_seen(c, s, key))) c.weights[paged_vec(c.a, mine, h, key & page_mask)] = (key < s.first ? old : 0.f) + paid;
    };
#pragma unroll
    for (int i = 0; i < W::kRing - 1; ++i)
        if (i < count) request(i);
    for (int i = 0; i < count; ++i) {
        if (i + W::kRing - 1 < count) {
            request(i + W::kRing - 1);
            wait_requests<(W::kRing - 1) * W::kRequests>();
        } else wait_requests<0>();
        const int base = key0 + i * 128, last = base + 31;
        if (last <= p_lo && !odd && (!c.window || p_hi - base < c.window || last < c.sinks)) take(i, std::false_type{});
        else take(i, std::true_type{});
    }
}

// Many rows (prompts and pieces of them): bound by products and exponentials, so the keys stay in registers, 64 to a wave and 256 to a workgroup, and the rows come
// through LDS, 32 at a time, requested one tile ahead and read by all four waves.
//   S = Q K^T with 32x32x16 products: lane (n, hh) = (lane & 31, lane >> 5) gets key n's scores of rows 8 i + 4 hh + 0..3 of a tile, i = 0..3, and adds their
//   exponentials up; the halves of the wave are added at the end.
// The rows that see a tile of keys are cut into c.splits ranges; with more than one each leaves its sums for k_weigh_join.
// 2048 rows after 6145 positions, 32 heads of 128: 168 us with the join's 5 (725 Tflop/s).  By the counters a SIMD is busy for 41 cycles with the 64 scores of a wave's instruction: 16 of
// them products, and 4.3 vector instructions besides (an fma, an exponential, an addition, the rest addresses, statistics and tile ends), 21 cycles at 4 each and 8 for the exponential
// (measured alone: 8.2 an exponential, 2.5 an fma with two waves and more).  16 and 21 are nine tenths of 41: the two hardly overlap; matrix cores are busy for 38 %, vector issue, the
// products' own included, for 55 %.
// The next tile's products between this one's exponentials (registers for two waves to a SIMD instead of three) took 213 us, all of a tile's queries read before its products as
// long as this.  Keys are loaded whether or not any row of the range sees them, and a sequence of few rows beside a long piece goes through here range by range.
template <typename CT, int HD>
__global__ __launch_bounds__(256, 2) void k_weigh_many(PagedWeigh c) {
    constexpr int KS = HD / 16, kRowBytes = HD * 2, kTileBytes = 32 * kRowBytes, kReq = kTileBytes / 4096;     // requests of 1 KB to a wave (HD 32: half a one)
    __shared__ __align__(1024) char lds[2 * kTileBytes];
    __shared__ __align__(16) float nls[2][32];               // -lse in bits, -inf where a row pays nothing
    __shared__ int odd[2];                                   // whether there is such a row
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int h = (int)blockIdx.x % c.a.n_kv, rest = (int)blockIdx.x / c.a.n_kv, split = rest % c.splits, key0 = rest / c.splits * 256, my0 = key0 + wave * 64;
    const PagedSeq s = paged_seq(c.a, blockIdx.y);
    const int rows = s.n_rows * c.group;
    if (rows == 0 || key0 >= s.kv) return;
    // tiles of rows that see any of the workgroup's keys, and this range's of them
    const int last_key = min(key0 + 255, s.kv - 1);
    int t0 = max(key0 - s.first, 0) * c.group / 32, t1 = (rows + 31) / 32;
    if (c.window && key0 >= c.sinks) t1 = (int)min((long)t1, max(((long)last_key + c.window - s.first) * c.group + 31, 0l) / 32);
    const int per = max((t1 - t0 + c.splits - 1) / c.splits, 0);
    t0 += split * per;
    t1 = min(t1, t0 + per);
    const int page_mask = (1 << c.a.page_shift) - 1;
    size_t vec[2];
    bool live[2];
    bf16x8_t k[2][KS];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int key = my0 + 32 * b + n, page = key < s.kv ? paged_page(c.a, s, key) : -1;
        live[b] = page >= 0;
        vec[b] = paged_vec(c.a, max(page, 0), h, key & page_mask);
        const float f = sizeof(CT) == 1 ? exp2_of(c.a.ks[vec[b]]) : 0.f;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const int d = 16 * i + 8 * hh;
            if constexpr (sizeof(CT) == 1) {
                const u32x2_t w = *(gptr<u32x2_t>)((const uint8_t *)c.a.k + vec[b] * HD + d);
                k[b][i] = __builtin_bit_cast(bf16x8_t, u32x4_t{fp8_bf16x2<false>(w.x, f), fp8_bf16x2<true>(w.x, f), fp8_bf16x2<false>(w.y, f), fp8_bf16x2<true>(w.y, f)});
            } else k[b][i] = __builtin_bit_cast(bf16x8_t, *(gptr<u32x4_t>)((const bf16_t *)c.a.k + vec[b] * HD + d));
        }
    }
    // ---- staging: a request is 16 bytes to a lane, whose address goes on by 32 rows a tile without a product
    const uint32_t base = lds_address(lds);
    constexpr int kPieces = kReq > 0 ? kReq : 1;
    const bool asks = kReq > 0 || wave < 2;
    int rem[kPieces], row_of[kPieces];
    const bf16_t *from[kPieces];
    const int step_tok = 32 / c.group, step_rem = 32 % c.group;
    const long step = step_tok * c.q.row_stride + step_rem * c.q.head_stride, wrap = c.q.row_stride - c.group * c.q.head_stride;
    const bf16_t *first_row = (const bf16_t *)c.q.p + (size_t)s.row0 * c.q.row_stride + (size_t)(h * c.group) * c.q.head_stride;
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
        const int at = (kReq > 0 ? wave * kReq + e : wave & 1) * 1024 + lane * 16;
        row_of[e] = at / kRowBytes;
        const int r = t0 * 32 + row_of[e], tok = r / c.group;
        rem[e] = r % c.group;
        from[e] = first_row + tok * c.q.row_stride + rem[e] * c.q.head_stride + ((at % kRowBytes >> 4) ^ lds_swizzle<kRowBytes>(row_of[e])) * 8;
    }
    int z_row = t0 * 32 + lane, z_tok = z_row / c.group, z_rem = z_row % c.group;          // wave 0, lanes 0 .. 31: the tile's lse
    auto request = [&](int t) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(base + (t & 1) * kTileBytes + (kReq > 0 ? wave * kReq : wave & 1) * 1024);
        if (!asks) return;
#pragma unroll
        for (int e = 0; e < kPieces; ++e) {
            if (t * 32 + 32 <= rows) request_pieces(from[e], to + e * 1024);
            else request_pieces(t * 32 + row_of[e] < rows ? from[e] : first_row, to + e * 1024);       // past the last row: a row whose scores are left out
            from[e] += step;
            if (step_rem) {
                rem[e] += step_rem;
                from[e] += rem[e] >= c.group ? wrap : 0;
                rem[e] -= rem[e] >= c.group ? c.group : 0;
            }
        }
    };
    auto next_lse = [&] {
        float z = -INFINITY;
        if (wave) return z;
        if (lane < 32 && z_row < rows) z = c.lse[(size_t)(s.row0 + z_tok) * c.n_heads + h * c.group + z_rem];
        z_row += 32;
        z_tok += step_tok;
        z_rem += step_rem;
        if (z_rem >= c.group) { z_rem -= c.group; ++z_tok; }
        return z;
    };
    auto put_lse = [&](int t, float z) {
        if (wave) return;
        const uint64_t none = __ballot(lane < 32 && z == -INFINITY);
        if (lane < 32) nls[t & 1][lane] = z == -INFINITY ? -INFINITY : -1.4426950408889634f * z;
        if (lane == 0) odd[t & 1] = none != 0;
    };
    const uint32_t q_at = base + n * kRowBytes + ((hh ^ lds_swizzle<kRowBytes>(n)) << 4);
    float sum[2] = {0.f, 0.f};
    int p_tok = t0 * 32 / c.group, p_rem = t0 * 32 % c.group;                              // the tile's first row
    auto take = [&](int t, auto edge_c) {
        constexpr bool EDGE = decltype(edge_c)::value;
        f32x16_t sc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const bf16x8_t q = *(__attribute__((address_space(3))) bf16x8_t *)(uintptr_t)((q_at ^ (32 * i)) + (t & 1) * kTileBytes);
            sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k[0][i], sc[0], 0, 0, 0);
            sc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k[1][i], sc[1], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4e_t nl = *(const f32x4e_t *)&nls[t & 1][8 * i + 4 * hh];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                int pos = 0;
                bool pays = true;
                if constexpr (EDGE) {
                    const int r = t * 32 + 8 * i + 4 * hh + e;
                    pos = s.first + r / c.group;
                    pays = r < rows && nl[e] != -INFINITY;
                }
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][4 * i + e], c.c2, nl[e]));
                    if constexpr (EDGE) x = pays && weigh_sees(c, pos, my0 + 32 * b + n) ? x : 0.f;
                    sum[b] += x;
                }
            }
        }
    };
    if (t0 < t1) {
        const float first = next_lse();
        request(t0);
        put_lse(t0, first);
        for (int t = t0; t < t1; ++t) {
            wait_requests<0>();
            __syncthreads();
            float coming = 0.f;
            if (t + 1 < t1) {
                coming = next_lse();
                request(t + 1);
            }
            const int p_lo = s.first + p_tok;
            p_tok += step_tok;
            p_rem += step_rem;
            if (p_rem >= c.group) { p_rem -= c.group; ++p_tok; }
            const int p_next = s.first + p_tok;              // no row of this tile is past the next one's first
            if (p_next >= my0) {
                if (my0 + 63 <= p_lo && !odd[t & 1] && (!c.window || p_next - my0 < c.window || my0 + 63 < c.sinks)) take(t, std::false_type{});
                else take(t, std::true_type{});
            }
            if (t + 1 < t1) put_lse(t + 1, coming);
        }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        sum[b] += __shfl_xor(sum[b], 32, kWave);
        const int key = my0 + 32 * b + n;
        if (hh == 0 && live[b]) {
            if (c.splits > 1) c.part[(((size_t)split * gridDim.y + blockIdx.y) * c.a.n_kv + h) * c.part_keys + key] = sum[b];
            else if (weigh_seen(c, s, key)) c.weights[vec[b]] = (key < s.first ? c.weights[vec[b]] : 0.f) + sum[b];
        }
    }
}

// The ranges' sums of a position, in their order, on top of what it had
__global__ __launch_bounds__(256) void k_weigh_join(PagedWeigh c) {
    const int h = (int)blockIdx.y, key = (int)blockIdx.x * 256 + (int)threadIdx.x;
    const PagedSeq s = paged_seq(c.a, blockIdx.z);
    if (s.n_rows == 0 || key >= min(s.kv, c.part_keys)) return;
    const int page = paged_page(c.a, s, key);
    if (page < 0 || !weigh_seen(c, s, key)) return;
    float *w = c.weights + paged_vec(c.a, page, h, key & ((1 << c.a.page_shift) - 1));
    float sum = key < s.first ? *w : 0.f;
    const size_t apart = (size_t)gridDim.z * c.a.n_kv * c.part_keys;
    const float *p = c.part + ((size_t)blockIdx.z * c.a.n_kv + h) * c.part_keys + key;
    for (int i = 0; i < c.splits; ++i) sum += p[i * apart];
    *w = sum;
}

}  // namespace ead
