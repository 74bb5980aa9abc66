// Attention of many rows per KV head over a paged cache: bf16 products on the matrix cores with K and V in LDS.
#pragma once
#include "paged.hpp"

namespace ead {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

constexpr int kChunkKeys = 64;       // keys of a tile
constexpr int kChunkRows = 128;      // rows of a workgroup, 32 to a wave

// Four waves take 32 rows each of a tile of 128, all of them every tile of 64 keys, which is requested before the one before is worked on and lands in LDS
// meanwhile, though as built a wave waits for it before its first product, whose operand Q the compiler loaded (a bf16 cache: straight from memory, 1 KB a request; an 8-bit cache: its codes, which each
// wave turns into bf16 for the quarter of the keys that it asked for; in registers meanwhile, they cost 50 spilled ones).
//   S^T = K Q^T with 32x32x16 products: lane (n, h) = (lane & 31, lane >> 5) gets row n's scores for keys 8 i + 4 h + 0..3, i = 0..3, of a block
//   of 32: its statistics are its own up to one exchange of the wave's halves, and the scores of 16 keys, rounded to bf16, are the
//   operand that O^T = V^T P^T wants if V's keys are taken in the same order.  V^T's operand comes from LDS by transposing reads.
//
//  Probabilities enter the second product as bf16: in two terms (TWO), or in one away from the masks' edges where the caller asks for that.  One term of each is off
//  by up to 2^-8 of it, which beside the rounding of the output makes the result's error against 64 bits 0.0022 to 0.0023 of its norm instead of 0.0017,
//  over 600 keys as over 16000; a second term (what the first leaves, rounded) takes that away for half as many products again (2048 rows of
//  32 heads over up to 4096, 9000 and 16000 bf16 keys: 129, 356 and 538 us with one term, 172, 461 and 708 with two; 8-bit keys 152, 395, 631 and 181, 492, 765).
template <typename CT, int HD, bool TWO>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(PagedAttn c) {
    constexpr bool F8 = sizeof(CT) == 1;
    constexpr int kRowBytes = HD * 2, kHalf = kChunkKeys * kRowBytes, kBuf = 2 * kHalf;    // K, then V
    constexpr int KS = HD / 16, CB = HD / 32;
    constexpr int kReq = F8 ? HD / 64 : HD / 32;                         // requests of 1 KB per wave, tile and operand (8-bit HD 32: one for both)
    constexpr int EB = HD / 4 < 16 ? HD / 4 : 16, NL = HD / 4 / EB;      // 8-bit: bytes of a load, loads per lane, tile and operand
    static_assert(paged_many_splits(HD) * kChunkRows * 8 <= kBuf, "the table of the join lies there too");
    // an 8-bit cache: one tile as bf16, and per wave two tiles' codes and exponents as they came
    constexpr int kCodes = 2 * 16 * HD, kRaw = kCodes + 256, kRawRequests = (HD == 32 ? 1 : 2 * kReq) + 1;
    __shared__ __align__(1024) char lds[F8 ? kBuf + 8 * kRaw : 2 * kBuf];
    __shared__ int last_one;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int h = (int)blockIdx.x % c.a.n_kv, rest = (int)blockIdx.x / c.a.n_kv;
    const int split = rest % c.splits, tile = c.row_tiles - 1 - rest / c.splits;
    const PagedSeq s = paged_seq(c.a, blockIdx.y);
    if (s.n_rows * c.group <= c.few_rows) return;                        // k_paged_attn's
    const PagedTile t = paged_tile<kChunkKeys>(c, s, tile, kChunkRows);
    if (t.rows == 0) return;
    const int per = max(c.split_tiles, (t.tiles + c.splits - 1) / c.splits), used = max(1, (t.tiles + per - 1) / per);
    if (split >= used) return;
    const int begin = split * per, count = min(begin + per, t.tiles) - begin;

    // this wave's rows, and this lane's
    const int w0 = t.r0 + 32 * wave, w_rows = min(max(t.r0 + t.rows - w0, 0), 32);
    const int p_lo = s.first + w0 / c.group, p_hi = s.first + (w0 + max(w_rows, 1) - 1) / c.group;
    const int my_tok = (w0 + n) / c.group, my_head = h * c.group + (w0 + n) % c.group, my_pos = s.first + my_tok;
    bf16x8_t q[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        u32x4_t x = {0u, 0u, 0u, 0u};
        if (n < w_rows) {
            const bf16_t *p = (const bf16_t *)c.q.p + (size_t)(s.row0 + my_tok) * c.q.row_stride + (size_t)my_head * c.q.head_stride + 16 * i + 8 * hh;
            if (c.q.vec) x = *(gptr<u32x4_t>)p;
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (uint32_t)p[2 * e].u | (uint32_t)p[2 * e + 1].u << 16;
        }
        q[i] = __builtin_bit_cast(bf16x8_t, x);
    }
    f32x16_t o[CB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    // where this lane reads: K's piece 2 i + hh of key n at k_at ^ 32 i; V's four elements 32 i + .. of keys 4 hh + (lane & 15) / 4 (+ 8) at v_at[..] ^ 64 i
    // (rows of LDS start at multiples of their size, so that the permuted piece is an exclusive or away)
    const uint32_t base = lds_address(lds);
    const uint32_t k_at = base + n * kRowBytes + ((hh ^ lds_swizzle<kRowBytes>(n)) << 4);
    uint32_t v_at[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int key = 8 * e + 4 * hh + ((lane & 15) >> 2), piece = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        v_at[e] = base + kHalf + key * kRowBytes + ((piece ^ lds_swizzle<kRowBytes>(key)) << 4) + (lane & 1) * 8;
    }

    // ---- staging.  Wave w brings keys 16 w .. 16 w + 15 of every tile.  The pages of 16 tiles are looked up at a time (lane 4 i + g: tile i, keys 16 g).
    const int page_mask = (1 << c.a.page_shift) - 1;
    auto key_base = [&](int i) { const int v = begin + i; return (v < t.n_sink ? v : v - t.n_sink + t.t_lo) * kChunkKeys; };
    auto look_up = [&](int i0) {
        const int i = i0 + (lane >> 2);
        if (i >= count) return -1;
        const int pos = key_base(i) + 16 * (lane & 3);
        return pos < s.kv ? paged_page(c.a, s, pos) : -1;
    };
    int pages = look_up(0), pages_next = count > 16 ? look_up(16) : -1;
    uint64_t held = __ballot(pages >= 0);
    uint32_t from[F8 ? 1 : kReq];
#pragma unroll
    for (int i = 0; i < (F8 ? 1 : kReq); ++i) {
        const int at = i * 1024 + lane * 16, r = at / kRowBytes, piece = at % kRowBytes >> 4;
        from[i] = F8 ? lane * 16 : r * kRowBytes + ((piece ^ lds_swizzle<kRowBytes>(r)) << 4);
    }
    const uint32_t raw = base + kBuf + wave * 2 * kRaw;                  // 8-bit: this wave's codes
    auto request = [&](int i) {                  // bit g of the answer: keys 16 g of the tile have a page
        if ((i & 15) == 0 && i) {
            pages = pages_next;
            held = __ballot(pages >= 0);
            pages_next = i + 16 < count ? look_up(i + 16) : -1;
        }
        const int page = max(__builtin_amdgcn_readlane(pages, 4 * (i & 15) + wave), 0), pos = key_base(i) + 16 * wave;
        const size_t vec = scalar(paged_vec(c.a, page, h, pos & page_mask));
        if constexpr (F8) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(raw + (i & 1) * kRaw);
            const char *k = (const char *)c.a.k + vec * HD, *v = (const char *)c.a.v + vec * HD;
            if constexpr (HD == 32) request_pieces((lane < 32 ? k : v) + (lane & 31) * 16, to);
            else
#pragma unroll
                for (int e = 0; e < kReq; ++e) {
                    request_tile((const bf16_t *)(k + e * 1024), from[0], to + e * 1024);
                    request_tile((const bf16_t *)(v + e * 1024), from[0], to + 16 * HD + e * 1024);
                }
            request_words((lane & 4 ? c.a.vs : c.a.ks) + vec + 4 * (lane & 3), to + kCodes);
        } else {
            const uint32_t to = __builtin_amdgcn_readfirstlane(base + (i & 1) * kBuf + wave * 16 * kRowBytes);
#pragma unroll
            for (int e = 0; e < kReq; ++e) request_tile((const bf16_t *)c.a.k + vec * HD, from[e], to + e * 1024);
#pragma unroll
            for (int e = 0; e < kReq; ++e) request_tile((const bf16_t *)c.a.v + vec * HD, from[e], to + kHalf + e * 1024);
        }
        return (int)(held >> (4 * (i & 15))) & 15;
    };
    auto place = [&](int i) {                    // 8-bit: this wave's keys of a tile that is here to the tile of bf16
        if constexpr (F8) {
            const uint32_t codes = raw + (i & 1) * kRaw;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                for (int e = 0; e < NL; ++e) {
                    const int at = (e * 64 + lane) * EB, r = at / HD, piece = at % HD >> 3;
                    uint32_t w[4];
                    if constexpr (EB == 8) { const u32x2_t x = lds_read<u32x2_t>(codes + kv * 16 * HD + at); w[0] = x.x; w[1] = x.y; }
                    else { const u32x4_t x = lds_read<u32x4_t>(codes + kv * 16 * HD + at); w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; }
                    const float f = exp2_of((int)lds_read<uint8_t>(codes + kCodes + 16 * kv + r));
                    const uint32_t row = base + kv * kHalf + (wave * 16 + r) * kRowBytes;
#pragma unroll
                    for (int x = 0; x < EB / 8; ++x)
                        *(__attribute__((address_space(3))) u32x4_t *)(uintptr_t)(row + (((piece + x) ^ lds_swizzle<kRowBytes>(r)) << 4)) =
                            u32x4_t{fp8_bf16x2<false>(w[2 * x], f), fp8_bf16x2<true>(w[2 * x], f), fp8_bf16x2<false>(w[2 * x + 1], f), fp8_bf16x2<true>(w[2 * x + 1], f)};
                }
        }
    };

    auto work = [&](int i, int valid, auto edge_c) {
        constexpr bool EDGE = decltype(edge_c)::value;
        const uint32_t buf = F8 ? 0 : (i & 1) * kBuf;
        const int key0 = key_base(i);
        f32x16_t sc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
#pragma unroll
            for (int e = 0; e < KS; ++e) {
                const bf16x8_t k = *(__attribute__((address_space(3))) bf16x8_t *)(uintptr_t)(((k_at + buf) ^ (32 * e)) + b * 32 * kRowBytes);
                sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[e], sc[b], 0, 0, 0);
            }
        }
        if constexpr (EDGE) {
            int pos = my_pos, from_key = 4 * hh;
            asm volatile("" : "+v"(pos), "+v"(from_key));        // computed here, not kept in registers beside every tile's work (191 -> 168 us)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = key0 + from_key + 32 * b + 8 * (e >> 2) + (e & 3);
                    sc[b][e] = (valid >> (2 * b + (e >> 3)) & 1) && paged_sees(c, pos, key) ? sc[b][e] : -INFINITY;
                }
        }
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[b][e]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * c.c2;
        if (__any(top > m + 8.f)) {
            const float to = top > m + 8.f ? top : m, f = top > m + 8.f ? __builtin_amdgcn_exp2f(m - to) : 1.f;
            m = to;
            l *= f;
#pragma unroll
            for (int x = 0; x < CB; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[x][e] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        using tr_t = __attribute__((address_space(3))) bf16x4_t;
        union Operand { bf16x4_t v[2]; u32x4_t w; };
        auto read_v = [&](int j, int x, Operand &a) {        // V^T's operand: dimensions 32 x .., the tile's keys 16 j ..
            a.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((tr_t *)(uintptr_t)(((v_at[0] + buf) ^ (64 * x)) + j * 16 * kRowBytes));
            a.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((tr_t *)(uintptr_t)(((v_at[1] + buf) ^ (64 * x)) + j * 16 * kRowBytes));
        };
        auto multiply = [&](int x, const Operand &a, const uint32_t *p) {
            o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a.w), __builtin_bit_cast(bf16x8_t, u32x4_t{p[0], p[1], p[2], p[3]}), o[x], 0, 0, 0);
        };
        bool odd = false;
        if constexpr (TWO || EDGE) {
            uint32_t p[2][8], p_lo[2][8];            // the probabilities' two bf16 terms
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][2 * e], c.c2, -ref)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][2 * e + 1], c.c2, -ref));
                    l += x + y;
                    p[b][e] = upper_bf16(x, y);
                    p_lo[b][e] = rest_bf16(x, y);
                }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < CB; ++x) {
                    Operand a;
                    read_v(j, x, a);
                    if constexpr (EDGE) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool b0 = (a.w[e] & 0x7F80u) == 0x7F80u, b1 = (a.w[e] & 0x7F800000u) == 0x7F800000u;
                            odd |= b0 || b1;
                            a.w[e] &= (b0 ? 0xFFFF0000u : 0xFFFFFFFFu) & (b1 ? 0xFFFFu : 0xFFFFFFFFu);
                        }
                    }
                    multiply(x, a, p[j >> 1] + 4 * (j & 1));
                    multiply(x, a, p_lo[j >> 1] + 4 * (j & 1));
                }
        } else {
            // With one term there are registers to read V's operands of 16 keys while those of the 16 before are multiplied, and to take the second
            // block's exponentials beside the first one's products (4096 rows over 12289 .. 16384 keys 1045 -> 1020 us; with two terms 168 -> 179 us
            // for 17 sequences over 8-bit pages: there the compiler's own order stands).
            uint32_t p[2][8];
            auto terms = [&](int b) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][2 * e], c.c2, -ref)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][2 * e + 1], c.c2, -ref));
                    l += x + y;
                    p[b][e] = pack_bf16(x, y);
                }
            };
            Operand a[2][CB];
            auto read_all = [&](int j) {
#pragma unroll
                for (int x = 0; x < CB; ++x) read_v(j, x, a[j & 1][x]);
            };
            auto multiply_all = [&](int j) {
#pragma unroll
                for (int x = 0; x < CB; ++x) multiply(x, a[j & 1][x], p[j >> 1] + 4 * (j & 1));
            };
            read_all(0);
            terms(0);
            read_all(1);
            __builtin_amdgcn_sched_barrier(0);
            multiply_all(0);
            terms(1);
            __builtin_amdgcn_sched_barrier(0);
            read_all(2);
            multiply_all(1);
            __builtin_amdgcn_sched_barrier(0);
            read_all(3);
            multiply_all(2);
            __builtin_amdgcn_sched_barrier(0);
            multiply_all(3);
        }
        if constexpr (EDGE) {
            if (__any(odd)) {
                // infinities and NaN, left out of the product, go to the rows that see them (PagedWave::add_odd)
                int from_dim = 4 * hh;
                asm volatile("" : "+v"(from_dim));
                for (int k = 0; k < kChunkKeys; ++k) {
                    const int key = key0 + k;
                    if (!(valid >> (k >> 4) & 1) || key > p_hi) continue;
                    const size_t vec = paged_vec(c.a, paged_page(c.a, s, key), h, key & page_mask);
                    const bool sees = n < w_rows && paged_sees(c, my_pos, key);
#pragma unroll
                    for (int x = 0; x < CB; ++x)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const size_t at = vec * HD + 32 * x + 8 * (e >> 2) + from_dim + (e & 3);
                            float v;
                            if constexpr (F8) v = (((const uint8_t *)c.a.v)[at] & 0x7F) == 0x7F ? __builtin_nanf("") : 0.f;
                            else v = to_f32(((const CT *)c.a.v)[at]);
                            o[x][e] += sees && !(__builtin_fabsf(v) <= 3.402823466e38f) ? v : 0.f;
                        }
                }
            }
        }
    };

    int valid = 0, valid_next = 0;
    if (count > 0) valid = request(0);
    if constexpr (F8) { if (count > 1) valid_next = request(1); }
    for (int i = 0; i < count; ++i) {
        int valid_then = 0;
        if constexpr (F8) {
            // this wave's codes are here, and every wave is done with the tile before; then every wave has placed its keys
            if (i + 1 < count) wait_requests<kRawRequests>();
            else wait_requests<0>();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            place(i);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (i + 2 < count) valid_then = request(i + 2);
            asm volatile("s_barrier" ::: "memory");
        } else {
            // tile i has landed for every wave, and every wave is done with the buffer of tile i - 1
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (i + 1 < count) valid_next = request(i + 1);
        }
        const int key0 = key_base(i), last = key0 + kChunkKeys - 1;
        const bool skip = w_rows == 0 || key0 > p_hi || (c.window && key0 >= c.sinks && p_lo - last >= c.window);
        if (!skip) {
            const bool whole = valid == 15 && last <= p_lo && (!c.window || p_hi - key0 < c.window || last < c.sinks);
            if (whole) work(i, valid, std::false_type{});
            else work(i, valid, std::true_type{});
        }
        valid = valid_next;
        valid_next = valid_then;
    }
    __syncthreads();

    // ---- the row's sum, and what goes out
    const auto sums = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sums[0]) + __uint_as_float(sums[1]);
    if (l != l && m == -INFINITY) m = 0.f;
    const size_t unit = ((size_t)blockIdx.y * c.a.n_kv + h) * c.row_tiles + tile;
    if (used == 1) {
        if (n >= w_rows) return;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16_t *p = (bf16_t *)c.out.p + (size_t)(s.row0 + my_tok) * c.out.row_stride + (size_t)my_head * c.out.head_stride;
#pragma unroll
        for (int x = 0; x < CB; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 32 * x + 8 * e + 4 * hh;
                const uint2 w = make_uint2(l == 0.f ? 0u : pack_bf16(o[x][4 * e] * inv, o[x][4 * e + 1] * inv), l == 0.f ? 0u : pack_bf16(o[x][4 * e + 2] * inv, o[x][4 * e + 3] * inv));
                if (c.out.vec) *(uint2 *)(p + d) = w;
                else {
                    p[d].u = (uint16_t)w.x; p[d + 1].u = (uint16_t)(w.x >> 16);
                    p[d + 2].u = (uint16_t)w.y; p[d + 3].u = (uint16_t)(w.y >> 16);
                }
            }
        if (c.lse && hh == 0) c.lse[(size_t)(s.row0 + my_tok) * c.n_heads + my_head] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
        return;
    }
    // a part's vectors in the order [wave][x][e][lane]: neighbouring lanes write neighbouring bytes
    const size_t slot = unit * c.splits + split;
    if (n < w_rows) {
        float *p = c.part_o + (slot * kChunkRows * HD / 4 + (size_t)wave * CB * 256 + lane) * 4;
#pragma unroll
        for (int x = 0; x < CB; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) st_coherent4(p + (x * 4 + e) * 256, f32x4e_t{o[x][4 * e], o[x][4 * e + 1], o[x][4 * e + 2], o[x][4 * e + 3]});
        if (hh == 0) {
            float *pm = (float *)(c.part_ml + slot * kChunkRows + 32 * wave + n);
            st_coherent(pm, m);
            st_coherent(pm + 1, l);
        }
    }
    if (!paged_last<false>(c, unit, used, &last_one)) return;
    paged_join<bf16_t, HD, 16, false>(c, s, t, h, used, kChunkRows, kChunkRows * (HD / 4), (float2 *)lds, [&](int i) { return unit * c.splits + i; },
                               [](int e) { return PagedWhere{e / (CB * 256) * 32 + (e & 31), e / 256 % CB * 32 + e / 64 % 4 * 8 + (e & 32) / 8}; });
}

}  // namespace ead
