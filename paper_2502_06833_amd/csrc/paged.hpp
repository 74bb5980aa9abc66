// A paged K/V cache in the caller's memory: rows written to it (rounded to its type), read back from it, and
// attention of rows over it.
//
// Pages are [page][KV head][slot][head_dim]: what one head holds of a page is contiguous, so a wave that takes 16 keys
// of a head reads (or writes) 16 * head_dim elements in a row, whatever the page size.
#pragma once
#include <type_traits>

#include "common.hpp"
#include "paged_rules.hpp"

namespace ead {

struct fp8_t { uint8_t u; };      // an e4m3 code
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

struct PagedArgs {
    const void *k, *v;
    const uint8_t *ks, *vs;                       // exponents of an 8-bit cache
    int n_pages, page_shift, n_kv;
    const int *table, *q_starts, *kv_lens;
    int table_stride, table_width, rows;
};

// A sequence as the device arrays have it, cut to what the host vouched for: row0 + n_rows <= rows, 0 <= kv <= table.  Rows keep the positions that the
// uncut length gives them: where a table ends before its sequence, what lies past it are holes.
struct PagedSeq {
    int row0, n_rows, kv, first;                  // kv: positions that the table reaches; first: position of its first row (below 0 where it has more rows than positions)
    const int *table;
};
__device__ __forceinline__ PagedSeq paged_seq_of(const PagedArgs &a, int start, int end, int len, const int *table) {
    PagedSeq s;
    s.row0 = min(max(start, 0), a.rows);
    s.n_rows = min(max(end, s.row0), a.rows) - s.row0;
    s.kv = min(max(len, 0), (int)min((long)a.table_width << a.page_shift, (long)0x7FFFFF00));
    s.first = max(len, 0) - s.n_rows;
    s.table = table;
    return s;
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs &a, int b) {
    // (b is the workgroup's: the readfirstlanes say so, which keeps what follows from these in scalar registers)
    return paged_seq_of(a, __builtin_amdgcn_readfirstlane(a.q_starts[b]), __builtin_amdgcn_readfirstlane(a.q_starts[b + 1]), __builtin_amdgcn_readfirstlane(a.kv_lens[b]),
                        a.table + (size_t)b * a.table_stride);
}
// the same for a number that differs from lane to lane
__device__ __forceinline__ PagedSeq paged_seq_lane(const PagedArgs &a, int b) { return paged_seq_of(a, a.q_starts[b], a.q_starts[b + 1], a.kv_lens[b], nullptr); }
// The page of a position 0 <= pos < kv; -1: a hole
__device__ __forceinline__ int paged_page(const PagedArgs &a, const PagedSeq &s, int pos) {
    const int id = s.table[pos >> a.page_shift];
    return (unsigned)id < (unsigned)a.n_pages ? id : -1;
}
// Vector (page, head, slot)'s number in the pool: 64 bits, since a pool may hold more than 2^31 elements
__device__ __forceinline__ size_t paged_vec(const PagedArgs &a, int page, int h, int slot) {
    return (((size_t)page * a.n_kv + h) << a.page_shift) + slot;
}

// ---- 8 bits: e4m3 codes times a power of two per vector --------------------------------------
// e4m3 reaches from 2^-9 to 448 with three fraction bits; a power-of-two scale moves that range over the vector and
// costs no fraction bit, so the scale is a byte and codes times scale are exact in bf16 (8 fraction bits).
__device__ __forceinline__ int fp8_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);     // 448 = 1.75 * 2^8
    return min(max(e, 1), 254);
}
__device__ __forceinline__ float exp2_of(int biased) { return __uint_as_float((uint32_t)biased << 23); }
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// two codes of a word (its low or high half) times a power of two, as a pair of bf16
template <bool HIGH>
__device__ __forceinline__ uint32_t fp8_bf16x2(uint32_t w, float scale) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}

// ---- write and read ----------------------------------------------------------------------------
struct RowsArg {
    const void *p;
    long row_stride, head_stride;
    int vec;                        // every vector starts on a 16-byte boundary
};

template <bool STREAM, typename T>
__device__ __forceinline__ void load8(const T *p, int vec, float (&f)[8]) {
    if (vec) {
        Vec8<T> x;
        if constexpr (STREAM) x.load_stream(p);
        else x.load(p);
        x.unpack(f);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = to_f32(p[e]);
    }
}
// eight floats as bf16, NaN kept (the conversion instruction)
__device__ __forceinline__ u32x4_t bf16x8_of(const float (&f)[8]) {
    return u32x4_t{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}

template <bool STREAM, typename V> __device__ __forceinline__ void put(V *p, V v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool STREAM> __device__ __forceinline__ void put8f(float *p, const float (&f)[8]) {
    put<STREAM>((f32x4e_t *)p, f32x4e_t{f[0], f[1], f[2], f[3]});
    put<STREAM>((f32x4e_t *)p + 1, f32x4e_t{f[4], f[5], f[6], f[7]});
}

// One vector's eight elements of this lane to the cache.  The HD / 8 lanes that share a vector call it together.
template <typename CT, int HD, bool STREAM>
__device__ __forceinline__ void put8(void *pool, uint8_t *scales, size_t vec, int lane, float (&f)[8], bool live) {
    if constexpr (sizeof(CT) == 1) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = __builtin_fabsf(f[e]);
            m = a <= 3.402823466e38f ? fmaxf(m, a) : m;
        }
#pragma unroll
        for (int o = HD / 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
        const int ex = fp8_exponent(m);
        const float inv = exp2_of(254 - ex);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __builtin_fabsf(f[e]) <= 3.402823466e38f ? f[e] * inv : __builtin_nanf("");
        if (live) {
            put<STREAM>((u32x2_t *)((uint8_t *)pool + vec * HD + lane * 8), u32x2_t{fp8_pack4(f[0], f[1], f[2], f[3]), fp8_pack4(f[4], f[5], f[6], f[7])});
            if (lane == 0) scales[vec] = (uint8_t)ex;
        }
    } else if constexpr (sizeof(CT) == 2) {
        if (live) put<STREAM>((u32x4_t *)((bf16_t *)pool + vec * HD + lane * 8), bf16x8_of(f));
    } else {
        if (live) put8f<STREAM>((float *)pool + vec * HD + lane * 8, f);
    }
}

// The rows' vectors are taken in the order [token][head], the HD / 8 lanes of a vector side by side; blocks of 2 to 64 tokens of a head at a time, which write
// runs of slots, took as long, and so did four vectors to a lane.  Bound by memory.  STREAM: non-temporal accesses, for calls that move more than the
// second-level caches hold: 27000 rows of 8 heads to 8 bits 44 -> 40 us (4.4 TB/s), 55000 rows back as bf16 74 -> 67 us (5.6 TB/s; a large copy runs at 4.9).
struct PagedCopy {
    PagedArgs a;
    RowsArg k, v;
};

template <typename CT, typename RT, int HD, bool STREAM>
__global__ __launch_bounds__(256) void k_paged_write(PagedCopy c) {
    constexpr int L = HD / 8, kVecs = 256 / L;
    const PagedSeq s = paged_seq(c.a, blockIdx.y);
    const int total = s.n_rows * c.a.n_kv;
    const int lane = (int)threadIdx.x % L;
    for (int i = (int)blockIdx.x * kVecs + (int)threadIdx.x / L; i < total; i += (int)gridDim.x * kVecs) {
        const int t = i / c.a.n_kv, h = i % c.a.n_kv, pos = s.first + t;
        bool live = pos >= 0 && pos < s.kv;
        float fk[8] = {}, fv[8] = {};
        size_t vec = 0;
        if (live) {
            const size_t row = (size_t)(s.row0 + t);
            load8<STREAM>((const RT *)c.k.p + row * c.k.row_stride + h * c.k.head_stride + lane * 8, c.k.vec, fk);
            load8<STREAM>((const RT *)c.v.p + row * c.v.row_stride + h * c.v.head_stride + lane * 8, c.v.vec, fv);
            const int page = paged_page(c.a, s, pos);
            live = page >= 0;
            vec = paged_vec(c.a, max(page, 0), h, pos & ((1 << c.a.page_shift) - 1));
        }
        put8<CT, HD, STREAM>((void *)c.a.k, (uint8_t *)c.a.ks, vec, lane, fk, live);
        put8<CT, HD, STREAM>((void *)c.a.v, (uint8_t *)c.a.vs, vec, lane, fv, live);
    }
}

template <typename CT, int HD, bool STREAM>
__device__ __forceinline__ void get8(const void *pool, const uint8_t *scales, size_t vec, int lane, float (&f)[8]) {
    if constexpr (sizeof(CT) == 1) {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        const u32x2_t *p = (const u32x2_t *)((const uint8_t *)pool + vec * HD + lane * 8);
        const u32x2_t w = STREAM ? __builtin_nontemporal_load(p) : *p;
        const float scale = exp2_of(scales[vec]);
        const f32x2_t p0 = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, false), p1 = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, true);
        const f32x2_t p2 = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, false), p3 = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, true);
        f[0] = p0.x * scale; f[1] = p0.y * scale; f[2] = p1.x * scale; f[3] = p1.y * scale;
        f[4] = p2.x * scale; f[5] = p2.y * scale; f[6] = p3.x * scale; f[7] = p3.y * scale;
    } else {
        load8<STREAM>((const CT *)pool + vec * HD + lane * 8, 1, f);
    }
}
template <bool STREAM, typename RT>
__device__ __forceinline__ void set8(RT *p, int vec, const float (&f)[8]) {
    if (vec) {
        if constexpr (sizeof(RT) == 2) put<STREAM>((u32x4_t *)p, bf16x8_of(f));
        else put8f<STREAM>(p, f);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (sizeof(RT) == 2) p[e].u = (uint16_t)pack_bf16(f[e], 0.f);
        else p[e] = f[e];
    }
}

template <typename CT, typename RT, int HD, bool STREAM>
__global__ __launch_bounds__(256) void k_paged_read(PagedCopy c) {
    constexpr int L = HD / 8, kVecs = 256 / L;
    const PagedSeq s = paged_seq(c.a, blockIdx.y);
    const int total = s.n_rows * c.a.n_kv;
    const int lane = (int)threadIdx.x % L;
    for (int i = (int)blockIdx.x * kVecs + (int)threadIdx.x / L; i < total; i += (int)gridDim.x * kVecs) {
        const int t = i / c.a.n_kv, h = i % c.a.n_kv, pos = s.first + t;
        const int page = pos >= 0 && pos < s.kv ? paged_page(c.a, s, pos) : -1;
        float fk[8] = {}, fv[8] = {};
        if (page >= 0) {
            const size_t vec = paged_vec(c.a, page, h, pos & ((1 << c.a.page_shift) - 1));
            get8<CT, HD, STREAM>(c.a.k, c.a.ks, vec, lane, fk);
            get8<CT, HD, STREAM>(c.a.v, c.a.vs, vec, lane, fv);
        }
        const size_t row = (size_t)(s.row0 + t);
        set8<STREAM>((RT *)c.k.p + row * c.k.row_stride + h * c.k.head_stride + lane * 8, c.k.vec, fk);
        set8<STREAM>((RT *)c.v.p + row * c.v.row_stride + h * c.v.head_stride + lane * 8, c.v.vec, fv);
    }
}

// ---- attention -----------------------------------------------------------------------------------
struct PagedAttn {
    PagedArgs a;
    RowsArg q, out;
    float *lse;
    int n_heads, group;             // group: query heads per KV head
    float c2;                       // scale * log2(e): scores are kept in units of one bit
    int window, sinks;
    int once;                       // every key is read by one workgroup: requests are non-temporal (request_tile)
    int few_rows;                   // sequences with at most this many rows per KV head are k_paged_attn's, the others k_paged_chunk's
    int row_tiles, splits, split_tiles;   // k_paged_chunk: grid.x = row_tiles * splits * n_kv; at least split_tiles key tiles to a split
    int pairs, shares, min_share;   // k_paged_attn: (sequence, tile of rows) pairs, 0: a workgroup to a unit; grid.x; fewest groups of tiles to a workgroup
    float *part_o;                  // [part][tile row][head_dim], relative to the part's maximum
    float2 *part_ml;                // [part][tile row]: maximum (in bits), sum
    int *tickets;                   // [(sequence, KV head, tile of rows)] in cache lines of their own, zero between launches
};

constexpr int kKeyTile = 32;

// Two bf16 terms of probabilities: the upper halves of their words, and what those leave, rounded (16 bits in all).  The rest gets 2^-22 of the probability on top
// and is never 0 where that is not: times an infinity of V both terms are that infinity, where a rest of 0 or of the other sign would make it NaN.
__device__ __forceinline__ uint32_t upper_bf16(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ uint32_t rest_bf16(float a, float b) {
    auto rest = [](float p) { return __builtin_fmaf(p, 1.f + 0x1p-22f, -__uint_as_float(__float_as_uint(p) & 0xFFFF0000u)); };
    return pack_bf16(rest(a), rest(b));
}

// What a tile of rows sees.  Rows of a KV head are (token, head of the group) pairs, token first: row = token * group + head.
struct PagedTile {
    int r0, rows;                   // first row, rows in the tile (0: none)
    int p_lo, p_hi;                 // positions of its first and last row
    int n_sink, t_lo, tiles;        // key tiles: n_sink ones from position 0, the others from tile t_lo on
};
template <int KEYS>
__device__ __forceinline__ PagedTile paged_tile(const PagedAttn &c, const PagedSeq &s, int tile, int tile_rows) {
    PagedTile t;
    t.r0 = tile * tile_rows;
    t.rows = min(max(s.n_rows * c.group - t.r0, 0), tile_rows);
    t.p_lo = s.first + t.r0 / c.group;
    t.p_hi = s.first + (t.r0 + max(t.rows, 1) - 1) / c.group;
    t.t_lo = c.window ? max(0, max(t.p_lo, 0) - c.window + 1) / KEYS : 0;
    t.n_sink = c.window ? min((min(c.sinks, s.kv) + KEYS - 1) / KEYS, t.t_lo) : 0;
    t.tiles = t.rows > 0 && t.p_hi >= 0 ? t.n_sink + max(min(t.p_hi, s.kv - 1) / KEYS + 1 - t.t_lo, 0) : 0;
    return t;
}
__device__ __forceinline__ bool paged_sees(const PagedAttn &c, int pos, int key) {
    return key <= pos && (!c.window || pos - key < c.window || key < c.sinks);
}

// N bytes (a multiple of 16) of device memory as words
template <int N> struct Raw {
    uint32_t w[N / 4];
    __device__ __forceinline__ void load(const void *p) {
#pragma unroll
        for (int i = 0; i < N / 16; ++i) {
            const u32x4_t x = ((gptr<u32x4_t>)p)[i];
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
    }
};

// ---- LDS by its address ----------------------------------------------------------------------------
using lds_byte = __attribute__((address_space(3))) char;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(lds_byte *)p; }
template <typename T> __device__ __forceinline__ T lds_read(uint32_t at) { return *(__attribute__((address_space(3))) T *)(uintptr_t)at; }
// 4 bytes per lane, each from its own address, to LDS at lds + 4 lane (M0 as in request_tile)
__device__ __forceinline__ void request_words(const void *p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory");
}
// 16 bytes per lane likewise, to lds + 16 lane
__device__ __forceinline__ void request_pieces(const void *p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory");
}
// a value that is the same in every lane, kept in scalar registers
__device__ __forceinline__ size_t scalar(size_t v) {
    return (size_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v) | (size_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
}
template <int N> __device__ __forceinline__ void wait_requests() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Rows of K and V (one key each, ROW bytes) lie one after the other in LDS, their 16-byte pieces permuted by an exclusive or with this
// number of the key: the 16-byte reads of K (one piece of 16 or 32 keys) and the transposing reads of V (4 or 8 keys, a few neighbouring
// pieces each) spread over the banks.  No conflicts in k_paged_chunk over bf16; over 8 bits, whose transposing reads take 8 bytes and whose codes are read and
// written besides, they are 23 % of its LDS cycles and 42 % of k_paged_attn's (10 % of the time LDS is busy there).
template <int ROW> __device__ __forceinline__ int lds_swizzle(int key) {
    if (ROW >= 256) return ((key & 3) << 2) | ((key >> 2) & 3);
    if (ROW == 128) return (((key >> 1) & 1) << 2) | ((key >> 2) & 3);
    if (ROW == 64) return (key >> 2) & 3;
    return (key >> 3) & 1;
}

// One wave's piece of attention: tiles of 32 keys against NB blocks of 16 rows.
//
//  Tiles come to a ring in LDS that is the wave's own, in requests of 1 KB of neighbouring bytes: no barrier, no registers, and whole
//  cache lines (loads in the products' operand layout, 64 bytes of a key at a time, ran at 4.9 TB/s where these reach 6.8).
//  S^T = K Q^T: the keys are the M of the product, rows the N, so lane (n, g) = (lane & 15, lane >> 4) gets the scores of row n
//  for keys 4g .. 4g+3 of each half of the tile: statistics are the lane's own up to two exchanges over g, and the lane
//  already holds what the second product, O^T = V^T P^T, wants of P: its contraction runs over the keys in the order
//  (j < 4 ? 4g + j : 16 + 4g + j - 4), in which V's transposing reads from LDS take them.  Float V needs no transposing: there a lane
//  reads VW neighbouring elements of each of its keys, and product c takes element c of every lane.
template <typename CT, int HD, int NB>
struct PagedWave {
    static constexpr bool F32 = sizeof(CT) == 4, F8 = sizeof(CT) == 1;
    static constexpr int kRow = HD * (int)sizeof(CT);                        // bytes of a key
    static constexpr int kPart = kKeyTile * kRow, kTile = 2 * kPart + (F8 ? 256 : 0);   // K, V, exponents
    static constexpr int kReq = 16 * kRow / 1024 > 0 ? 16 * kRow / 1024 : 1;  // requests for 16 keys of K or V (8-bit HD 32: for 32 keys)
    static constexpr bool kShort = 16 * kRow < 1024;
    static constexpr int kRequests = (kShort ? 2 : 4 * kReq) + (F8 ? 1 : 0);  // for a tile
    static constexpr int kRing = kTile > 16384 + 256 ? 1 : kTile * 2 > 8192 ? 2 : 8192 / kTile;   // tiles
    static constexpr int VW = HD / 16 < 4 ? HD / 16 : 4;                     // float: neighbouring elements of V in one read
    static constexpr int KE = F32 ? 4 : F8 ? (HD >= 64 ? 16 : 8) : 8;        // neighbouring elements of K in one read
    static constexpr int KL = HD / 4 / KE;                                   // reads per key
    static constexpr int kCodeBits = 9;                                      // 8 bits: V's codes are taken times 2^kCodeBits
    static constexpr int QW = F32 ? HD / 4 : HD / 8;                         // words of Q per lane

    uint32_t q[NB][QW];
    f32x4_t o[NB][HD / 16];
    float m[NB], l[NB];             // in bits; l: this lane's keys only
    uint32_t from[kReq], k_at[KL], v_at[F32 ? 1 : HD / 16];

    // element KE (4 i + g) + .. of the row's queries belongs to K's read i: the contraction's order is free as long as both have the same
    __device__ __forceinline__ void init(const PagedAttn &c, const PagedSeq &s, const PagedTile &t, int h, int lane) {
        const int n = lane & 15, g = lane >> 4;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int row = b * 16 + n;
            m[b] = -INFINITY;
            l[b] = 0.f;
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) o[b][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < QW; ++i) q[b][i] = 0u;
            if (row < t.rows) {
                const int r = t.r0 + row, tok = r / c.group, qh = h * c.group + r % c.group;
                const size_t at = (size_t)(s.row0 + tok) * c.q.row_stride + (size_t)qh * c.q.head_stride;
#pragma unroll
                for (int i = 0; i < KL; ++i) {
                    const int d = (4 * i + g) * KE;
                    if constexpr (F32) {
                        const float *p = (const float *)c.q.p + at + d;
                        if (c.q.vec) { Raw<16> x; x.load(p); for (int e = 0; e < 4; ++e) q[b][i * 4 + e] = x.w[e]; }
                        else for (int e = 0; e < 4; ++e) q[b][i * 4 + e] = __float_as_uint(p[e]);
                    } else {
                        const bf16_t *p = (const bf16_t *)c.q.p + at + d;
                        if (c.q.vec) { Raw<KE * 2> x; x.load(p); for (int e = 0; e < KE / 2; ++e) q[b][i * (KE / 2) + e] = x.w[e]; }
                        else for (int e = 0; e < KE / 2; ++e) q[b][i * (KE / 2) + e] = (uint32_t)p[2 * e].u | (uint32_t)p[2 * e + 1].u << 16;
                    }
                }
            }
        }
#pragma unroll
        for (int e = 0; e < kReq; ++e) {                     // where this lane's piece of a request lies among 16 keys
            const int at = e * 1024 + lane * 16, key = at / kRow, piece = at % kRow >> 4;
            from[e] = (kShort ? key & 15 : key) * kRow + ((piece ^ lds_swizzle<kRow>(key)) << 4);
        }
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            const int byte = (4 * i + g) * KE * (int)sizeof(CT);
            k_at[i] = n * kRow + (((byte >> 4) ^ lds_swizzle<kRow>(n)) << 4) + (byte & 15);
        }
        if constexpr (!F32) {
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) {
                const int key = F8 ? key_of(0, n >> 1, g) : 4 * g + (n >> 2), byte = F8 ? 16 * i + 8 * (n & 1) : 32 * i + 8 * (n & 3);
                v_at[i] = kPart + key * kRow + (((byte >> 4) ^ lds_swizzle<kRow>(key)) << 4) + (byte & 15);
            }
        }
    }

    // Requests a tile.  Every address is inside the pool: halves without a page (-1: holes, positions past the end) read page 0 and are masked
    template <bool ONCE>
    __device__ __forceinline__ void request(const PagedAttn &c, int base, int page0, int page1, int h, int lane, uint32_t to) const {
        const int mask = (1 << c.a.page_shift) - 1;
        const size_t vec0 = scalar(paged_vec(c.a, max(page0, 0), h, base & mask)), vec1 = scalar(paged_vec(c.a, max(page1, 0), h, (base + 16) & mask));
        to = __builtin_amdgcn_readfirstlane(to);
        if constexpr (kShort) {
            const size_t at = (lane < 32 ? vec0 : vec1) * kRow + from[0];
            request_pieces((const char *)c.a.k + at, to);
            request_pieces((const char *)c.a.v + at, to + kPart);
        } else {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const char *p = (const char *)(part ? c.a.v : c.a.k);
#pragma unroll
                for (int e = 0; e < kReq; ++e) request_tile<ONCE>((const bf16_t *)(p + vec0 * kRow), from[e], to + part * kPart + e * 1024);
#pragma unroll
                for (int e = 0; e < kReq; ++e) request_tile<ONCE>((const bf16_t *)(p + vec1 * kRow), from[e], to + part * kPart + (kReq + e) * 1024);
            }
        }
        // words 0..7: exponents of K, 8..15: of V (the other lanes repeat them)
        if constexpr (F8) request_words((lane & 8 ? c.a.vs : c.a.ks) + (lane & 4 ? vec1 : vec0) + 4 * (lane & 3), to + 2 * kPart);
    }

    __device__ __forceinline__ static int key_of(int base, int j, int g) { return base + (j < 4 ? 4 * g + j : 12 + 4 * g + j); }

    // Whether every row of the tile sees all of these keys
    __device__ __forceinline__ static bool whole(const PagedAttn &c, const PagedTile &t, int base, int page0, int page1) {
        const int last = base + kKeyTile - 1;
        return page0 >= 0 && page1 >= 0 && last <= t.p_lo && (!c.window || t.p_hi - base < c.window || last < c.sinks);
    }

    template <bool EDGE>
    __device__ __forceinline__ void take(const PagedAttn &c, const PagedSeq &s, const PagedTile &t, int h, int lane, int base, int page0, int page1, uint32_t at) {
        const int n = lane & 15, g = lane >> 4;
        // ---- scores
        f32x4_t sc[NB][2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int b = 0; b < NB; ++b) sc[b][half] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            float ks = 1.f;
            if constexpr (F8) ks = exp2_of((int)lds_read<uint8_t>(at + 2 * kPart + 16 * half + n));
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const uint32_t k_from = at + k_at[i] + half * 16 * kRow;
                if constexpr (F32) {
                    const f32x4_t k = lds_read<f32x4_t>(k_from);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            sc[b][half] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], __uint_as_float(q[b][i * 4 + e]), sc[b][half], 0, 0, 0);
                } else {
                    uint32_t k[4];
                    if constexpr (KE * sizeof(CT) == 8) { const u32x2_t x = lds_read<u32x2_t>(k_from); k[0] = x.x; k[1] = x.y; }
                    else { const u32x4_t x = lds_read<u32x4_t>(k_from); k[0] = x.x; k[1] = x.y; k[2] = x.z; k[3] = x.w; }
#pragma unroll
                    for (int e = 0; e < KE / 8; ++e) {
                        u32x4_t kw;
                        if constexpr (F8) kw = u32x4_t{fp8_bf16x2<false>(k[2 * e], ks), fp8_bf16x2<true>(k[2 * e], ks), fp8_bf16x2<false>(k[2 * e + 1], ks), fp8_bf16x2<true>(k[2 * e + 1], ks)};
                        else kw = u32x4_t{k[0], k[1], k[2], k[3]};
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            const int w = i * (KE / 2) + e * 4;
                            const u32x4_t qw = {q[b][w], q[b][w + 1], q[b][w + 2], q[b][w + 3]};
                            sc[b][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kw), __builtin_bit_cast(bf16x8_t, qw), sc[b][half], 0, 0, 0);
                        }
                    }
                }
            }
        }
        if constexpr (EDGE) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int pos = s.first + (t.r0 + b * 16 + n) / c.group;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool sees = (j < 4 ? page0 : page1) >= 0 && paged_sees(c, pos, key_of(base, j, g));
                    sc[b][j >> 2][j & 3] = sees ? sc[b][j >> 2][j & 3] : -INFINITY;
                }
            }
        }
        // ---- running maximum and sum.  The maximum that the sums refer to follows the true one only when that is more
        // than 8 bits above it: exponentials stay below 2^8, and the output is seldom rescaled.
        float p[NB][8];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float top = fmaxf(fmaxf(fmaxf(sc[b][0][0], sc[b][0][1]), fmaxf(sc[b][0][2], sc[b][0][3])), fmaxf(fmaxf(sc[b][1][0], sc[b][1][1]), fmaxf(sc[b][1][2], sc[b][1][3])));
            const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
            const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(r32[0]), __uint_as_float(r32[1])) * c.c2;
            if (__any(top > m[b] + 8.f)) {           // rows that need none keep theirs: what a row gets is its own affair
                const float to = top > m[b] + 8.f ? top : m[b], f = top > m[b] + 8.f ? __builtin_amdgcn_exp2f(m[b] - to) : 1.f;
                m[b] = to;
                l[b] *= f;
#pragma unroll
                for (int i = 0; i < HD / 16; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[b][i][r] *= f;
            }
            const float ref = m[b] == -INFINITY ? 0.f : m[b];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][j >> 2][j & 3], c.c2, -ref));
            l[b] += ((p[b][0] + p[b][1]) + (p[b][2] + p[b][3])) + ((p[b][4] + p[b][5]) + (p[b][6] + p[b][7]));
        }
        // ---- output.  At an edge, infinities and NaN among the values are left out of the product (0 times what a row does not see
        // has to be 0, whatever lies there) and added to the rows that see them.
        bool odd = false;
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < HD / 16 / VW; ++i) {
                    const int key = key_of(0, j, g), byte = 4 * VW * (16 * i + n);
                    const uint32_t v_from = at + kPart + key * kRow + (((byte >> 4) ^ lds_swizzle<kRow>(key)) << 4) + (byte & 15);
                    uint32_t w[4];
                    if constexpr (VW == 2) { const u32x2_t x = lds_read<u32x2_t>(v_from); w[0] = x.x; w[1] = x.y; }
                    else { const u32x4_t x = lds_read<u32x4_t>(v_from); w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; }
#pragma unroll
                    for (int e = 0; e < VW; ++e) {
                        if constexpr (EDGE) {
                            const bool bad = (w[e] & 0x7F800000u) == 0x7F800000u;
                            odd |= bad;
                            w[e] = bad ? 0u : w[e];
                        }
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            o[b][i * VW + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), p[b][j], o[b][i * VW + e], 0, 0, 0);
                    }
                }
        } else {
            if constexpr (F8) {                      // the values' powers of two go to the probabilities, but for 2^kCodeBits, which the codes take: up to 2^8 times 2^127 overflows
                const uint32_t s0 = lds_read<uint32_t>(at + 2 * kPart + 32 + 4 * g), s1 = lds_read<uint32_t>(at + 2 * kPart + 48 + 4 * g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int e = (int)(((j < 4 ? s0 : s1) >> (8 * (j & 3))) & 0xFFu) - (127 + kCodeBits);
#pragma unroll
                    for (int b = 0; b < NB; ++b) p[b][j] = __builtin_amdgcn_ldexpf(p[b][j], e);
                }
            }
            // two bf16 terms of every probability
            u32x4_t hi[NB], lo[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    hi[b][e] = upper_bf16(p[b][2 * e], p[b][2 * e + 1]);
                    lo[b][e] = rest_bf16(p[b][2 * e], p[b][2 * e + 1]);
                }
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) {
                u32x4_t v;
                if constexpr (F8) {
                    typedef int i32x2_t __attribute__((ext_vector_type(2)));
                    const i32x2_t x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2_t *)(uintptr_t)(at + v_at[i]));
                    constexpr float up = 1 << kCodeBits;
                    v = u32x4_t{fp8_bf16x2<false>((uint32_t)x.x, up), fp8_bf16x2<true>((uint32_t)x.x, up), fp8_bf16x2<false>((uint32_t)x.y, up), fp8_bf16x2<true>((uint32_t)x.y, up)};
                } else {
                    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
                    using tr_t = __attribute__((address_space(3))) bf16x4_t;
                    union { bf16x4_t x[2]; u32x4_t w; } a;
                    a.x[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((tr_t *)(uintptr_t)(at + v_at[i]));
                    a.x[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((tr_t *)(uintptr_t)(at + v_at[i] + 16 * kRow));
                    v = a.w;
                }
                if constexpr (EDGE) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool b0 = (v[e] & 0x7F80u) == 0x7F80u, b1 = (v[e] & 0x7F800000u) == 0x7F800000u;
                        odd |= b0 || b1;
                        v[e] &= (b0 ? 0xFFFF0000u : 0xFFFFFFFFu) & (b1 ? 0xFFFFu : 0xFFFFFFFFu);
                    }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    o[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, hi[b]), o[b][i], 0, 0, 0);
                    o[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, lo[b]), o[b][i], 0, 0, 0);
                }
            }
        }
        if (EDGE && __any(odd)) add_odd(c, s, t, h, lane, base, page0, page1);
    }

    // Output element i (0 .. HD/16-1), r of this lane is dimension dim_of(i, r, g) of its row
    __device__ __forceinline__ static int dim_of(int i, int r, int g) {
        return F32 ? (i / VW) * 16 * VW + VW * (4 * g + r) + i % VW : 16 * i + 4 * g + r;
    }

    // Infinities and NaN among the values of a tile that some rows see and others do not: they were left out of the
    // product, where a row that does not see them would have got 0 * NaN, and are added to the rows that do.
    __device__ __forceinline__ void add_odd(const PagedAttn &c, const PagedSeq &s, const PagedTile &t, int h, int lane, int base, int page0, int page1) {
        const int n = lane & 15, g = lane >> 4;
        for (int k = 0; k < kKeyTile; ++k) {
            const int key = base + k, page = k < 16 ? page0 : page1;
            if (page < 0 || key > t.p_hi) continue;
            const size_t vec = paged_vec(c.a, page, h, key & ((1 << c.a.page_shift) - 1));
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int row = b * 16 + n, pos = s.first + (t.r0 + row) / c.group;
                if (row >= t.rows || !paged_sees(c, pos, key)) continue;
#pragma unroll
                for (int i = 0; i < HD / 16; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v;
                        if constexpr (F8) v = (((const uint8_t *)c.a.v)[vec * HD + dim_of(i, r, g)] & 0x7F) == 0x7F ? __builtin_nanf("") : 0.f;
                        else v = to_f32(((const CT *)c.a.v)[vec * HD + dim_of(i, r, g)]);
                        o[b][i][r] += __builtin_fabsf(v) <= 3.402823466e38f ? 0.f : v;
                    }
            }
        }
    }
};

// Outputs d .. d + 3 of a tile's row from its maximum, sum and weighted values; with d = 0 its log-sum-exp
template <typename OT>
__device__ __forceinline__ void paged_finish(const PagedAttn &c, const PagedSeq &s, const PagedTile &t, int h, int row, int d, float M, float L, f32x4e_t v) {
    const int r = t.r0 + row, tok = r / c.group, qh = h * c.group + r % c.group;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (L == 0.f) v = f32x4e_t{0.f, 0.f, 0.f, 0.f};
    v *= inv;
    OT *p = (OT *)c.out.p + (size_t)(s.row0 + tok) * c.out.row_stride + (size_t)qh * c.out.head_stride + d;
    if (c.out.vec) {
        if constexpr (sizeof(OT) == 4) *(f32x4e_t *)p = v;
        else *(u32x2_t *)p = u32x2_t{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(OT) == 4) p[i] = v[i];
            else p[i].u = (uint16_t)pack_bf16(v[i], 0.f);
        }
    }
    if (c.lse && d == 0) c.lse[(size_t)(s.row0 + tok) * c.n_heads + qh] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994531f;
}

// 16 bytes written through to memory, as st_coherent (wait_stores before they are signalled)
__device__ __forceinline__ void st_coherent4(float *p, f32x4e_t v) { asm volatile("global_store_dwordx4 %0, %1, off sc1" ::"v"(p), "v"(v) : "memory"); }

// What others wrote through, read past the caches that may hold something older
__device__ __forceinline__ float2 ld_coherent2(const float2 *p) {
    const unsigned long long v = __hip_atomic_load((const unsigned long long *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ f32x4e_t ld_coherent4(const float *p) {
    const float2 a = ld_coherent2((const float2 *)p), b = ld_coherent2((const float2 *)p + 1);
    return f32x4e_t{a.x, a.y, b.x, b.y};
}

// How a join reads its parts: past the caches (PAST), 8 bytes at a time, or by plain loads after an acquire of the device's scope, which empties the caches for
// every workgroup of the XCD.  Few rows: PAST (16 sequences of 2000 8-bit keys 21 us, 30 with the acquire); 128 rows of k_paged_chunk have
// enough to read for the acquire (256 rows after 2000 keys 46 us, 53 with PAST).
template <bool PAST> __device__ __forceinline__ float2 join_load2(const float2 *p) {
    if constexpr (PAST) return ld_coherent2(p);
    else return *p;
}
template <bool PAST> __device__ __forceinline__ f32x4e_t join_load4(const float *p) {
    if constexpr (PAST) return ld_coherent4(p);
    else return *(gptr<f32x4e_t>)p;
}

// Whether this workgroup is the last of a unit's `used` to have written its part (its stores were st_coherent); leaves the ticket at zero
template <bool PAST>
__device__ __forceinline__ bool paged_last(const PagedAttn &c, size_t unit, int used, int *shared) {
    wait_stores();
    __syncthreads();
    int *ticket = c.tickets + unit * kPagedTicketInts;
    if (threadIdx.x == 0) *shared = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == used - 1;
    __syncthreads();
    if (!*shared) return false;
    if (threadIdx.x == 0) st_coherent(ticket, 0);
    if constexpr (!PAST) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    return true;
}

// The parts of a unit joined, part i of `used` at place_of(i): their order is that of the key ranges, whoever arrived last.
// A part is tile_rows * HD / 4 vectors of four outputs, of which the first `items` are looked at; where(e) says which row and outputs vector e is.  `table`: LDS for used * tile_rows maxima and
// sums.  A thread has FLIGHT vectors on their way at a time, P parts of FLIGHT / P of its own (the last part again where there are fewer than
// P, then taken as zeros: a weight of 0 would make NaN of its infinities): this is one workgroup's work while others may be done, and latency is what it costs.
struct PagedWhere { int row, d; };
template <typename OT, int HD, int P, int FLIGHT, bool PAST, typename F, typename G>
__device__ __forceinline__ void paged_join_by(const PagedAttn &c, const PagedSeq &s, const PagedTile &t, int h, int used, int items, size_t part_vecs, const float2 *table, F place_of, G where) {
    constexpr int kItems = FLIGHT / P;
    for (int e0 = (int)threadIdx.x; e0 < items; e0 += 256 * kItems) {
        float M[kItems], L[kItems];
        f32x4e_t v[kItems];
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int row = min(where(min(e0 + 256 * k, items - 1)).row, t.rows - 1);
            M[k] = -INFINITY; L[k] = 0.f;
            v[k] = f32x4e_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (int i = 0; i < used; ++i) M[k] = fmaxf(M[k], table[i * t.rows + row].x);
        }
        for (int i0 = 0; i0 < used; i0 += P) {
            f32x4e_t x[kItems][P];
#pragma unroll
            for (int k = 0; k < kItems; ++k)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    x[k][i] = f32x4e_t{0.f, 0.f, 0.f, 0.f};
                    if (where(min(e0 + 256 * k, items - 1)).row < t.rows)        // the others were not written
                        x[k][i] = join_load4<PAST>(c.part_o + ((size_t)place_of(min(i0 + i, used - 1)) * part_vecs + min(e0 + 256 * k, items - 1)) * 4);
                }
#pragma unroll
            for (int k = 0; k < kItems; ++k) {
                const int row = min(where(min(e0 + 256 * k, items - 1)).row, t.rows - 1);
                const float ref = M[k] == -INFINITY ? 0.f : M[k];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 y = table[min(i0 + i, used - 1) * t.rows + row];
                    const float f = i0 + i < used ? __builtin_amdgcn_exp2f(y.x - ref) : 0.f;
                    L[k] += f * y.y;
                    v[k] += f * (i0 + i < used ? x[k][i] : f32x4e_t{0.f, 0.f, 0.f, 0.f});
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int e = e0 + 256 * k;
            const PagedWhere w = where(min(e, items - 1));
            if (e < items && w.row < t.rows) paged_finish<OT>(c, s, t, h, w.row, w.d, M[k], L[k], v[k]);
        }
    }
}
template <typename OT, int HD, int FLIGHT, bool PAST, typename F, typename G>
__device__ __forceinline__ void paged_join(const PagedAttn &c, const PagedSeq &s, const PagedTile &t, int h, int used, int tile_rows, int items, float2 *table, F place_of, G where) {
    const size_t part_vecs = (size_t)tile_rows * (HD / 4);
    for (int e = (int)threadIdx.x; e < used * t.rows; e += 256) table[e] = join_load2<PAST>(c.part_ml + (size_t)place_of(e / t.rows) * tile_rows + e % t.rows);
    __syncthreads();
    if (used <= 4) paged_join_by<OT, HD, 4, FLIGHT, PAST>(c, s, t, h, used, items, part_vecs, table, place_of, where);
    else if (used <= 8) paged_join_by<OT, HD, 8, FLIGHT, PAST>(c, s, t, h, used, items, part_vecs, table, place_of, where);
    else paged_join_by<OT, HD, FLIGHT, FLIGHT, PAST>(c, s, t, h, used, items, part_vecs, table, place_of, where);
}

// Sum over the lanes up to this one, by moves between lanes (DPP: within rows of 16, then row to row)
__device__ __forceinline__ int sum_to_lane(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);      // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);      // row_bcast:31 into rows 2 and 3
    return v;
}

// A unit is a KV head of a (sequence, tile of rows) pair; its work is counted in groups of kGroup key tiles, one tile to each of a workgroup's waves.
constexpr int kGroup = 4;
struct PagedUnit {
    int pair, h;
    int first, groups;              // number of its first group among all units', how many it has
};

// Attention of few rows per KV head, and of float32 models' rows however many.
//  The groups of all units, in the order (pair, KV head), are cut into equal shares, a share to a workgroup: sequences of all lengths keep
//  every compute unit busy to the end, whatever the host knows of the lengths (each wave adds up the pairs' groups itself, 64 at a time).
//  A share is some whole units and up to two parts of units; a part's result goes to memory and the unit's last workgroup to arrive joins them.
//  Where there are more pairs than a wave adds up in a reasonable time, a workgroup takes a unit (c.pairs = 0).
//  A workgroup has NB blocks of 16 rows and all four waves work on the same ones, each on every fourth key tile; they are joined through LDS.
template <typename CT, int HD, int NB>
__global__ __launch_bounds__(256, (NB * HD < 256 && PagedWave<CT, HD, NB>::kRing * PagedWave<CT, HD, NB>::kTile <= 20480) ? 2 : 1) void k_paged_attn(PagedAttn c) {
    using W = PagedWave<CT, HD, NB>;
    using OT = typename std::conditional<sizeof(CT) == 4, float, bf16_t>::type;
    constexpr int kRows = NB * 16, kWaveBytes = W::kRing * W::kTile, kJoin = 4 * 16 * (HD + 4) * 4;
    constexpr int kBytes = 4 * kWaveBytes > kJoin ? 4 * kWaveBytes : kJoin;
    __shared__ __align__(1024) char lds[kBytes];
    __shared__ float2 ml[4][kRows];
    __shared__ int last_one;
    float (*ob)[16][HD + 4] = (float (*)[16][HD + 4])lds;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;

    // ---- which groups are this workgroup's.  The first 64 pairs stay in registers, lane by lane.
    auto pair_of = [&](int pair, PagedSeq &s) {  // a pair's groups of one KV head; at least 1 where there are rows, since they have to be written
        if (pair >= c.pairs && c.pairs) return 0;
        s = paged_seq_lane(c.a, c.row_tiles == 1 ? pair : pair / c.row_tiles);
        if (s.n_rows * c.group > c.few_rows) return 0;                   // k_paged_chunk's
        const PagedTile t = paged_tile<kKeyTile>(c, s, c.row_tiles == 1 ? 0 : pair % c.row_tiles, kRows);
        return t.rows == 0 ? 0 : max(1, (t.tiles + kGroup - 1) / kGroup);
    };
    int pos = 0, end = 0, share = 1, start;      // (the host sees to it that all groups fit 30 bits)
    PagedSeq first64{};
    int groups64 = 0, sum64 = 0;
    auto locate = [&](int at, PagedUnit &u, PagedSeq &s) {
        int before = 0;
        for (int p0 = 0; p0 < c.pairs; p0 += kWave) {
            PagedSeq x = first64;
            const int mine = p0 ? pair_of(p0 + lane, x) : groups64, sum = p0 ? sum_to_lane(mine) : sum64;
            const int first = (before + sum - mine) * c.a.n_kv;
            const uint64_t hit = __ballot(mine > 0 && first <= at && at < first + mine * c.a.n_kv);
            if (hit) {
                const int i = __builtin_ctzll(hit);
                u.pair = p0 + i;
                u.groups = __builtin_amdgcn_readlane(mine, i);
                u.first = __builtin_amdgcn_readlane(first, i);
                u.h = (at - u.first) / u.groups;
                u.first += u.h * u.groups;
                s.row0 = __builtin_amdgcn_readlane(x.row0, i);
                s.n_rows = __builtin_amdgcn_readlane(x.n_rows, i);
                s.kv = __builtin_amdgcn_readlane(x.kv, i);
                s.first = __builtin_amdgcn_readlane(x.first, i);
                s.table = c.a.table + (size_t)(u.pair / c.row_tiles) * c.a.table_stride;
                return true;
            }
            before += __builtin_amdgcn_readlane(sum, kWave - 1);
        }
        return false;                            // not while the lengths stay what they were when the groups were counted
    };
    PagedUnit u{};
    PagedSeq s;
    if (c.pairs) {
        groups64 = pair_of(lane, first64);
        sum64 = sum_to_lane(groups64);
        int total = __builtin_amdgcn_readlane(sum64, kWave - 1), most = groups64;
        for (int p0 = kWave; p0 < c.pairs; p0 += kWave) {
            PagedSeq x;
            const int mine = pair_of(p0 + lane, x);
            most = max(most, mine);
            total += __builtin_amdgcn_readlane(sum_to_lane(mine), kWave - 1);
        }
        total *= c.a.n_kv;
        // equal shares, none smaller than is worth a workgroup, and none so small that LDS could not hold the maxima and sums of a unit's parts
        constexpr int kParts = kBytes / (kRows * 8) - 2;
        share = max(c.min_share, (int)((unsigned)(total + c.shares - 1) / (unsigned)c.shares));
        if (total / c.a.n_kv > share * kParts) {
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, kWave));
            share = max(share, __builtin_amdgcn_readfirstlane(most) / kParts + 1);
        }
        const long from = (long)share * blockIdx.x;
        if (from >= total) return;
        pos = (int)from;
        end = (int)min(from + share, (long)total);
        if (!locate(pos, u, s)) return;
    } else {
        u.pair = (int)blockIdx.x / c.a.n_kv;
        u.h = (int)blockIdx.x % c.a.n_kv;
        PagedSeq x;
        u.groups = end = __builtin_amdgcn_readfirstlane(pair_of(u.pair, x));
        if (end == 0) return;
        s = paged_seq(c.a, u.pair / c.row_tiles);
    }

    start = pos;
    for (;;) {
        const int h = u.h, pair = u.pair;
        const PagedTile t = paged_tile<kKeyTile>(c, s, pair % c.row_tiles, kRows);
        // groups g0 .. g1 of the unit; the whole of it, or one of `used` parts
        const int g0 = pos - u.first, g1 = min(end, u.first + u.groups) - u.first;
        const bool part = g1 - g0 < u.groups;
        const int begin = g0 * kGroup, stop = min(g1 * kGroup, t.tiles);

        // This wave's tiles are begin + wave + 4 i, i < count.  Pages are looked up 32 tiles at a time: lane 2 i + half (and waited for there, where they are checked).
        const int count = stop - begin > wave ? (stop - begin - wave + 3) / 4 : 0;
        auto key_base = [&](int i) { const int v = begin + wave + 4 * i; return (v < t.n_sink ? v : v - t.n_sink + t.t_lo) * kKeyTile; };
        auto look_up = [&](int i0) {
            const int i = i0 + (lane >> 1);
            if (i >= count) return -1;
            const int at = key_base(i) + 16 * (lane & 1);
            return at < s.kv ? paged_page(c.a, s, at) : -1;
        };
        // pages of the tiles being requested, of the next 32, and of the 32 that are worked on
        int pages = look_up(0), pages_next = count > 32 ? look_up(32) : -1, pages_old = pages;
        W w;
        w.init(c, s, t, h, lane);
        if (count > 0) {
            const uint32_t ring = lds_address(lds) + wave * kWaveBytes;
            auto request = [&](int i) {
                if ((i & 31) == 0 && i) {
                    pages_old = pages;
                    pages = pages_next;
                    pages_next = i + 32 < count ? look_up(i + 32) : -1;
                }
                const int p0 = __builtin_amdgcn_readlane(pages, 2 * (i & 31)), p1 = __builtin_amdgcn_readlane(pages, 2 * (i & 31) + 1);
                const uint32_t to = ring + (i % W::kRing) * W::kTile;
                if (c.once) w.template request<true>(c, key_base(i), p0, p1, h, lane, to);
                else w.template request<false>(c, key_base(i), p0, p1, h, lane, to);
            };
#pragma unroll
            for (int i = 0; i < W::kRing; ++i)
                if (i < count) request(i);
            int asked = min(count, W::kRing);
            for (int i = 0; i < count; ++i) {
                // Of the tiles asked for, all but this one may still be on their way.  (As built they seldom are: the compiler does not count these requests, and waits
                // for everything before the first product, whose operand Q it loaded itself.)
                if (asked - i >= W::kRing) wait_requests<(W::kRing - 1) * W::kRequests>();
                else wait_requests<0>();
                const int base = key_base(i), from = (asked - 1) >> 5 == i >> 5 ? pages : pages_old;
                const int p0 = __builtin_amdgcn_readlane(from, 2 * (i & 31)), p1 = __builtin_amdgcn_readlane(from, 2 * (i & 31) + 1);
                const uint32_t at = ring + (i % W::kRing) * W::kTile;
                if (W::whole(c, t, base, p0, p1)) w.template take<false>(c, s, t, h, lane, base, p0, p1, at);
                else w.template take<true>(c, s, t, h, lane, base, p0, p1, at);
                if (asked < count) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // what was read of the tile is here: its place is free
                    request(asked++);
                }
            }
        }

        // ---- the four waves' results
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            w.l[b] += __shfl_xor(w.l[b], 16, kWave);
            w.l[b] += __shfl_xor(w.l[b], 32, kWave);
            if (w.l[b] != w.l[b] && w.m[b] == -INFINITY) w.m[b] = 0.f;      // nothing but NaN: a NaN, not an empty row
            if (g == 0) ml[wave][b * 16 + n] = make_float2(w.m[b], w.l[b]);
        }
        __syncthreads();
        // a part's place: 2 to a workgroup, the first for the unit that its share begins with
        const size_t place = 2 * (size_t)blockIdx.x + (pos == start ? 0 : 1);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float M = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) M = fmaxf(M, ml[i][b * 16 + n].x);
            const float f = w.m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m[b] - M);
            if (b) __syncthreads();
#pragma unroll
            for (int i = 0; i < HD / 16; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) ob[wave][n][W::dim_of(i, r, g)] = w.m[b] == -INFINITY ? 0.f : w.o[b][i][r] * f;
            __syncthreads();
            for (int e = (int)threadIdx.x; e < 16 * (HD / 4); e += 256) {
                const int row = e / (HD / 4), d = e % (HD / 4) * 4;
                if (b * 16 + row >= t.rows) break;
                float R = -INFINITY, L = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) R = fmaxf(R, ml[i][b * 16 + row].x);
#pragma unroll
                for (int i = 0; i < 4; ++i) { const float2 e = ml[i][b * 16 + row]; L += e.x == -INFINITY ? 0.f : e.y * __builtin_amdgcn_exp2f(e.x - R); }
                f32x4e_t v = *(const f32x4e_t *)&ob[0][row][d];
#pragma unroll
                for (int i = 1; i < 4; ++i) v += *(const f32x4e_t *)&ob[i][row][d];
                if (!part) {
                    paged_finish<OT>(c, s, t, h, b * 16 + row, d, R, L, v);
                } else {
                    st_coherent4(c.part_o + (place * kRows + b * 16 + row) * HD + d, v);
                    if (d == 0) {
                        float *p = (float *)(c.part_ml + place * kRows + b * 16 + row);
                        st_coherent(p, R);
                        st_coherent(p + 1, L);
                    }
                }
            }
        }
        if (part) {
            const int w0 = u.first / share, used = (u.first + u.groups - 1) / share - w0 + 1;
            if (paged_last<true>(c, ((size_t)(pair / c.row_tiles) * c.a.n_kv + h) * c.row_tiles + pair % c.row_tiles, used, &last_one)) {
                const int skew = u.first == w0 * share ? 0 : 1;
                paged_join<OT, HD, 32, true>(c, s, t, h, used, kRows, t.rows * (HD / 4), (float2 *)lds, [&](int i) { return 2 * (w0 + i) + (i == 0 ? skew : 0); },
                                         [](int e) { return PagedWhere{e / (HD / 4), e % (HD / 4) * 4}; });
            }
        }
        pos = u.first + g1;
        if (pos >= end) return;
        __syncthreads();
        if (++u.h < c.a.n_kv) u.first += u.groups;
        else if (!locate(pos, u, s)) return;
    }
}

}  // namespace ead
