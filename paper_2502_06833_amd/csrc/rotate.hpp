// Norms of queries and keys for each head with the position rotation in the same pass: from rows to rows, and on the way to a paged cache.
#pragma once
#include "paged.hpp"

namespace ead {

struct RotateArgs {
    PagedArgs a;                         // the cache and the batch (k_append); of k_rotate only a.rows
    RowsArg q, k, v, q_out, k_out;
    const int *positions;                // [rows], or null: the batch's own
    const double *inv_freq;              // [rotary_dim / 2]: radians a position
    const float *q_gain, *k_gain;        // null: that one is not normalised
    long q_gain_stride, k_gain_stride;   // from head to head, 0: one gain for all
    float eps;
    int n_heads, n_kv, rotary, interleaved;
    int groups;                          // units of a row's heads (rotate_unit)
};

// Sine and cosine of a quarter turn's fraction: |r| <= 1/2, the angle r pi / 2 is at most pi / 4 in magnitude, where the Taylor series up to x^9 and x^10 are off by
// less than 2^-28.  With the roundings of pi / 2, of x and of the sums the sine is off by at most 1.23 * 2^-24 (2.2 units in its last place, where it is small), the cosine by
// 1.44 * 2^-24: the largest over all floats r of 2^-25 and more; r's own rounding adds 0.4 * 2^-24 at most.
__device__ __forceinline__ void sincos_quarter(float r, float &s, float &c) {
    const float x = r * 1.57079632679489662f, y = x * x;
    s = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
    s = __builtin_fmaf(x * y, s, x);
    c = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f);
    c = __builtin_fmaf(y, c, 1.f);
}
// The angle position * freq in 64 bits, brought to a quarter turn's fraction there: far positions (2^20 and more turns of the fastest pair) lose nothing that a float holds.
__device__ __forceinline__ void sincos_of(double position, double freq, float &s, float &c) {
    double turns = position * freq * 0.15915494309189533577;
    turns = 4.0 * (turns - __builtin_rint(turns));
    const double n = __builtin_rint(turns);
    sincos_quarter((float)(turns - n), s, c);
    const int quarter = (int)n;                                // -2 .. 2
    if (quarter & 1) { const float t = s; s = c; c = -t; }
    if (quarter & 2) { s = -s; c = -c; }
}

// HD / 16 lanes share a vector; each holds two runs of 8 elements, at `at` and `too`: of the rotated part those that are turned against each other (halves: i and
// i + rotary / 2; interleaved: 2 i and 2 i + 1, so the runs follow each other), and past it whatever is left.
struct RotateLane {
    int at, too;
    bool turns;
};
__device__ __forceinline__ RotateLane rotate_lane(int lane, int rotary, int interleaved) {
    const int half = rotary / 16;                              // lanes that turn something
    RotateLane l;
    l.turns = lane < half;
    l.at = interleaved ? 16 * lane : l.turns ? 8 * lane : 2 * 8 * lane;
    l.too = !interleaved && l.turns ? l.at + rotary / 2 : l.at + 8;
    return l;
}

template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

template <int HD>
__device__ __forceinline__ void norm_turn(float (&x)[8], float (&y)[8], const float (&gx)[8], const float (&gy)[8], bool norm, float eps, bool turns, bool interleaved,
                                          const float (&sn)[8], const float (&cs)[8]) {
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], __builtin_fmaf(y[e], y[e], sum));
        sum = lanes_sum<HD / 16>(sum);
        const float f = 1.f / sqrtf(sum * (1.f / HD) + eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[e] *= f * gx[e]; y[e] *= f * gy[e]; }
    }
    if (!turns) return;
    if (interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = x[2 * e], b = x[2 * e + 1], c = y[2 * e], d = y[2 * e + 1];
            x[2 * e] = __builtin_fmaf(a, cs[e], -(b * sn[e])); x[2 * e + 1] = __builtin_fmaf(b, cs[e], a * sn[e]);
            y[2 * e] = __builtin_fmaf(c, cs[4 + e], -(d * sn[4 + e])); y[2 * e + 1] = __builtin_fmaf(d, cs[4 + e], c * sn[4 + e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[e], b = y[e];
            x[e] = __builtin_fmaf(a, cs[e], -(b * sn[e]));
            y[e] = __builtin_fmaf(b, cs[e], a * sn[e]);
        }
    }
}

// The sixteen elements of this lane to the cache, rounded to its type (as put8 in paged.hpp, which has eight to a lane)
template <typename CT, int HD, bool STREAM>
__device__ __forceinline__ void put16(void *pool, uint8_t *scales, size_t vec, int lane, const RotateLane &l, float (&x)[8], float (&y)[8], bool live) {
    if constexpr (sizeof(CT) == 1) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = __builtin_fabsf(x[e]), b = __builtin_fabsf(y[e]);
            m = a <= 3.402823466e38f ? fmaxf(m, a) : m;
            m = b <= 3.402823466e38f ? fmaxf(m, b) : m;
        }
#pragma unroll
        for (int o = HD / 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
        const int ex = fp8_exponent(m);
        const float inv = exp2_of(254 - ex);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = __builtin_fabsf(x[e]) <= 3.402823466e38f ? x[e] * inv : __builtin_nanf("");
            y[e] = __builtin_fabsf(y[e]) <= 3.402823466e38f ? y[e] * inv : __builtin_nanf("");
        }
        if (live) {
            put<STREAM>((u32x2_t *)((uint8_t *)pool + vec * HD + l.at), u32x2_t{fp8_pack4(x[0], x[1], x[2], x[3]), fp8_pack4(x[4], x[5], x[6], x[7])});
            put<STREAM>((u32x2_t *)((uint8_t *)pool + vec * HD + l.too), u32x2_t{fp8_pack4(y[0], y[1], y[2], y[3]), fp8_pack4(y[4], y[5], y[6], y[7])});
            if (lane == 0) scales[vec] = (uint8_t)ex;
        }
    } else if (live) {
        set8<STREAM>((CT *)pool + vec * HD + l.at, 1, x);
        set8<STREAM>((CT *)pool + vec * HD + l.too, 1, y);
    }
}

// A group of HD / 16 lanes takes EACH heads of one kind (queries, keys, or values on their way to the pages) of a row, all of them requested before the first is worked
// on; the row's sines and cosines are computed once for them, meanwhile.  Bound by memory, with vector instructions (the sines above all) at two thirds of their rate
// beside it: 16381 rows of 40 heads of 128 in bf16 73 us (4.6 TB/s; a large copy runs at 5.2), with values to bf16 pages, 28504 rows, 127 us (5.5 TB/s).  Four heads: eight took
// 81 and 134 us (registers), one head in a loop 125 and 170.  STREAM: non-temporal accesses, for calls that move more than the second-level caches hold.
struct RotateUnit {
    int kind, first, heads;              // 0: queries, 1: keys, 2: values; heads first .. first + heads - 1
};
template <int EACH>
__device__ __forceinline__ RotateUnit rotate_unit(const RotateArgs &c, int u) {
    const int uq = (c.n_heads + EACH - 1) / EACH, uk = (c.n_kv + EACH - 1) / EACH;
    RotateUnit r;
    r.kind = u < uq ? 0 : u < uq + uk ? 1 : 2;
    r.first = (u - (r.kind == 0 ? 0 : r.kind == 1 ? uq : uq + uk)) * EACH;
    r.heads = min(EACH, (r.kind == 0 ? c.n_heads : c.n_kv) - r.first);
    return r;
}

// Eight elements at any alignment
__device__ __forceinline__ void rotate_gather(Vec8<float> &v, const float *p) {
    v.lo = f32x4e_t{p[0], p[1], p[2], p[3]};
    v.hi = f32x4e_t{p[4], p[5], p[6], p[7]};
}
__device__ __forceinline__ void rotate_gather(Vec8<bf16_t> &v, const bf16_t *p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v.raw[e] = (uint32_t)p[2 * e].u | (uint32_t)p[2 * e + 1].u << 16;
}

template <typename CT, typename RT, int HD, int EACH, bool STREAM, bool APPEND>
__device__ __forceinline__ void rotate_row(const RotateArgs &c, const RotateUnit &u, size_t row, int position, int lane, const RotateLane &l, size_t page_vec, bool live) {
    const RowsArg &from = u.kind == 0 ? c.q : u.kind == 1 ? c.k : c.v;
    const RT *p = (const RT *)from.p + row * from.row_stride + u.first * from.head_stride;
    // (as they lie in memory, and without a branch between them: unpacked one by one they were waited for one by one)
    Vec8<RT> rx[EACH], ry[EACH];
    if (from.vec) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const RT *v = p + min(e, u.heads - 1) * from.head_stride;
            if constexpr (STREAM) { rx[e].load_stream(v + l.at); ry[e].load_stream(v + l.too); }
            else { rx[e].load(v + l.at); ry[e].load(v + l.too); }
        }
    } else {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const RT *v = p + min(e, u.heads - 1) * from.head_stride;
            rotate_gather(rx[e], v + l.at);
            rotate_gather(ry[e], v + l.too);
        }
    }
    const float *gain = u.kind == 0 ? c.q_gain : u.kind == 1 ? c.k_gain : nullptr;
    const long apart = u.kind == 0 ? c.q_gain_stride : c.k_gain_stride;
    float gx[8] = {}, gy[8] = {}, sn[8] = {}, cs[8] = {};
    auto gains = [&](int h) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { gx[e] = gain[h * apart + l.at + e]; gy[e] = gain[h * apart + l.too + e]; }
    };
    if (gain && !apart) gains(0);
    const bool turns = l.turns && u.kind < 2;
    if (turns) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sincos_of((double)position, c.inv_freq[8 * lane + e], sn[e], cs[e]);
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        if (e >= u.heads) continue;
        const int h = u.first + e;
        float x[8], y[8];
        rx[e].unpack(x);
        ry[e].unpack(y);
        if (gain && apart) gains(h);
        norm_turn<HD>(x, y, gx, gy, gain != nullptr, c.eps, turns, c.interleaved, sn, cs);
        if (u.kind == 0 || !APPEND) {
            const RowsArg &to = u.kind == 0 ? c.q_out : c.k_out;
            RT *o = (RT *)to.p + row * to.row_stride + h * to.head_stride;
            set8<STREAM>(o + l.at, to.vec, x);
            set8<STREAM>(o + l.too, to.vec, y);
        } else {
            put16<CT, HD, STREAM>((void *)(u.kind == 1 ? c.a.k : c.a.v), (uint8_t *)(u.kind == 1 ? c.a.ks : c.a.vs), page_vec + ((size_t)h << c.a.page_shift), lane, l, x, y, live);
        }
    }
}

template <typename RT, int HD, int EACH, bool STREAM>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs c) {
    constexpr int L = HD / 16, kGroups = 256 / L;
    const int lane = (int)threadIdx.x % L;
    const RotateLane l = rotate_lane(lane, c.rotary, c.interleaved);
    const unsigned total = (unsigned)c.a.rows * (unsigned)c.groups;            // below 2^30
    for (unsigned i = blockIdx.x * kGroups + threadIdx.x / L; i < total; i += gridDim.x * kGroups) {
        const unsigned row = i / (unsigned)c.groups;
        rotate_row<RT, RT, HD, EACH, STREAM, false>(c, rotate_unit<EACH>(c, (int)(i % (unsigned)c.groups)), row, c.positions ? c.positions[row] : 0, lane, l, 0, false);
    }
}

// Rows of no sequence are not touched; keys and values of rows below position 0, past the table or in holes go nowhere.
template <typename CT, typename RT, int HD, int EACH, bool STREAM>
__global__ __launch_bounds__(256) void k_append(RotateArgs c) {
    constexpr int L = HD / 16, kGroups = 256 / L;
    const int lane = (int)threadIdx.x % L;
    const RotateLane l = rotate_lane(lane, c.rotary, c.interleaved);
    const PagedSeq s = paged_seq(c.a, blockIdx.y);
    const unsigned total = (unsigned)s.n_rows * (unsigned)c.groups;
    for (unsigned i = blockIdx.x * kGroups + threadIdx.x / L; i < total; i += gridDim.x * kGroups) {
        const int t = (int)(i / (unsigned)c.groups), pos = s.first + t;
        const RotateUnit u = rotate_unit<EACH>(c, (int)(i % (unsigned)c.groups));
        const size_t row = (size_t)(s.row0 + t);
        const int page = u.kind && pos >= 0 && pos < s.kv ? paged_page(c.a, s, pos) : -1;
        const size_t vec = paged_vec(c.a, max(page, 0), 0, pos & ((1 << c.a.page_shift) - 1));
        rotate_row<CT, RT, HD, EACH, STREAM, true>(c, u, row, c.positions ? c.positions[row] : pos, lane, l, vec, page >= 0);
    }
}

}  // namespace ead
