// How much of the rows' attention every cached position gets, added to what it had: the weights that a cache is cut by.
#pragma once
#include "paged.hpp"

namespace ead {

struct PagedWeigh {
    PagedArgs a;
    RowsArg q;
    const float *lse;               // [row][query head]
    float *weights;                 // [page][KV head][slot]
    int n_heads, group;             // group: query heads per KV head
    float c2;                       // scale * log2(e)
    int window, sinks;
};
__device__ __forceinline__ bool weigh_sees(const PagedWeigh &c, int pos, int key) {
    return key <= pos && (!c.window || pos - key < c.window || key < c.sinks);
}

// A wave takes 16 keys against blocks of 16 rows (a row: a token and a head of the group): S = Q K^T with the rows as the M of the product and the keys as its N, so
// that lane (n, g) = (lane & 15, lane >> 4) gets key n's scores of rows 4 g .. 4 g + 3 and adds their exponentials up by itself; the four g are added at the end.
// Every position has one owner: no atomics, and the sums' order is fixed.
template <typename CT, int HD>
__global__ __launch_bounds__(256) void k_weigh(PagedWeigh c) {
    constexpr bool F32 = sizeof(CT) == 4;
    constexpr int KE = F32 ? 4 : 8, KL = HD / 4 / KE;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4, h = (int)blockIdx.y;
    const PagedSeq s = paged_seq(c.a, blockIdx.z);
    const int rows = s.n_rows * c.group;
    if (rows == 0) return;
    for (int base = ((int)blockIdx.x * 4 + wave) * 16; base < s.kv; base += (int)gridDim.x * 64) {
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
        for (int r0 = 0; r0 < rows; r0 += 16) {
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
        if (g == 0 && key < s.kv) {
            float *w = c.weights + vec;
            *w = key < s.first ? *w + sum : sum;
        }
    }
}

}  // namespace ead
