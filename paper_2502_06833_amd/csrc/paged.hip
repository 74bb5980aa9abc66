// Host side of the paged cache: the C entry points ead_paged_*, their checks and launches.
#include "../../include/ead.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "paged.hpp"
#include "paged_chunk.hpp"
#include "paged_rules.hpp"

namespace ead { ead_status report(ead_status st, const char *text); }

using namespace ead;

namespace {

ead_status refuse(ead_status st, const char *fmt, ...) {
    char buf[256];
    va_list ap; va_start(ap, fmt); vsnprintf(buf, sizeof buf, fmt, ap); va_end(ap);
    return report(st, buf);
}
#define PAGED_TRY(expr) do { ead_status s_ = (expr); if (s_ != EAD_OK) return s_; } while (0)

constexpr float kLog2e = 1.4426950408889634f;
int element_bytes(int dtype) { return dtype == EAD_F32 ? 4 : dtype == EAD_BF16 ? 2 : 1; }

ead_status check_cache(const ead_paged_cache *c) {
    if (!c) return refuse(EAD_ERR_INVALID_ARG, "cache is null");
    if (c->dtype != EAD_F32 && c->dtype != EAD_BF16 && c->dtype != EAD_FP8) return refuse(EAD_ERR_INVALID_ARG, "cache: unknown dtype %d", c->dtype);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535) return refuse(EAD_ERR_SHAPE, "cache: need n_pages >= 1 and 1 <= n_kv_heads <= 65535");
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
        return refuse(EAD_ERR_SHAPE, "cache: page_size %d is not one of 16, 32, 64, 128, 256", c->page_size);
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return refuse(EAD_ERR_SHAPE, "cache: head_dim %d is not one of 32, 64, 128", c->head_dim);
    if (!c->k || !c->v) return refuse(EAD_ERR_INVALID_ARG, "cache: k or v is null");
    if ((c->dtype == EAD_FP8) != (c->k_scale && c->v_scale) || (c->dtype != EAD_FP8 && (c->k_scale || c->v_scale)))
        return refuse(EAD_ERR_INVALID_ARG, "cache: k_scale and v_scale go with EAD_FP8 and with nothing else");
    if (((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 15)
        return refuse(EAD_ERR_INVALID_ARG, "cache: pages and scales have to be 16-byte aligned");
    return EAD_OK;
}

ead_status check_batch(const ead_paged_batch *b, long heads) {
    if (!b) return refuse(EAD_ERR_INVALID_ARG, "batch is null");
    if (!b->page_table || !b->q_starts || !b->kv_lens) return refuse(EAD_ERR_INVALID_ARG, "batch: page_table, q_starts or kv_lens is null");
    if (b->batch < 1 || b->batch > 65535) return refuse(EAD_ERR_INVALID_ARG, "batch: %d sequences, 1 .. 65535 are allowed", b->batch);
    if (b->rows < 0 || b->max_q < 0 || b->min_q < 0 || b->min_q > b->max_q || b->max_q > b->rows || b->max_kv < 0)
        return refuse(EAD_ERR_INVALID_ARG, "batch: need 0 <= min_q <= max_q <= rows and max_kv >= 0");
    if (b->table_width < 1 || b->table_stride < b->table_width) return refuse(EAD_ERR_INVALID_ARG, "batch: need 1 <= table_width <= table_stride");
    if ((long)b->rows * heads >= 1l << 30) return refuse(EAD_ERR_SHAPE, "batch: %d rows of %ld heads, fewer than 2^30 in all are allowed", b->rows, heads);
    return EAD_OK;
}

PagedArgs args_of(const ead_paged_cache *c, const ead_paged_batch *b) {
    PagedArgs a{};
    a.k = c->k; a.v = c->v; a.ks = c->k_scale; a.vs = c->v_scale;
    a.n_pages = c->n_pages; a.page_shift = __builtin_ctz((unsigned)c->page_size); a.n_kv = c->n_kv_heads;
    a.table = b->page_table; a.q_starts = b->q_starts; a.kv_lens = b->kv_lens;
    a.table_stride = b->table_stride; a.table_width = b->table_width; a.rows = b->rows;
    return a;
}

ead_status rows_of(const ead_rows *r, int dtype, const char *name, RowsArg *out) {
    if (!r || !r->data) return refuse(EAD_ERR_INVALID_ARG, "%s is null", name);
    const int per = 16 / element_bytes(dtype);
    if ((uintptr_t)r->data % element_bytes(dtype)) return refuse(EAD_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    *out = RowsArg{r->data, (long)r->row_stride, (long)r->head_stride,
                   ((uintptr_t)r->data & 15) == 0 && r->row_stride % per == 0 && r->head_stride % per == 0};
    return EAD_OK;
}

int compute_units() {
    static const int n = [] {
        int dev = 0, v = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v < 1) v = 256;
        return v;
    }();
    return n;
}

ead_status launched(const char *name) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? EAD_OK : refuse(EAD_ERR_DEVICE, "%s: %s", name, hipGetErrorString(e));
}

// f<cache type, head_dim>
template <typename CT, typename F> void with_dim(int hd, F f) {
    if (hd == 32) f(CT{}, std::integral_constant<int, 32>{});
    else if (hd == 64) f(CT{}, std::integral_constant<int, 64>{});
    else f(CT{}, std::integral_constant<int, 128>{});
}
template <typename F> void with_cache(const ead_paged_cache *c, F f) {
    if (c->dtype == EAD_F32) with_dim<float>(c->head_dim, f);
    else if (c->dtype == EAD_BF16) with_dim<bf16_t>(c->head_dim, f);
    else with_dim<fp8_t>(c->head_dim, f);
}

ead_status copy_rows(const ead_paged_cache *cache, const ead_paged_batch *batch, int32_t dtype, const ead_rows *k, const ead_rows *v,
                     hipStream_t st, bool write) {
    PAGED_TRY(check_cache(cache));
    PAGED_TRY(check_batch(batch, cache->n_kv_heads));
    if (dtype != EAD_F32 && dtype != EAD_BF16) return refuse(EAD_ERR_INVALID_ARG, "rows: unknown dtype %d", dtype);
    if (batch->rows == 0) return EAD_OK;
    PagedCopy c{};
    PAGED_TRY(rows_of(k, dtype, "k", &c.k));
    PAGED_TRY(rows_of(v, dtype, "v", &c.v));
    c.a = args_of(cache, batch);
    const long vecs = (long)batch->max_q * cache->n_kv_heads, per = 256 / (cache->head_dim / 8);
    const bool stream = paged_copy_streams(batch->rows, cache->n_kv_heads, cache->head_dim, element_bytes(dtype) + element_bytes(cache->dtype));
    const dim3 grid((unsigned)std::clamp((vecs + per - 1) / per, 1l, 1l << 20), (unsigned)batch->batch);     // the kernels go on past their grid
    with_cache(cache, [&](auto ct, auto hd) {
        using CT = decltype(ct);
        constexpr int HD = decltype(hd)::value;
        auto go = [&](auto rt, auto stream) {
            using RT = decltype(rt);
            constexpr bool STREAM = decltype(stream)::value;
            if (write) hipLaunchKernelGGL((k_paged_write<CT, RT, HD, STREAM>), grid, dim3(256), 0, st, c);
            else hipLaunchKernelGGL((k_paged_read<CT, RT, HD, STREAM>), grid, dim3(256), 0, st, c);
        };
        if (dtype == EAD_F32) { if (stream) go(0.f, std::true_type{}); else go(0.f, std::false_type{}); }
        else { if (stream) go(bf16_t{}, std::true_type{}); else go(bf16_t{}, std::false_type{}); }
    });
    return launched(write ? "ead_paged_write" : "ead_paged_read");
}

ead_status check_attention(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_attn *at) {
    PAGED_TRY(check_cache(cache));
    if (!at) return refuse(EAD_ERR_INVALID_ARG, "attn is null");
    if (at->n_heads < 1 || at->n_heads % cache->n_kv_heads || at->n_heads / cache->n_kv_heads > 64)
        return refuse(EAD_ERR_SHAPE, "n_heads / n_kv_heads = %d / %d is no integer from 1 to 64", at->n_heads, cache->n_kv_heads);
    PAGED_TRY(check_batch(batch, at->n_heads));
    if (at->dtype != (cache->dtype == EAD_F32 ? EAD_F32 : EAD_BF16))
        return refuse(EAD_ERR_INVALID_ARG, "queries are EAD_F32 over an EAD_F32 cache, EAD_BF16 over the others: got %d over %d", at->dtype, cache->dtype);
    if (at->window < 0 || at->sinks < 0) return refuse(EAD_ERR_INVALID_ARG, "window and sinks are 0 or more");
    if (!(at->scale > 0.f) || !(at->scale * kLog2e < INFINITY)) return refuse(EAD_ERR_INVALID_ARG, "scale has to be positive, and scale / ln 2 finite");
    return EAD_OK;
}

// k_paged_attn for a cache and a number of blocks, and how many of its workgroups the device holds
struct FewKernel {
    void (*fn)(PagedAttn);
    long resident;
};
template <typename CT, int HD, int NB> FewKernel few_kernel() {
    static const int per_cu = [] {
        int n = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_paged_attn<CT, HD, NB>, 256, 0) != hipSuccess || n < 1) { (void)hipGetLastError(); n = 1; }
        return n;
    }();
    return {k_paged_attn<CT, HD, NB>, (long)per_cu * compute_units()};
}
FewKernel few_kernel(const ead_paged_cache *c, int nb) {
    FewKernel k{};
    with_cache(c, [&](auto ct, auto hd) {
        using CT = decltype(ct);
        constexpr int HD = decltype(hd)::value;
        if (nb == 1) k = few_kernel<CT, HD, 1>();
        else if (nb == 2) k = few_kernel<CT, HD, 2>();
        else if constexpr (paged_max_blocks(HD) == 4) k = few_kernel<CT, HD, 4>();
    });
    return k;
}

thread_local double g_small_work = kPagedSmallWork;    // ead_test_paged's, for the calls of its thread
thread_local bool g_always_shares = false;

// The launches of a call: sequences with few rows (of a float32 cache: all), then those with many
struct PagedCall {
    bool few, many;
    int few_rows;
    FewKernel kernel;
    PagedShares f;
    PagedPlan m;
    uint64_t f_bytes, m_bytes;
};
PagedCall plan_of(const ead_paged_cache *c, const ead_paged_batch *b, const ead_paged_attn *at) {
    const long capacity = (long)b->table_width * c->page_size;
    const int held = (int)std::min((long)b->max_kv, capacity), group = at->n_heads / c->n_kv_heads, cus = compute_units();
    const bool f32 = c->dtype == EAD_F32;
    const long rows = (long)b->max_q * group;
    PagedCall p{};
    const double work = paged_work(b->batch, c->n_kv_heads, c->head_dim, group, rows, held, at->window, at->sinks);
    const double kv_bytes = 2.0 * b->batch * c->n_kv_heads * c->head_dim * element_bytes(c->dtype) * (double)paged_keys(16, 32, group, held, at->window, at->sinks);
    p.few_rows = f32 || work <= g_small_work ? 0x7FFFFFFF : paged_few_rows(c->head_dim);
    p.few = (long)b->min_q * group <= p.few_rows;
    p.many = rows > p.few_rows;
    if (p.few) {
        const long few = std::min(rows, (long)p.few_rows);
        const int nb = paged_blocks(f32, few, paged_max_blocks(c->head_dim), work, kv_bytes);
        p.kernel = few_kernel(c, nb);
        p.f = paged_few(b->batch, c->n_kv_heads, few, nb, group, held, capacity, at->window, at->sinks, p.kernel.resident,
                        g_always_shares ? 0 : kPagedWholeGroups, g_always_shares ? 0 : kPagedWholeTiles);
        p.f_bytes = paged_workspace(p.f.units, p.f.parts, 16 * nb, c->head_dim);
    }
    if (p.many) {
        p.m = paged_many(b->batch, c->n_kv_heads, group, rows, held, at->window, at->sinks, cus, c->head_dim);
        p.m_bytes = paged_workspace(p.m.units, p.m.splits > 1 ? p.m.units * p.m.splits : 0, p.m.tile_rows, c->head_dim);
    }
    return p;
}

void set_workspace(PagedAttn &c, void *ws, long units, long parts, int tile_rows) {
    c.tickets = (int *)ws;
    c.part_ml = (float2 *)((char *)ws + units * kPagedTicketInts * 4);
    c.part_o = (float *)(c.part_ml + (size_t)parts * tile_rows);
}

}  // namespace

extern "C" {

ead_status ead_paged_write(const ead_paged_cache *cache, const ead_paged_batch *batch, int32_t dtype, const ead_rows *k, const ead_rows *v,
                           void *hip_stream) {
    return copy_rows(cache, batch, dtype, k, v, (hipStream_t)hip_stream, true);
}

ead_status ead_paged_read(const ead_paged_cache *cache, const ead_paged_batch *batch, int32_t dtype, const ead_rows *k, const ead_rows *v,
                          void *hip_stream) {
    return copy_rows(cache, batch, dtype, k, v, (hipStream_t)hip_stream, false);
}

ead_status ead_paged_workspace(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_attn *attn, uint64_t *bytes) {
    if (!bytes) return refuse(EAD_ERR_INVALID_ARG, "bytes is null");
    *bytes = 0;
    PAGED_TRY(check_attention(cache, batch, attn));
    const PagedCall p = plan_of(cache, batch, attn);
    *bytes = p.f_bytes + p.m_bytes;
    return EAD_OK;
}

ead_status ead_paged_attention(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_attn *attn, const ead_rows *q,
                               const ead_rows *out, float *lse, void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    PAGED_TRY(check_attention(cache, batch, attn));
    if (batch->rows == 0) return EAD_OK;
    PagedAttn c{};
    PAGED_TRY(rows_of(q, attn->dtype, "q", &c.q));
    PAGED_TRY(rows_of(out, attn->dtype, "out", &c.out));
    const PagedCall p = plan_of(cache, batch, attn);
    const uint64_t need = p.f_bytes + p.m_bytes;
    if ((p.few && p.f.groups >= 1 << 24) || (p.many && (long)p.m.row_tiles * p.m.splits * cache->n_kv_heads >= 1 << 24))
        return refuse(EAD_ERR_SHAPE, "batch: max_q of %d rows for each of %d sequences needs 2^24 workgroups or more", batch->max_q, batch->batch);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
        return refuse(EAD_ERR_INVALID_ARG, "workspace: %llu bytes, 16-byte aligned, are needed", (unsigned long long)need);
    c.a = args_of(cache, batch);
    c.lse = lse;
    c.n_heads = attn->n_heads;
    c.group = attn->n_heads / cache->n_kv_heads;
    c.c2 = attn->scale * kLog2e;
    c.window = attn->window;
    c.sinks = attn->sinks;
    c.few_rows = p.few_rows;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (p.few) {
        set_workspace(c, workspace, p.f.units, p.f.parts, 16 * p.f.nb);
        c.row_tiles = p.f.row_tiles; c.pairs = p.f.pairs; c.shares = (int)p.f.groups; c.min_share = p.f.min_share;
        c.once = p.f.row_tiles == 1;
        hipLaunchKernelGGL(p.kernel.fn, dim3((unsigned)p.f.groups), dim3(256), 0, st, c);
    }
    if (p.many) {
        set_workspace(c, (char *)workspace + p.f_bytes, p.m.units, p.m.units * p.m.splits, p.m.tile_rows);
        c.row_tiles = p.m.row_tiles; c.splits = p.m.splits; c.split_tiles = p.m.split_tiles;
        const dim3 grid((unsigned)((long)p.m.row_tiles * p.m.splits * c.a.n_kv), (unsigned)batch->batch);
        with_cache(cache, [&](auto ct, auto hd) {
            using CT = decltype(ct);
            if constexpr (sizeof(CT) != 4) {
                if (attn->one_term) hipLaunchKernelGGL((k_paged_chunk<CT, decltype(hd)::value, false>), grid, dim3(256), 0, st, c);
                else hipLaunchKernelGGL((k_paged_chunk<CT, decltype(hd)::value, true>), grid, dim3(256), 0, st, c);
            }
        });
    }
    return launched("ead_paged_attention");
}

// For the Python classes, in no header: the number of the capture that a stream is in, 0 where nothing is captured
ead_status ead_stream_capture(void *hip_stream, uint64_t *id) {
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    unsigned long long n = 0;
    const hipError_t e = hipStreamGetCaptureInfo((hipStream_t)hip_stream, &status, &n);
    if (e != hipSuccess) return refuse(EAD_ERR_DEVICE, "hipStreamGetCaptureInfo: %s", hipGetErrorString(e));
    *id = status == hipStreamCaptureStatusActive ? n : 0;
    return EAD_OK;
}

// For the tests alone, in no header: the work up to which one kernel takes a call alone (-1: as ever), and whether units are always cut into shares, for
// the calling thread.
ead_status ead_test_paged(double small_work, int32_t always_shares) {
    g_small_work = small_work < 0 ? kPagedSmallWork : small_work;
    g_always_shares = always_shares != 0;
    return EAD_OK;
}

}  // extern "C"
