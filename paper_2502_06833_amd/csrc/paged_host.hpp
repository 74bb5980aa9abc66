// What the host sides of the calls over a paged cache share: their checks, the kernels' arguments, the choice of a template by a cache's type.
#pragma once
#include "../../include/ead.h"

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <type_traits>

#include "paged.hpp"

namespace ead {

ead_status report(ead_status st, const char *text);

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

}  // namespace

}  // namespace ead
