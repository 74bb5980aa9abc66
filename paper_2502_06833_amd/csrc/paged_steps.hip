// Host side of the steps around a paged cache's attention: ead_rotate, ead_paged_append, ead_paged_weigh, ead_paged_evict.
#include <math.h>

#include <atomic>

#include "evict.hpp"
#include "paged_host.hpp"
#include "paged_rules.hpp"
#include "rotate.hpp"
#include "weigh.hpp"

using namespace ead;

namespace {

ead_status check_rotary(const ead_rotary *r, int head_dim) {
    if (!r) return refuse(EAD_ERR_INVALID_ARG, "rotary is null");
    if (r->head_dim != 32 && r->head_dim != 64 && r->head_dim != 128) return refuse(EAD_ERR_SHAPE, "rotary: head_dim %d is not one of 32, 64, 128", r->head_dim);
    if (head_dim && r->head_dim != head_dim) return refuse(EAD_ERR_SHAPE, "rotary: head_dim %d, the cache's is %d", r->head_dim, head_dim);
    if (r->rotary_dim < 0 || r->rotary_dim > r->head_dim || r->rotary_dim % 16)
        return refuse(EAD_ERR_SHAPE, "rotary: rotary_dim %d is no multiple of 16 from 0 to head_dim", r->rotary_dim);
    if (r->rotary_dim && !r->inv_freq) return refuse(EAD_ERR_INVALID_ARG, "rotary: inv_freq is null");
    if (!(r->eps >= 0.f) || r->eps == INFINITY) return refuse(EAD_ERR_INVALID_ARG, "rotary: eps has to be finite and 0 or more");
    if (((uintptr_t)r->inv_freq & 7) || (((uintptr_t)r->q_gain | (uintptr_t)r->k_gain) & 3)) return refuse(EAD_ERR_INVALID_ARG, "rotary: inv_freq or a gain is not aligned to its elements");
    return EAD_OK;
}

void set_rotary(RotateArgs &c, const ead_rotary *r) {
    c.inv_freq = r->inv_freq;
    c.q_gain = r->q_gain; c.k_gain = r->k_gain;
    c.q_gain_stride = r->gain_per_head ? r->head_dim : 0;
    c.k_gain_stride = c.q_gain_stride;
    c.eps = r->eps;
    c.rotary = r->rotary_dim;
    c.interleaved = r->interleaved != 0;
}

template <typename F> void with_head_dim(int hd, F f) {
    if (hd == 32) f(std::integral_constant<int, 32>{});
    else if (hd == 64) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 128>{});
}

ead_status check_weigh(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_attn *at) {
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

// positions of a sequence at most, as paged_seq cuts them
int held_of(const ead_paged_cache *c, const ead_paged_batch *b) { return (int)std::min({(long)b->max_kv, (long)b->table_width * c->page_size, 0x7FFFFF00l}); }

// LDS that k_evict_choose may use on the current device beside its own arrays
int evict_room() {
    constexpr int kDevices = 64;
    static std::atomic<int> room[kDevices];              // 0: not asked yet
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kDevices) return kEvictPlainLds;
    int n = room[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        n = kEvictLds;
        if (hipFuncSetAttribute((const void *)k_evict_choose, hipFuncAttributeMaxDynamicSharedMemorySize, kEvictLds) != hipSuccess) {
            (void)hipGetLastError();
            n = kEvictPlainLds;
        }
        room[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// How a call of ead_paged_weigh is cut: the workspace is the same whatever the queries' alignment lets it do
struct WeighCall {
    bool few;
    int blocks, tiles;
    WeighPlan m;
    uint64_t bytes;
};
WeighCall weigh_of(const ead_paged_cache *c, const ead_paged_batch *b, const ead_paged_attn *at) {
    const long rows = (long)b->max_q * (at->n_heads / c->n_kv_heads);
    const int held = std::max(1, held_of(c, b));
    WeighCall w{};
    w.few = rows <= weigh_few_rows(c->dtype == EAD_F32, c->head_dim);
    w.blocks = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    w.tiles = weigh_tiles((long)b->batch * c->n_kv_heads, held, compute_units());
    if (!w.few && c->dtype != EAD_F32) {
        w.m = weigh_many(b->batch, c->n_kv_heads, rows, held, compute_units());
        if (w.m.splits > 1) w.bytes = (uint64_t)w.m.splits * b->batch * c->n_kv_heads * w.m.part_keys * 4;
    }
    return w;
}

}  // namespace

extern "C" {

ead_status ead_rotate(const ead_rotary *rotary, int32_t dtype, int32_t rows, int32_t n_heads, int32_t n_kv_heads, const int32_t *positions, const ead_rows *q,
                      const ead_rows *k, const ead_rows *q_out, const ead_rows *k_out, void *hip_stream) {
    PAGED_TRY(check_rotary(rotary, 0));
    if (dtype != EAD_F32 && dtype != EAD_BF16) return refuse(EAD_ERR_INVALID_ARG, "rows: unknown dtype %d", dtype);
    if (rows < 0 || n_heads < 0 || n_kv_heads < 0 || n_heads + (long)n_kv_heads < 1) return refuse(EAD_ERR_INVALID_ARG, "need rows >= 0 and at least one head");
    if ((long)rows * ((long)n_heads + n_kv_heads) >= 1l << 30) return refuse(EAD_ERR_SHAPE, "%d rows of %ld heads, fewer than 2^30 in all are allowed", rows, (long)n_heads + n_kv_heads);
    if (rows == 0) return EAD_OK;
    if (!positions && rotary->rotary_dim) return refuse(EAD_ERR_INVALID_ARG, "positions is null");
    RotateArgs c{};
    if (n_heads) { PAGED_TRY(rows_of(q, dtype, "q", &c.q)); PAGED_TRY(rows_of(q_out, dtype, "q_out", &c.q_out)); }
    if (n_kv_heads) { PAGED_TRY(rows_of(k, dtype, "k", &c.k)); PAGED_TRY(rows_of(k_out, dtype, "k_out", &c.k_out)); }
    set_rotary(c, rotary);
    c.a.rows = rows;
    c.positions = positions;
    c.n_heads = n_heads; c.n_kv = n_kv_heads;
    const long total = (long)n_heads + n_kv_heads, per_group = 256 / (rotary->head_dim / 16);
    const bool wide = rotate_wide(rows, total, rotary->head_dim, element_bytes(dtype));
    c.groups = (int)rotate_units(n_heads, n_kv_heads, 0, wide ? kRotateEach : 1);
    const dim3 grid((unsigned)std::clamp(((long)rows * c.groups + per_group - 1) / per_group, 1l, 1l << 20));       // the kernel goes on past its grid
    with_head_dim(rotary->head_dim, [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        auto go = [&](auto rt) {
            using RT = decltype(rt);
            if (!wide) hipLaunchKernelGGL((k_rotate<RT, HD, 1, false>), grid, dim3(256), 0, (hipStream_t)hip_stream, c);
            else if constexpr (rotate_shares(sizeof(RT), HD)) hipLaunchKernelGGL((k_rotate<RT, HD, kRotateEach, true>), grid, dim3(256), 0, (hipStream_t)hip_stream, c);
        };
        if (dtype == EAD_F32) go(0.f);
        else go(bf16_t{});
    });
    return launched("ead_rotate");
}

ead_status ead_paged_append(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_rotary *rotary, int32_t dtype, int32_t n_heads,
                            const int32_t *positions, const ead_rows *q, const ead_rows *k, const ead_rows *v, const ead_rows *q_out, void *hip_stream) {
    PAGED_TRY(check_cache(cache));
    PAGED_TRY(check_rotary(rotary, cache->head_dim));
    if (n_heads < 0) return refuse(EAD_ERR_INVALID_ARG, "n_heads is 0 or more");
    const long total = (long)n_heads + 2l * cache->n_kv_heads;
    PAGED_TRY(check_batch(batch, total));
    if (dtype != EAD_F32 && dtype != EAD_BF16) return refuse(EAD_ERR_INVALID_ARG, "rows: unknown dtype %d", dtype);
    if (batch->rows == 0) return EAD_OK;
    RotateArgs c{};
    if (n_heads) { PAGED_TRY(rows_of(q, dtype, "q", &c.q)); PAGED_TRY(rows_of(q_out, dtype, "q_out", &c.q_out)); }
    PAGED_TRY(rows_of(k, dtype, "k", &c.k));
    PAGED_TRY(rows_of(v, dtype, "v", &c.v));
    set_rotary(c, rotary);
    c.a = args_of(cache, batch);
    c.positions = positions;
    c.n_heads = n_heads; c.n_kv = cache->n_kv_heads;
    const bool wide = rotate_wide(batch->rows, total, cache->head_dim, element_bytes(dtype));
    c.groups = (int)rotate_units(n_heads, cache->n_kv_heads, cache->n_kv_heads, wide ? kRotateEach : 1);
    const long per_group = 256 / (cache->head_dim / 16);
    const dim3 grid((unsigned)std::clamp(((long)batch->max_q * c.groups + per_group - 1) / per_group, 1l, 1l << 20), (unsigned)batch->batch);
    with_cache(cache, [&](auto ct, auto hd) {
        using CT = decltype(ct);
        constexpr int HD = decltype(hd)::value;
        auto go = [&](auto rt) {
            using RT = decltype(rt);
            if (!wide) hipLaunchKernelGGL((k_append<CT, RT, HD, 1, false>), grid, dim3(256), 0, (hipStream_t)hip_stream, c);
            else if constexpr (rotate_shares(sizeof(RT), HD)) hipLaunchKernelGGL((k_append<CT, RT, HD, kRotateEach, true>), grid, dim3(256), 0, (hipStream_t)hip_stream, c);
        };
        if (dtype == EAD_F32) go(0.f);
        else go(bf16_t{});
    });
    return launched("ead_paged_append");
}

ead_status ead_paged_weigh_workspace(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_attn *attn, uint64_t *bytes) {
    if (!bytes) return refuse(EAD_ERR_INVALID_ARG, "bytes is null");
    *bytes = 0;
    PAGED_TRY(check_weigh(cache, batch, attn));
    *bytes = weigh_of(cache, batch, attn).bytes;
    return EAD_OK;
}

ead_status ead_paged_weigh(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_attn *attn, const ead_rows *q, const float *lse,
                           float *weights, void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    PAGED_TRY(check_weigh(cache, batch, attn));
    if (batch->rows == 0) return EAD_OK;
    if (!lse || !weights) return refuse(EAD_ERR_INVALID_ARG, "lse or weights is null");
    if (((uintptr_t)lse | (uintptr_t)weights) & 3) return refuse(EAD_ERR_INVALID_ARG, "lse or weights is not aligned to its elements");
    PagedWeigh c{};
    PAGED_TRY(rows_of(q, attn->dtype, "q", &c.q));
    const WeighCall w = weigh_of(cache, batch, attn);
    if (w.bytes && (!workspace || workspace_bytes < w.bytes || ((uintptr_t)workspace & 15)))
        return refuse(EAD_ERR_INVALID_ARG, "workspace: %llu bytes, 16-byte aligned, are needed", (unsigned long long)w.bytes);
    c.a = args_of(cache, batch);
    c.lse = lse; c.weights = weights;
    c.n_heads = attn->n_heads; c.group = attn->n_heads / cache->n_kv_heads;
    c.c2 = attn->scale * kLog2e;
    c.window = attn->window; c.sinks = attn->sinks;
    const int held = std::max(1, held_of(cache, batch));
    const hipStream_t st = (hipStream_t)hip_stream;
    const long few_groups = (held + 128l * w.tiles - 1) / (128l * w.tiles) * cache->n_kv_heads, many_groups = (long)cache->n_kv_heads * w.m.splits * (w.m.part_keys / 256);
    if ((w.few ? few_groups : many_groups) >= 1l << 24)
        return refuse(EAD_ERR_SHAPE, "batch: max_kv of %d positions for each of %d KV heads needs 2^24 workgroups or more", batch->max_kv, cache->n_kv_heads);
    if (w.few) {
        c.tiles = w.tiles;
        const dim3 grid((unsigned)few_groups, (unsigned)batch->batch);
        with_cache(cache, [&](auto ct, auto hd) {
            using CT = decltype(ct);
            constexpr int HD = decltype(hd)::value;
            if (w.blocks == 1) hipLaunchKernelGGL((k_weigh_few<CT, HD, 1>), grid, dim3(256), 0, st, c);
            else if (w.blocks == 2) hipLaunchKernelGGL((k_weigh_few<CT, HD, 2>), grid, dim3(256), 0, st, c);
            else if constexpr (weigh_few_rows(sizeof(CT) == 4, HD) == 64) hipLaunchKernelGGL((k_weigh_few<CT, HD, 4>), grid, dim3(256), 0, st, c);
        });
    } else if (cache->dtype != EAD_F32 && c.q.vec) {
        c.splits = w.m.splits; c.part_keys = w.m.part_keys;
        c.part = (float *)workspace;
        const dim3 grid((unsigned)many_groups, (unsigned)batch->batch);
        with_cache(cache, [&](auto ct, auto hd) {
            using CT = decltype(ct);
            if constexpr (sizeof(CT) != 4) hipLaunchKernelGGL((k_weigh_many<CT, decltype(hd)::value>), grid, dim3(256), 0, st, c);
        });
        if (w.m.splits > 1)
            hipLaunchKernelGGL(k_weigh_join, dim3((unsigned)(w.m.part_keys / 256), (unsigned)cache->n_kv_heads, (unsigned)batch->batch), dim3(256), 0, st, c);
    } else {
        const dim3 grid(weigh_simple_groups(held), (unsigned)cache->n_kv_heads, (unsigned)batch->batch);
        with_cache(cache, [&](auto ct, auto hd) { hipLaunchKernelGGL((k_weigh<decltype(ct), decltype(hd)::value>), grid, dim3(256), 0, st, c); });
    }
    return launched("ead_paged_weigh");
}

ead_status ead_paged_evict_workspace(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_eviction *ev, uint64_t *bytes) {
    if (!bytes) return refuse(EAD_ERR_INVALID_ARG, "bytes is null");
    *bytes = 0;
    PAGED_TRY(check_cache(cache));
    PAGED_TRY(check_batch(batch, 1));
    if (!ev) return refuse(EAD_ERR_INVALID_ARG, "eviction is null");
    if (ev->keep < 1 || ev->sinks < 0 || ev->recent < 0 || (long)ev->sinks + ev->recent > ev->keep)
        return refuse(EAD_ERR_INVALID_ARG, "eviction: need keep >= 1, sinks >= 0, recent >= 0 and sinks + recent <= keep");
    if (held_of(cache, batch) > kEvictMost) return refuse(EAD_ERR_SHAPE, "batch: sequences of up to 2^20 positions can be cut, max_kv is %d", batch->max_kv);
    const uint64_t units = (uint64_t)batch->batch * cache->n_kv_heads;
    *bytes = evict_moves_at(units) + (held_of(cache, batch) > ev->keep ? units * (uint64_t)(ev->keep - ev->sinks - ev->recent) * 8 : 0);      // (moves: only where something is cut)
    return EAD_OK;
}

ead_status ead_paged_evict(const ead_paged_cache *cache, const ead_paged_batch *batch, const ead_paged_eviction *ev, const float *scores, float *weights,
                           int32_t *kept, void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    uint64_t need = 0;
    PAGED_TRY(ead_paged_evict_workspace(cache, batch, ev, &need));
    if (!scores || !kept) return refuse(EAD_ERR_INVALID_ARG, "scores or kept is null");
    if ((uintptr_t)scores & 15) return refuse(EAD_ERR_INVALID_ARG, "scores have to be 16-byte aligned");
    if (((uintptr_t)weights | (uintptr_t)kept) & 3) return refuse(EAD_ERR_INVALID_ARG, "weights or kept is not aligned to its elements");
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))
        return refuse(EAD_ERR_INVALID_ARG, "workspace: %llu bytes, 16-byte aligned, are needed", (unsigned long long)need);
    PagedEvict c{};
    c.a = args_of(cache, batch);
    c.scores = scores; c.weights = weights; c.kept = kept;
    c.counts = (int *)workspace;
    c.moves = (int2 *)((char *)workspace + evict_moves_at((uint64_t)batch->batch * cache->n_kv_heads));
    c.keep = ev->keep; c.sinks = ev->sinks; c.recent = ev->recent;
    const int held = held_of(cache, batch), vec_bytes = cache->head_dim * element_bytes(cache->dtype);
    c.held = held;
    c.cached = evict_cached(held, evict_room());
    if (c.cached < 4) return refuse(EAD_ERR_SHAPE, "batch: max_kv %d is more than this device's local memory lets be cut", held);
    const EvictPlan p = evict_plan(batch->batch, cache->n_kv_heads, held, ev->keep, ev->recent, vec_bytes, compute_units());
    const size_t lds = (size_t)c.cached * 4 + (size_t)evict_words(held) * 8;
    hipLaunchKernelGGL(k_evict_choose, dim3((unsigned)cache->n_kv_heads, (unsigned)batch->batch), dim3(p.threads), lds, (hipStream_t)hip_stream, c);
    if (held > ev->keep) {
        auto move = [&](int steps, int columns, int shares, int threads) {
            c.steps = steps; c.shares = shares;
            c.columns = columns; c.column_bytes = vec_bytes / columns;
            const unsigned parts = 2 * columns + (cache->dtype == EAD_FP8 ? 2 : 0) + (weights ? 1 : 0);       // the weights are the last
            hipLaunchKernelGGL(k_evict_move, dim3((unsigned)(cache->n_kv_heads * shares), parts, (unsigned)batch->batch), dim3(threads), 0, (hipStream_t)hip_stream, c);
        };
        if (p.shares) {
            move(kEvictFill, 1, p.shares, 256);
            if (ev->recent) move(kEvictShift, p.columns, 1, p.shift_threads);
        } else move(kEvictFill | kEvictShift, p.columns, 1, p.shift_threads);
    }
    return launched("ead_paged_evict");
}

}  // extern "C"
