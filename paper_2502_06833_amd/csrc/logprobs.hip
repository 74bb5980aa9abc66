// Host side of ead_logprobs.
#include "logprobs.hpp"

#include <math.h>

#include <algorithm>

#include "paged_host.hpp"
#include "paged_rules.hpp"

using namespace ead;

namespace {

ead_status check_logprobs(const ead_logprob_call *c) {
    if (!c) return refuse(EAD_ERR_INVALID_ARG, "call is null");
    if (c->dtype != EAD_F32 && c->dtype != EAD_BF16) return refuse(EAD_ERR_INVALID_ARG, "logits: unknown dtype %d", c->dtype);
    if (c->rows < 0 || c->rows > 1 << 22) return refuse(EAD_ERR_SHAPE, "%d rows, 0 .. 2^22 are allowed", c->rows);
    if (c->vocab < 1 || c->vocab > 1 << 24) return refuse(EAD_ERR_SHAPE, "vocab %d is not in 1 .. 2^24", c->vocab);
    if (c->top < 0 || c->top > kTopMost || c->top > c->vocab) return refuse(EAD_ERR_INVALID_ARG, "top %d is not in 0 .. %d", c->top, std::min(kTopMost, c->vocab));
    if (c->unit != EAD_NATS && c->unit != EAD_BITS) return refuse(EAD_ERR_INVALID_ARG, "unit must be 0 or 1");
    if (c->rows > 1 && c->row_stride < 0) return refuse(EAD_ERR_INVALID_ARG, "row_stride is 0 or more");
    return EAD_OK;
}

constexpr uint64_t kStatsAt = (uint64_t)kLogprobTickets * kLpTicketInts * 4;       // tickets first, as many whatever the shape: calls of any shape follow each other
uint64_t logprob_bytes(const ead_logprob_call *c, const LogprobPlan &p) {
    if (p.parts == 1) return 0;
    const uint64_t cells = (uint64_t)c->rows * p.parts;
    return kStatsAt + cells * sizeof(LpPartial) + cells * c->top * 8;
}

}  // namespace

extern "C" {

ead_status ead_logprobs_workspace(const ead_logprob_call *call, uint64_t *bytes) {
    if (!bytes) return refuse(EAD_ERR_INVALID_ARG, "bytes is null");
    *bytes = 0;
    PAGED_TRY(check_logprobs(call));
    *bytes = logprob_bytes(call, logprob_plan(call->rows, call->vocab, kSet, compute_units()));
    return EAD_OK;
}

ead_status ead_logprobs(const ead_logprob_call *call, void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    PAGED_TRY(check_logprobs(call));
    if (call->rows == 0) return EAD_OK;
    const int esz = element_bytes(call->dtype);
    if (!call->logits || (uintptr_t)call->logits % esz) return refuse(EAD_ERR_INVALID_ARG, "logits is null or not aligned to its elements");
    if (!call->tokens && (call->logprob || call->rank)) return refuse(EAD_ERR_INVALID_ARG, "logprob and rank go with tokens");
    if (call->top && (!call->top_tokens || !call->top_logprobs)) return refuse(EAD_ERR_INVALID_ARG, "top_tokens or top_logprobs is null");
    if (((uintptr_t)call->tokens | (uintptr_t)call->logprob | (uintptr_t)call->rank | (uintptr_t)call->H | (uintptr_t)call->top_tokens | (uintptr_t)call->top_logprobs) & 3)
        return refuse(EAD_ERR_INVALID_ARG, "tokens or an output is not aligned to its elements");
    const LogprobPlan p = logprob_plan(call->rows, call->vocab, kSet, compute_units());
    const uint64_t need = logprob_bytes(call, p);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
        return refuse(EAD_ERR_INVALID_ARG, "workspace: %llu bytes, 16-byte aligned, are needed", (unsigned long long)need);
    LogprobArgs a{};
    a.logits = call->logits; a.stride = call->row_stride; a.rows = call->rows; a.V = call->vocab;
    a.tokens = call->logprob || call->rank ? call->tokens : nullptr;
    a.top = call->top; a.unit = call->unit; a.parts = p.parts; a.part_sets = p.part_sets;
    a.logprob = call->logprob; a.H = call->H; a.rank = call->rank; a.top_tokens = call->top_tokens; a.top_logprobs = call->top_logprobs;
    if (p.parts > 1) {
        const uint64_t cells = (uint64_t)call->rows * p.parts;
        a.tickets = (int *)workspace;
        a.stats = (LpPartial *)((char *)workspace + kStatsAt);
        a.list_value = (float *)(a.stats + cells);
        a.list_token = (int *)(a.list_value + cells * call->top);
    }
    const dim3 grid((unsigned)((long)call->rows * p.parts));
    const hipStream_t st = (hipStream_t)hip_stream;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (call->top) hipLaunchKernelGGL((k_logprobs<T, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_logprobs<T, false>), grid, dim3(256), 0, st, a);
    };
    if (call->dtype == EAD_BF16) go(bf16_t{});
    else go(0.f);
    return launched("ead_logprobs");
}

}  // extern "C"
