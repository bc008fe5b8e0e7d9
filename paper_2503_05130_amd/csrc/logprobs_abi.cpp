// C ABI of token log probabilities.  All checks of their arguments are here.
#include <cstdint>

#include "abi.h"
#include "logprobs.h"

using namespace iefwd;

namespace {

void check_sizes(uint32_t rows, uint32_t vocab, uint32_t n_top) {
    if (rows == 0 || rows > (1u << 22) || vocab == 0 || vocab > (1u << 24) || (uint64_t)rows * vocab > (1ull << 35))
        fail(IEFWD_EINVAL, "rows must be in [1, 2^22], vocab in [1, 2^24] and their product at most 2^35");
    if (n_top > (uint32_t)kMaxTop || n_top > vocab) fail(IEFWD_EINVAL, "n_top must be at most 32 and at most vocab");
}

void check_logits(const char *what, uint32_t type, const void *p, uint64_t stride, uint32_t vocab) {
    if (type > IEFWD_F32) fail(IEFWD_EINVAL, "unknown type");
    if (!p || (uintptr_t)p % (type == IEFWD_F32 ? 4 : 2)) fail(IEFWD_EINVAL, std::string(what) + " is NULL or not aligned");
    if (stride < vocab || stride > (1ull << 40)) fail(IEFWD_EINVAL, "the row stride must be at least vocab and at most 2^40");
}

void check_scale(float scale) {
    if (!(scale >= 0x1p-30f && scale <= 0x1p30f)) fail(IEFWD_EINVAL, "scale must be in [2^-30, 2^30]");
}

}  // namespace

extern "C" {

int iefwd_token_logprobs_workspace(uint32_t rows, uint32_t vocab, uint32_t n_top, size_t *bytes) {
    return guarded([&] {
        if (!bytes) fail(IEFWD_EINVAL, "bytes is NULL");
        check_sizes(rows, vocab, n_top);
        *bytes = logprobs_workspace((int)rows, (int)vocab, (int)n_top);
    });
}

int iefwd_token_logprobs(uint32_t type, const void *logits, uint64_t stride, uint32_t rows, uint32_t vocab,
                         const int64_t *tokens, float scale, float *logprobs, float *entropy, float *stats, uint32_t n_top,
                         int32_t *top_ids, float *top_logprobs, void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&] {
        check_sizes(rows, vocab, n_top);
        check_logits("logits", type, logits, stride, vocab);
        check_scale(scale);
        if (!tokens || !logprobs || (n_top && (!top_ids || !top_logprobs))) fail(IEFWD_EINVAL, "NULL pointer");
        const size_t need = logprobs_workspace((int)rows, (int)vocab, (int)n_top);
        if (workspace_bytes < need || (need && (!workspace || !aligned16(workspace))))
            fail(IEFWD_EINVAL, "workspace of " + std::to_string(need) + " bytes (16-byte aligned) needed, " +
                                   std::to_string(workspace_bytes) + " given");
        LogprobArgs a{};
        a.logits = logits;
        a.tokens = tokens;
        a.logprobs = logprobs;
        a.entropy = entropy;
        a.stats = stats;
        a.top_ids = top_ids;
        a.top_logprobs = top_logprobs;
        a.workspace = workspace;
        a.stride = (int64_t)stride;
        a.rows = (int)rows;
        a.vocab = (int)vocab;
        a.top = (int)n_top;
        a.scale = scale;
        a.f32 = type == IEFWD_F32;
        hip_check(launch_logprobs(a, (hipStream_t)stream), "log probabilities launch");
    });
}

int iefwd_token_logprobs_grad(uint32_t type, const void *logits, uint64_t stride, uint32_t rows, uint32_t vocab,
                              const int64_t *tokens, float scale, const float *stats, const float *entropy,
                              const float *grad_logprobs, const float *grad_entropy, void *out, uint64_t out_stride,
                              void *stream) {
    return guarded([&] {
        check_sizes(rows, vocab, 0);
        check_logits("logits", type, logits, stride, vocab);
        check_logits("out", type, out, out_stride, vocab);
        check_scale(scale);
        if (!tokens || !stats) fail(IEFWD_EINVAL, "NULL pointer");
        if (!grad_logprobs && !grad_entropy) fail(IEFWD_EINVAL, "grad_logprobs and grad_entropy are both NULL");
        if (grad_entropy && !entropy) fail(IEFWD_EINVAL, "grad_entropy needs the entropy");
        if (out == logits && out_stride != stride) fail(IEFWD_EINVAL, "out in the place of logits needs their row stride");
        LogprobGradArgs a{};
        a.logits = logits;
        a.tokens = tokens;
        a.stats = stats;
        a.entropy = entropy;
        a.grad_logprobs = grad_logprobs;
        a.grad_entropy = grad_entropy;
        a.out = out;
        a.stride = (int64_t)stride;
        a.out_stride = (int64_t)out_stride;
        a.rows = (int)rows;
        a.vocab = (int)vocab;
        a.scale = scale;
        a.f32 = type == IEFWD_F32;
        hip_check(launch_logprobs_grad(a, (hipStream_t)stream), "log probabilities gradient launch");
    });
}

}  // extern "C"
