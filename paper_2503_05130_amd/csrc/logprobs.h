// Log probabilities of given tokens over a vocabulary (csrc/logprobs.hip).  The
// launchers check nothing: the C entry points do.
#pragma once

#include "launch.h"

namespace iefwd {

constexpr int kMaxTop = 32;      // alternatives of a row

struct LogprobArgs {
    const void *logits;          // bf16 or fp32 [rows, vocab], rows stride elements apart
    const int64_t *tokens;       // [rows]; outside [0, vocab): no token
    float *logprobs;             // [rows]
    float *entropy;              // [rows] or null
    float *stats;                // [rows, 2] or null: the largest logit, and log sum exp(scale (x - largest))
    int32_t *top_ids;            // [rows, top]
    float *top_logprobs;         // [rows, top]
    void *workspace;
    int64_t stride;
    int rows, vocab, top;
    float scale;
    bool f32;
};

size_t logprobs_workspace(int rows, int vocab, int top);
hipError_t launch_logprobs(const LogprobArgs &a, hipStream_t stream);

struct LogprobGradArgs {
    const void *logits;
    const int64_t *tokens;
    const float *stats;
    const float *entropy;        // with grad_entropy
    const float *grad_logprobs, *grad_entropy;      // [rows], null: 0
    void *out;                   // as logits, rows out_stride apart
    int64_t stride, out_stride;
    int rows, vocab;
    float scale;
    bool f32;
};
hipError_t launch_logprobs_grad(const LogprobGradArgs &a, hipStream_t stream);

}  // namespace iefwd
