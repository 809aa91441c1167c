// Losses on the log probabilities of sampled tokens, and the gradient of their logits: internal launch interface.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace netmax {

// Row t of logits [tokens][vocab] (ld apart) and its label.  weight may be null (all 1); a row whose weight is 0 or whose label lies
// outside 0 .. vocab - 1 is not read and takes part in nothing.
struct TokenRows {
    int64_t tokens, vocab, ld; const void *logits; const int32_t *labels; const float *weight; int bf16;
};

struct PolicyArgs { const float *old_logp, *ref_logp, *advantage; float low, high, kl; float *loss, *logp; void *grad; int64_t ldg; };
void launch_policy_loss(hipStream_t s, const TokenRows &rows, const PolicyArgs &a);

// offsets [2 pairs + 1]: sequence q has rows offsets[q] .. offsets[q + 1] - 1; sequences 2 p (chosen) and 2 p + 1 (rejected) are a pair.
struct PreferenceArgs {
    int64_t pairs; const int32_t *offsets; const float *ref_logp; float beta, smoothing, scale; float *loss, *ratio; void *grad; int64_t ldg;
    float2 *stats; double *terms; float *slope;                     // workspace: [tokens], [tokens], [2 pairs]
};
void launch_preference_loss(hipStream_t s, const TokenRows &rows, const PreferenceArgs &a);

}  // namespace netmax
