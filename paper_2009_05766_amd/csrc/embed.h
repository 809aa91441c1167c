// Rows of an embedding table for given tokens, and the table's gradient: internal launch interface.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace netmax {

// Every matrix of the batch: ids [tokens], table [vocab][width], y [tokens][width] (or dy, and the table's gradient).
struct EmbedArgs {
    int64_t batch, tokens, vocab, width; int bf16, accumulate; float scale;
    const int32_t *ids; void *table; void *y;          // the lookup writes y, the gradient table
    int64_t s_ids, ldt, st, ldy, sy;
};

// The workgroups of a launch of the gradient, in order: `sums` that sum rows of tokens, `zeros` that clear rows of the table, and those that the shape of the launch adds, with nothing to do.
struct GradTurns {
    uint32_t sums, zeros;
    __host__ __device__ bool clears(uint32_t id) const { return id >= sums && id - sums < zeros; }
};

void launch_embed(hipStream_t s, const EmbedArgs &a);
int64_t embed_grad_workspace(const EmbedArgs &a);
void launch_embed_grad(hipStream_t s, const EmbedArgs &a, void *work);

}  // namespace netmax
