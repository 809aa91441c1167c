// Orthogonalised momentum updates: internal launch interface.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace netmax {

struct OrthArgs {
    int64_t batch, rows, cols; int bf16, steps, nesterov; float mu, a, b, c, eps, scale;
    const void *g; const float *m; float *m_out; void *out;         // m, m_out null: no momentum
    int64_t ldg, sg, ldm, sm, ldo, so;
};
int64_t orth_workspace(const OrthArgs &a);
void launch_orth(hipStream_t s, const OrthArgs &a, void *work);

}  // namespace netmax
