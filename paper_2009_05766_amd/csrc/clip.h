// The norm of all gradients of a model and their scaling to a largest norm: internal launch interface.
#pragma once
#include "../../include/netmax.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace netmax {

// out: null for the norm alone.  norm: one number for every model of the batch, or null.
struct ClipArgs { int64_t batch, n; const netmax_gradient *tensors; bool scale; float max_norm; float *norm; };
int64_t clip_workspace(int64_t batch, int64_t n, const netmax_gradient *tensors);
void launch_clip(hipStream_t s, const ClipArgs &a, void *work);

}  // namespace netmax
