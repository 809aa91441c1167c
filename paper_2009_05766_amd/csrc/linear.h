// Linear layers with an epilogue, and their gradients: internal launch interface.
#pragma once
#include "gemm.h"

namespace netmax {

struct LinearArgs {
    int64_t batch, rows, din, dout; int bf16, act;
    const void *x, *w, *bias, *residual; void *y, *z;
    int64_t ldx, ldw, ldr, ldy, ldz, sx, sw, sb, sr, sy, sz;
};
int64_t linear_workspace(const LinearArgs &a);
void launch_linear(hipStream_t s, const LinearArgs &a, void *work);

// dy, x, w, z as in the forward pass; dx, dw, db may be null.  db: [batch][dout], sdb from one to the next.
struct LinearGradArgs {
    int64_t batch, rows, din, dout; int bf16, act;
    const void *dy, *x, *w, *z; void *dx, *dw, *db;
    int64_t lddy, ldx, ldw, ldz, lddx, lddw, sdy, sx, sw, sz, sdx, sdw, sdb;
};
int64_t linear_grad_workspace(const LinearGradArgs &a);
void launch_linear_grad(hipStream_t s, const LinearGradArgs &a, void *work);

}  // namespace netmax
