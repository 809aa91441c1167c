// Norms before and after a block with its gate and the residual stream, and their gradients: internal launch interface.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace netmax {

struct Span { void *p; int64_t ld, s; };               // rows of values: first one, distances of rows and of matrices of the batch

enum Gate : int { GATE_NONE = 0, GATE_SIGMOID = 1, GATE_TANH = 2 };

struct NormArgs {
    int64_t batch, rows, width;
    int bf16, layer, act, gate_rows, post, pre; float x_scale, f_scale;
    double eps, share;                                 // share: 1 / width
    Span x, f, gate, post_gain, post_bias, pre_gain, pre_bias, h, y;
    Span dy, dh, dx, df, dgate, dpost_gain, dpost_bias, dpre_gain, dpre_bias;
};
void launch_block_norm(hipStream_t s, const NormArgs &a);
int64_t block_norm_grad_workspace(const NormArgs &a);
void launch_block_norm_grad(hipStream_t s, const NormArgs &a, void *work);

}  // namespace netmax
