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

struct Unit { float mean, rest, r; };                  // N(v) = ((v - mean) - rest) r

// What a row's gradients at one column need to know of all others.
struct RowSums { Unit post, pre; float mean_e, mean_eh; };

// The workspace of the gradients.  Sums over the rows, in order: dg1, db1, dg2, db2, dq.  The rows of a workgroup (of the rows' kernel, or of one that goes down the columns) leave their sums in its
// own row of partial sums [sums][padded].
constexpr int SUMS = 5;
struct Partials {
    float *p; int64_t padded, workgroups; int32_t place[SUMS]; int32_t sums; Span out[SUMS];  // place: which of the rows that are there, -1: none
    RowSums *rows;                                     // [batch][rows], where the sums are taken by a kernel of their own
    void *unwanted; int64_t row_workgroups;            // room for results that nobody wants: a row for each group of lanes of the rows' kernel, which has so many workgroups for a matrix
    int64_t bytes;                                     // of the whole workspace
    // Values before the row of one of the `groups` groups of lanes of a workgroup.
    __host__ __device__ int64_t unwanted_row(int64_t matrix, int64_t workgroup, int64_t group, int64_t groups) const { return ((matrix * row_workgroups + workgroup) * groups + group) * padded; }
};

void launch_block_norm(hipStream_t s, const NormArgs &a);
int64_t block_norm_grad_workspace(const NormArgs &a);
void launch_block_norm_grad(hipStream_t s, const NormArgs &a, void *work);

}  // namespace netmax
