// Internal interface between the host side of the model operators and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eager {

// A view of rows of heads (element strides).
struct Heads {
    void *data;
    long long row, head;
};

struct NormRopeArgs {
    Heads x[2], y[2];                // q, k: inputs; outputs (backward: gradients of the outputs)
    Heads dx[2];                     // backward
    const void *w[2];
    void *dw[2];
    const float *cos_table, *sin_table;
    const int *positions;
    float *partials;                 // backward: per workgroup, gradient of both gains
    long long tokens, table_rows;
    int heads[2];
    int dim;
    int per_block;                   // tokens a workgroup takes at a time
    int blocks;
    float eps, inv_dim;
};

struct AttentionArgs {
    Heads q, k, v, out, dout, dq, dk, dv;
    float *lse;
    float *delta, *start;            // backward, per row and head: -sum(dout * out), -lse / scale
    float *sums;                     // backward: dk, dv of each part, where there is more than one
    int parts;
    const int *cu;
    long long tokens;
    int q_heads, kv_heads, dim, sequences;
    float scale;
};

struct CrossEntropyArgs {
    const void *x, *w;
    const long long *target;
    float *loss, *lse;
    const float *dloss;
    void *dx, *dw;
    char *workspace;
    long long rows, x_stride, w_stride;
    int width, vocab;
    long long workspace_bytes;
};

hipError_t launch_norm_rope(const NormRopeArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_norm_rope_backward(const NormRopeArgs &a, bool bf16, hipStream_t stream);

hipError_t launch_attention(const AttentionArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_attention_backward(const AttentionArgs &a, bool bf16, hipStream_t stream);

hipError_t launch_cross_entropy(const CrossEntropyArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_cross_entropy_backward(const CrossEntropyArgs &a, bool bf16, hipStream_t stream);

}  // namespace eager
