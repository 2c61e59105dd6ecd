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

// A teacher's lists beside CrossEntropyArgs; index NULL: there are none.
struct TeacherArgs {
    const long long *index;
    const float *logits;
    float *picked;
    int entries;
    float temperature;
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
    TeacherArgs teacher;             // distillation: its lists take the targets' place
};

// A view of rows (element stride); data may be NULL where an array is not wanted.
struct Rows {
    void *data;
    long long stride;
};

struct LayerNormArgs {
    Rows x, residual;                // backward: s, gradient of s
    Rows sum, y;                     // backward: gradient of x, gradient of y
    const void *w, *b;
    void *dw, *db;
    float *stats;                    // [2][rows]: mean, 1 / deviation
    float *partials;                 // backward, per workgroup: gradients of gain and bias
    long long rows;
    int width, blocks;
    float eps, inv_width;
};

struct RotaryArgs {
    Heads x[2], y[2];                // q, k
    const float *cos_table, *sin_table;
    const int *positions;
    long long tokens, table_rows;
    int heads[2], groups[2];         // groups: of heads that a thread takes one after the other
    int dim, half;                   // half: pairs of a head
    int moved[2];                    // elements of a head that are read and written
    float sign;                      // of the sines
};

struct TableArgs {
    double quarters[64];             // quarter turns a position, per pair
    double magnitude;
    float *cos_table, *sin_table;
    long long positions;
    int half;
};

hipError_t launch_norm_rope(const NormRopeArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_norm_rope_backward(const NormRopeArgs &a, bool bf16, hipStream_t stream);

hipError_t launch_attention(const AttentionArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_attention_backward(const AttentionArgs &a, bool bf16, hipStream_t stream);

hipError_t launch_cross_entropy(const CrossEntropyArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_cross_entropy_backward(const CrossEntropyArgs &a, bool bf16, hipStream_t stream);

hipError_t launch_layer_norm(const LayerNormArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_layer_norm_backward(const LayerNormArgs &a, bool bf16, hipStream_t stream);

hipError_t launch_rotary(const RotaryArgs &a, bool bf16, bool interleaved, hipStream_t stream);
hipError_t launch_rotary_table(const TableArgs &a, hipStream_t stream);

}  // namespace eager
