// The rows that count in a backward pass, side by side: what workgroups of 1024 threads and kGathered rows each share.
#pragma once

#include "eager_matrix.h"
#include "eager_model_rules.h"

namespace eager {

struct Gather {
    const void *x;
    const long long *target;
    const float *lse, *dloss;
    long long rows, stride;
    int width;
    float by;                // of dloss
    const int *before;       // per workgroup: counted rows in front of them, or NULL: each counts them
    void *x_out;             // [counted][width]
    long long *target_out;
    float *lse_out, *dloss_out;
    int *place;              // per row: where it went, -1: nowhere
    int *counted;
    float *common;           // the first weight with an exponent of 0, or NULL
};

// By a wavefront: where the rows from `first` on go, `before` of those in front of them counted, each lane one row's target.
__device__ __forceinline__ void place_rows(const Gather &g, long long first, int before, long long target, int *place)
{
    const int lane = threadIdx.x & 63;
    const long long row = first + lane;
    const bool mine = lane < kGathered && row < g.rows, in = mine && ((target >= 0) & (g.dloss[row] != 0.0f));
    const unsigned long long mask = __ballot(in);
    const int to = in ? before + __popcll(mask & ((1ull << lane) - 1)) : -1;
    if (lane < kGathered) place[lane] = to;
    if (mine) g.place[row] = to;
    if (in) {
        const float weight = g.dloss[row] * g.by;
        g.target_out[to] = target;
        g.lse_out[to] = g.lse[row];
        g.dloss_out[to] = weight;
        if (g.common && to == 0) *g.common = __uint_as_float((__float_as_uint(weight) & 0x7fffff) | 0x3f800000);
    }
    if (lane == 0 && first + kGathered >= g.rows) {
        *g.counted = before + __popcll(mask);
        if (g.common && before == 0 && mask == 0) *g.common = 1.0f;
    }
}

// By a workgroup: the rows of x.
template <typename T>
__device__ __forceinline__ void move_rows(const Gather &g, long long first, const int *place)
{
    constexpr int E = 16 / sizeof(T);
    const int chunks = g.width / E;
#pragma unroll 4
    for (int i = threadIdx.x; i < kGathered * chunks; i += 1024) {
        const int in = i / chunks, at = (i - in * chunks) * E;
        if (place[in] >= 0)
            *reinterpret_cast<f32x4 *>(static_cast<T *>(g.x_out) + static_cast<long long>(place[in]) * g.width + at) =
                *reinterpret_cast<const f32x4 *>(static_cast<const T *>(g.x) + (first + in) * g.stride + at);
    }
}

}  // namespace eager
