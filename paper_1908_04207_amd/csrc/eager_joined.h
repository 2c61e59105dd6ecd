// What tiles of a product have left for every row, joined by workgroups that take kJoined rows each: 64 threads a row
// share its tiles, four loads of each under way at a time.
#pragma once

#include "eager_matrix.h"

namespace eager {

constexpr int kJoined = 16;                              // rows a workgroup of 1024 threads

__device__ __forceinline__ void join(float &top, float &sum, float2 q)
{
    const float both = fmaxf(top, q.x), zero = both == -__builtin_inff() ? 0.0f : both;
    sum = sum * exp2_fast(top - zero) + q.y * exp2_fast(q.x - zero);
    top = both;
}

// Maximum (as a power of two) and sum of row blockIdx.x * kJoined + threadIdx.x, in threads 0 .. kJoined - 1.
__device__ __forceinline__ float2 joined_statistics(const float2 *stats, long long rows, int tiles, float2 (&part)[16][kJoined])
{
    constexpr int Threads = 1024 / kJoined;                 // of a row
    const int in = threadIdx.x % kJoined, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + in;
    float top = -__builtin_inff(), sum = 0.0f;
    if (row < rows)
        for (int t = threadIdx.x / kJoined; t < tiles; t += 4 * Threads) {
            float2 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q[i] = t + Threads * i < tiles ? stats[(t + Threads * i) * rows + row] : make_float2(-__builtin_inff(), 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) join(top, sum, q[i]);
        }
#pragma unroll
    for (int other = kJoined; other < 64; other *= 2) {
        const float2 q = make_float2(__shfl_xor(top, other, 64), __shfl_xor(sum, other, 64));
        join(top, sum, q);
    }
    if (lane < kJoined) part[wave][in] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x < kJoined)
#pragma unroll
        for (int i = 1; i < 16; ++i) join(top, sum, part[i][in]);
    return make_float2(top, sum);
}

// The sum over the tiles of sums[tile * stride + row], in threads 0 .. kJoined - 1; row: of this thread, the same for all
// with its threadIdx.x % kJoined, or negative.
__device__ __forceinline__ float joined_sums(const float *sums, long long row, long long stride, int tiles, float (&part)[16][kJoined])
{
    const int in = threadIdx.x % kJoined, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float sum = 0.0f;
    if (row >= 0)
#pragma unroll 4
        for (int t = threadIdx.x / kJoined; t < tiles; t += 1024 / kJoined) sum += sums[t * stride + row];
#pragma unroll
    for (int other = kJoined; other < 64; other *= 2) sum += __shfl_xor(sum, other, 64);
    if (lane < kJoined) part[wave][in] = sum;
    __syncthreads();
    if (threadIdx.x >= kJoined) return sum;
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += part[i][in];
    return sum;
}

}  // namespace eager
