// RMS norm of every query and key head with a gain, then the rotation by position, and the
// gradients of both.
//
//   n = r x,  r = (mean(x^2) + eps)^(-1/2),  u = w n,  y = R(position) u
//   du = R^T dy,  dw = sum over rows of du n,  dn = w du,  dx = r (dn - n mean(dn n))
//
// A head of D values belongs to a group of lanes, each with V consecutive values of the first half
// and the V of the second half that they are rotated with, so the rotation needs no exchange and
// the two means are one butterfly over the group.
//
// Bound by memory: forward reads x and writes y once, backward reads x and dy and writes dx; 1/r is formed again from
// x, which is read anyway.  Means, norms and gains' sums are fp32.  Measured: fp32, 20011 tokens of 50 heads of 64
// (256 MB an array): forward 93 us (5.5 TB/s), backward 165 us (4.7 TB/s of three arrays) and 7 us for the gains' sums;
// bf16, 8192 tokens of 20 heads of 64 (21 MB, which the last cache holds): 11.4, 16.5 and 4.1 us; 37 tokens: 4.8 us, a launch.
#include "eager_launch.h"
#include "eager_matrix.h"
#include "eager_model.h"

namespace eager {
namespace {

template <typename T, int V> struct Piece;
template <> struct Piece<__bf16, 8> { typedef bf16x8 type; };
template <> struct Piece<__bf16, 4> { typedef bf16x4 type; };
template <> struct Piece<float, 4> { typedef f32x4 type; };

template <typename T, int V>
__device__ __forceinline__ void load(const T *p, float *x)
{
    const typename Piece<T, V>::type v = *reinterpret_cast<const typename Piece<T, V>::type *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = static_cast<float>(v[i]);
}

template <typename T, int V>
__device__ __forceinline__ void store(T *p, const float *x)
{
    typename Piece<T, V>::type v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = static_cast<T>(x[i]);
    *reinterpret_cast<typename Piece<T, V>::type *>(p) = v;
}

template <int V>
__device__ __forceinline__ void load_table(const float *p, float *x)
{
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + i);
        x[i] = v[0], x[i + 1] = v[1], x[i + 2] = v[2], x[i + 3] = v[3];
    }
}

template <int G>
__device__ __forceinline__ float group_sum(float x)
{
#pragma unroll
    for (int m = 1; m < G; m *= 2) x += __shfl_xor(x, m, 64);
    return x;
}

// cosines and sines of a token's lane; NaN where the position is outside the table
template <int V>
__device__ __forceinline__ void rotation(const NormRopeArgs &a, long long token, int at, float *c, float *s)
{
    const int pos = a.positions[token];
    if (pos >= 0 && pos < a.table_rows) {
        const long long o = static_cast<long long>(pos) * (a.dim >> 1) + at;
        load_table<V>(a.cos_table + o, c);
        load_table<V>(a.sin_table + o, s);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = s[i] = __builtin_nanf("");
    }
}

// G lanes a head (a power of two, dim / 2 <= G * V); a workgroup takes per_block tokens.
template <typename T, int V, int G>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormRopeArgs a)
{
    const int half = a.dim >> 1, at = (threadIdx.x % G) * V;
    const bool in = at < half;
    const int heads = a.heads[0] + a.heads[1];
    const long long t0 = static_cast<long long>(blockIdx.x) * a.per_block;
    const int items = static_cast<int>(min(static_cast<long long>(a.per_block), a.tokens - t0)) * heads;
    for (int item = threadIdx.x / G; item < items; item += 256 / G) {
        const int t = item / heads, h = item - t * heads;
        const int which = h >= a.heads[0];
        const long long token = t0 + t, head = which ? h - a.heads[0] : h;
        const T *x = static_cast<const T *>(a.x[which].data) + token * a.x[which].row + head * a.x[which].head + at;
        T *y = static_cast<T *>(a.y[which].data) + token * a.y[which].row + head * a.y[which].head + at;
        float p[V], q[V], c[V], s[V], wp[V], wq[V], sum = 0.0f;
        if (in) {
            load<T, V>(x, p);
            load<T, V>(x + half, q);
#pragma unroll
            for (int i = 0; i < V; ++i) sum = fmaf(p[i], p[i], fmaf(q[i], q[i], sum));
        }
        sum = group_sum<G>(sum);
        if (!in) continue;
        rotation<V>(a, token, at, c, s);
        const T *w = static_cast<const T *>(a.w[which]) + at;
        load<T, V>(w, wp);
        load<T, V>(w + half, wq);
        const float r = rsqrtf(fmaf(sum, a.inv_dim, a.eps));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float u = p[i] * r * wp[i], v = q[i] * r * wq[i];
            p[i] = fmaf(u, c[i], -(v * s[i]));
            q[i] = fmaf(v, c[i], u * s[i]);
        }
        store<T, V>(y, p);
        store<T, V>(y + half, q);
    }
}

// y holds the gradients of the outputs.  A lane sees the same columns of every head it takes, so the
// gains' gradients stay in its registers until the end; the lanes of a workgroup that share columns
// are added in shared memory in a fixed order, and the workgroups by the kernel after this one.
template <typename T, int V, int G>
__global__ __launch_bounds__(256) void norm_rope_backward_kernel(const NormRopeArgs a)
{
    __shared__ float part[256 / G][2 * V * G];
    const int half = a.dim >> 1, lane = threadIdx.x % G, at = lane * V;
    const bool in = at < half;
    float *out = a.partials + static_cast<long long>(blockIdx.x) * 2 * a.dim;
    for (int which = 0; which < 2; ++which) {
        const int heads = a.heads[which];
        float wp[V], wq[V], gp[V], gq[V];
#pragma unroll
        for (int i = 0; i < V; ++i) wp[i] = wq[i] = gp[i] = gq[i] = 0.0f;
        if (in) {
            load<T, V>(static_cast<const T *>(a.w[which]) + at, wp);
            load<T, V>(static_cast<const T *>(a.w[which]) + at + half, wq);
        }
        for (long long t0 = static_cast<long long>(blockIdx.x) * a.per_block; t0 < a.tokens;
             t0 += static_cast<long long>(a.blocks) * a.per_block) {
            const int items = static_cast<int>(min(static_cast<long long>(a.per_block), a.tokens - t0)) * heads;
            for (int item = threadIdx.x / G; item < items; item += 256 / G) {
                const int t = item / heads;
                const long long token = t0 + t, head = item - t * heads;
                const Heads &vx = a.x[which], &vy = a.y[which], &vd = a.dx[which];
                float p[V], q[V], dp[V], dq[V], c[V], s[V], sum = 0.0f, dot = 0.0f;
                if (in) {
                    const T *x = static_cast<const T *>(vx.data) + token * vx.row + head * vx.head + at;
                    const T *y = static_cast<const T *>(vy.data) + token * vy.row + head * vy.head + at;
                    load<T, V>(x, p);
                    load<T, V>(x + half, q);
                    load<T, V>(y, dp);
                    load<T, V>(y + half, dq);
                    rotation<V>(a, token, at, c, s);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        sum = fmaf(p[i], p[i], fmaf(q[i], q[i], sum));
                        const float u = fmaf(dp[i], c[i], dq[i] * s[i]), v = fmaf(dq[i], c[i], -(dp[i] * s[i]));
                        dp[i] = u, dq[i] = v;
                        dot = fmaf(u * wp[i], p[i], fmaf(v * wq[i], q[i], dot));
                    }
                }
                sum = group_sum<G>(sum);
                dot = group_sum<G>(dot);
                if (!in) continue;
                const float r = rsqrtf(fmaf(sum, a.inv_dim, a.eps));
                const float back = dot * a.inv_dim * r * r;         // mean(dn n) / r * r
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    gp[i] = fmaf(dp[i] * r, p[i], gp[i]);
                    gq[i] = fmaf(dq[i] * r, q[i], gq[i]);
                    p[i] = r * fmaf(-p[i], back, dp[i] * wp[i]);
                    q[i] = r * fmaf(-q[i], back, dq[i] * wq[i]);
                }
                T *d = static_cast<T *>(vd.data) + token * vd.row + head * vd.head + at;
                store<T, V>(d, p);
                store<T, V>(d + half, q);
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            part[threadIdx.x / G][lane * V + i] = gp[i];
            part[threadIdx.x / G][G * V + lane * V + i] = gq[i];
        }
        __syncthreads();
        if (threadIdx.x < a.dim) {
            const int col = threadIdx.x < half ? threadIdx.x : G * V + threadIdx.x - half;
            float sum = 0.0f;
            for (int g = 0; g < 256 / G; ++g) sum += part[g][col];
            out[which * a.dim + threadIdx.x] = sum;
        }
        __syncthreads();
    }
}

// The workgroups' records of 16 columns of one gain (blockIdx.y): 64 sums over every 64th record, then
// these in order.
template <typename T>
__global__ __launch_bounds__(1024) void norm_rope_gains_kernel(const NormRopeArgs a)
{
    __shared__ float part[64][17];
    const int in = threadIdx.x % 16, col = blockIdx.x * 16 + in, slice = threadIdx.x / 16;
    float sum = 0.0f;
    if (col < a.dim) {
        const float *p = a.partials + blockIdx.y * a.dim + col;
#pragma unroll 8
        for (int b = slice; b < a.blocks; b += 64) sum += p[static_cast<long long>(b) * 2 * a.dim];
    }
    part[slice][in] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && col < a.dim) {
#pragma unroll 8
        for (int i = 1; i < 64; ++i) sum += part[i][in];
        static_cast<T *>(a.dw[blockIdx.y])[col] = static_cast<T>(sum);
    }
}

template <typename T, int V, int G>
hipError_t enqueue(const NormRopeArgs &a, bool backward, hipStream_t stream)
{
    if (!backward) {
        const long long blocks = (a.tokens + a.per_block - 1) / a.per_block;
        return launch(norm_rope_kernel<T, V, G>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
    }
    hipError_t e = hipSuccess;
    if (a.blocks) e = launch(norm_rope_backward_kernel<T, V, G>, dim3(a.blocks), dim3(256), 0, stream, a);
    return e != hipSuccess ? e : launch(norm_rope_gains_kernel<T>, dim3((a.dim + 15) / 16, 2), dim3(1024), 0, stream, a);
}

// Lanes of 8 values need halves of a multiple of 8 (16-byte accesses in bf16); other head sizes take 4.
hipError_t dispatch(const NormRopeArgs &a, bool bf16, bool backward, hipStream_t stream)
{
    const int half = a.dim / 2;
    if (bf16 && half % 8 == 0) {
        if (half <= 8) return enqueue<__bf16, 8, 1>(a, backward, stream);
        if (half <= 16) return enqueue<__bf16, 8, 2>(a, backward, stream);
        if (half <= 32) return enqueue<__bf16, 8, 4>(a, backward, stream);
        return enqueue<__bf16, 8, 8>(a, backward, stream);
    }
    if (bf16) {
        if (half <= 16) return enqueue<__bf16, 4, 4>(a, backward, stream);
        return enqueue<__bf16, 4, 16>(a, backward, stream);
    }
    if (half <= 16) return enqueue<float, 4, 4>(a, backward, stream);
    if (half <= 32) return enqueue<float, 4, 8>(a, backward, stream);
    return enqueue<float, 4, 16>(a, backward, stream);
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs &a, bool bf16, hipStream_t stream)
{
    return dispatch(a, bf16, false, stream);
}

hipError_t launch_norm_rope_backward(const NormRopeArgs &a, bool bf16, hipStream_t stream)
{
    return dispatch(a, bf16, true, stream);
}

}  // namespace eager
