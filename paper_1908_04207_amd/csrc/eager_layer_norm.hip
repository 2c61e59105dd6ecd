// Residual sum and layer norm of rows of hidden states, and their gradients.
//
//   s = x + residual (as stored),  m = mean(s),  r = (mean((s - m)^2) + eps)^(-1/2),  n = (s - m) r,  y = n w + b
//   dn = dy w,  dx = ds + r (dn - mean(dn) - n mean(dn n)),  dw = sum over rows of dy n,  db = sum of dy
//
// A row is held by a group of lanes, 16 values each, from its first read to its last write: the mean, then the
// squares around it.  What the mean is off by goes into every value and into the squares, so its sum is formed in 64
// bits, and s - m with the mean's fp32 value and what that leaves: a row of one value gives zeros, and a row far from zero
// what the same row next to zero gives.  (With the sum in fp32 1600 values around 1e4 of deviation one were 8e-4 off and a row of
// 1234.567 had r = 315.99 for 316.23; the sum in 64 bits costs 65536 x 64 in bf16 9.2 us for 8.3, 8192 x 1024 12.9 for 12.4, fp32
// rows nothing.)  Squares are summed in fp32.  The backward pass takes m, rounded to fp32, and r from the forward pass; its
// workgroups go through rows at equal steps and keep the sums of dw and db in registers; the groups of a workgroup are added
// in shared memory in order, the workgroups by a second kernel.
//
// Bound by memory, every array once.  Measured (x, residual, s, y forward; dy, ds, s, dx backward): 20011 x 1600 fp32 (128 MB
// an array) forward 91 us (5.6 TB/s), backward 107 and 4.9 for the sums over rows; 8192 x 1024 bf16 (17 MB, which the last
// cache holds) 13.4, 13.5 and 3.8 us; 2047 x 8192 bf16 (x, y; dy, s, dx) 14.5, 19.8 and 4.0 us; 37 x 1024 forward 4.5 us, a launch.
#include "eager_launch.h"
#include "eager_model.h"
#include "eager_model_rules.h"
#include "eager_vector.h"

namespace eager {
namespace {

// Sums over a group, in each of its lanes.  Groups of more than a wavefront meet in `part`, of which there are two for
// calls in turn, so one barrier a call is enough.
template <int Lanes, typename S>
__device__ __forceinline__ S each_sum(S x) { return lanes_sum<Lanes>(x); }
template <int Lanes>
__device__ __forceinline__ float2 each_sum(float2 x) { return make_float2(lanes_sum<Lanes>(x.x), lanes_sum<Lanes>(x.y)); }

template <int Threads, typename S>
__device__ __forceinline__ S group_sums(S x, S *part)
{
    constexpr int Waves = Threads / 64;
    x = each_sum<(Threads < 64 ? Threads : 64)>(x);
    if (Waves <= 1) return x;
    const int wave = threadIdx.x >> 6, first = wave / (Waves > 0 ? Waves : 1) * Waves;
    if ((threadIdx.x & 63) == 0) part[wave] = x;
    __syncthreads();
    x = part[first];
#pragma unroll
    for (int i = 1; i < Waves; ++i) x += part[first + i];
    return x;
}

// The sum of 16 bytes' values in 64 bits.
template <int E>
__device__ __forceinline__ double chunk_sum(const float (&x)[E])
{
    double sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = E == 8 ? static_cast<double>(x[i]) + x[E - 4 + i] : static_cast<double>(x[i]);
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// Which of a workgroup's groups; a scalar where a wavefront belongs to one, and so are the addresses of its row then.
template <int Threads>
__device__ __forceinline__ int group_of()
{
    const int group = threadIdx.x / Threads;
    return Threads < 64 ? group : __builtin_amdgcn_readfirstlane(group);
}

template <int Threads> constexpr int kBlock = Threads < 256 ? 256 : Threads;
template <int Threads> constexpr int kBackwardBlock = Threads < kNormBackwardBlock ? kNormBackwardBlock : Threads;

template <typename T, int Threads, int C>
__global__ __launch_bounds__(kBlock<Threads>) void layer_norm_kernel(const LayerNormArgs a)
{
    constexpr int E = kVector<T>, Groups = kBlock<Threads> / Threads;
    __shared__ double sums[16];
    __shared__ float part[16];
    const int lane = threadIdx.x % Threads, group = group_of<Threads>();
    const double width = a.width, inv_width = 1.0 / width;
    // as many turns for every group of the workgroup
    for (long long first = static_cast<long long>(blockIdx.x) * Groups; first < a.rows; first += static_cast<long long>(gridDim.x) * Groups) {
        const long long row = first + group;
        const bool live = row < a.rows;
        float x[C][E];
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * Threads + lane) * E;
#pragma unroll
            for (int i = 0; i < E; ++i) x[c][i] = 0.0f;
            if (!live || at >= a.width) continue;
            const auto v = load16(static_cast<const T *>(a.x.data) + row * a.x.stride + at);
#pragma unroll
            for (int i = 0; i < E; ++i) x[c][i] = static_cast<float>(v[i]);
            if (a.residual.data) {
                const auto u = load16(static_cast<const T *>(a.residual.data) + row * a.residual.stride + at);
#pragma unroll
                for (int i = 0; i < E; ++i) x[c][i] = static_cast<float>(static_cast<T>(x[c][i] + static_cast<float>(u[i])));
                store16(static_cast<T *>(a.sum.data) + row * a.sum.stride + at, x[c]);
            }
            sum += chunk_sum(x[c]);
        }
        sum = group_sums<Threads>(sum, sums);
        // the quotient, with what its first rounding leaves: of width times a number it is that number
        double exact = sum * inv_width;
        exact = fma(fma(-exact, width, sum), inv_width, exact);
        const float mean = static_cast<float>(exact), rest = static_cast<float>(exact - mean);
        float squares = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if ((c * Threads + lane) * E >= a.width) continue;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                x[c][i] = x[c][i] - mean - rest;
                squares = fmaf(x[c][i], x[c][i], squares);
            }
        }
        squares = group_sums<Threads>(squares, part);
        if (!live) continue;
        const float r = rsqrtf(fmaf(squares, a.inv_width, a.eps));
        if (lane == 0) a.stats[row] = mean, a.stats[a.rows + row] = r;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * Threads + lane) * E;
            if (at >= a.width) continue;
            const auto w = load16(static_cast<const T *>(a.w) + at);
            if (a.b) {
                const auto b = load16(static_cast<const T *>(a.b) + at);
#pragma unroll
                for (int i = 0; i < E; ++i) x[c][i] = fmaf(x[c][i] * r, static_cast<float>(w[i]), static_cast<float>(b[i]));
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) x[c][i] = x[c][i] * r * static_cast<float>(w[i]);
            }
            store16(static_cast<T *>(a.y.data) + row * a.y.stride + at, x[c]);
        }
    }
}

// a.x: s, a.y: dy, a.residual: ds, a.sum: dx
template <typename T, int Threads, int C>
__global__ __launch_bounds__(kBackwardBlock<Threads>) void layer_norm_backward_kernel(const LayerNormArgs a)
{
    constexpr int E = kVector<T>, Block = kBackwardBlock<Threads>, Groups = Block / Threads;
    typedef typename Vector<T>::type vec;
    __shared__ float2 part[2][16];
    __shared__ __align__(16) float sums[Groups > 1 ? Groups : 1][Groups > 1 ? Threads * C * E : 4];
    const int lane = threadIdx.x % Threads, group = group_of<Threads>();
    // Where a row takes 1024 lanes their registers do not hold all of it: the sums of dw and db stand in shared memory, the
    // gain is read again for every row, and in fp32 the next row is not under way while one is worked on.
    constexpr bool Held = Threads == 1024, Ahead = !Held || sizeof(T) == 2;
    __shared__ f32x4 held[Held ? 2 : 1][Held ? C * E / 4 : 1][Held ? Threads : 1];
    vec w[C] = {}, s[C], g[C], d[C];
    float gain[C][E], bias[C][E], next_mean, next_r;
    auto fetch = [&](long long row) {
        next_mean = row < a.rows ? a.stats[row] : 0.0f;
        next_r = row < a.rows ? a.stats[a.rows + row] : 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * Threads + lane) * E;
            s[c] = g[c] = d[c] = vec{};
            if (row >= a.rows || at >= a.width) continue;
            s[c] = load16(static_cast<const T *>(a.x.data) + row * a.x.stride + at);
            g[c] = load16(static_cast<const T *>(a.y.data) + row * a.y.stride + at);
            if (a.residual.data) d[c] = load16(static_cast<const T *>(a.residual.data) + row * a.residual.stride + at);
        }
    };
    const long long step = static_cast<long long>(gridDim.x) * Groups;
    long long row = static_cast<long long>(blockIdx.x) * Groups + group;
    if (Ahead) fetch(row);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * Threads + lane) * E;
        if (!Held && at < a.width) w[c] = load16(static_cast<const T *>(a.w) + at);
#pragma unroll
        for (int i = 0; i < E; ++i) gain[c][i] = bias[c][i] = 0.0f;
        if (Held)
            for (int i = 0; i < E / 4; ++i) held[0][c * E / 4 + i][lane] = held[1][c * E / 4 + i][lane] = f32x4{};
    }
    int turn = 0;
    // as many turns for every group of the workgroup
    for (long long first = static_cast<long long>(blockIdx.x) * Groups; first < a.rows; first += step, row += step, turn ^= 1) {
        const bool live = row < a.rows;
        if (!Ahead) fetch(row);
        const float mean = next_mean, r = next_r;
        float n[C][E], dn[C][E];
        vec rest[C];
        float2 both = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            rest[c] = d[c];
            if (Held && (c * Threads + lane) * E < a.width) w[c] = load16(static_cast<const T *>(a.w) + (c * Threads + lane) * E);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float dy = static_cast<float>(g[c][i]);
                n[c][i] = (static_cast<float>(s[c][i]) - mean) * r;
                dn[c][i] = dy * static_cast<float>(w[c][i]);
                both.x += dn[c][i];
                both.y = fmaf(dn[c][i], n[c][i], both.y);
                if (Held) continue;
                gain[c][i] = fmaf(dy, n[c][i], gain[c][i]);
                bias[c][i] += dy;
            }
            if (Held)
#pragma unroll
                for (int i = 0; i < E / 4; ++i) {
                    f32x4 u = held[0][c * E / 4 + i][lane], v = held[1][c * E / 4 + i][lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float dy = static_cast<float>(g[c][4 * i + e]);
                        u[e] = fmaf(dy, n[c][4 * i + e], u[e]);
                        v[e] += dy;
                    }
                    held[0][c * E / 4 + i][lane] = u;
                    held[1][c * E / 4 + i][lane] = v;
                }
        }
        if (Ahead) fetch(row + step);
        both = group_sums<Threads>(both, part[turn]);
        if (!live) continue;
        const float even = both.x * a.inv_width, along = both.y * a.inv_width;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * Threads + lane) * E;
            if (at >= a.width) continue;
#pragma unroll
            for (int i = 0; i < E; ++i) n[c][i] = fmaf(r, fmaf(-n[c][i], along, dn[c][i] - even), static_cast<float>(rest[c][i]));
            store16(static_cast<T *>(a.sum.data) + row * a.sum.stride + at, n[c]);
        }
    }
    if (!a.dw && !a.db) return;
    float *out = a.partials + static_cast<long long>(blockIdx.x) * 2 * a.width;
    T *const to[2] = {static_cast<T *>(a.dw), static_cast<T *>(a.db)};
    const bool alone = gridDim.x == 1;                   // its sums are those of all rows
    if (Groups > 1) {
        // one sum after the other, so that shared memory holds those of all groups
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which) __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < E; i += 4) {
                    const float *x = (which ? bias[c] : gain[c]) + i;
                    *reinterpret_cast<f32x4 *>(&sums[group][(c * Threads + lane) * E + i]) = f32x4{x[0], x[1], x[2], x[3]};
                }
            __syncthreads();
            for (int at = threadIdx.x; at < a.width; at += Block) {
                float sum = sums[0][at];
#pragma unroll
                for (int g = 1; g < Groups; ++g) sum += sums[g][at];
                if (!alone) out[which * a.width + at] = sum;
                else if (to[which]) to[which][at] = static_cast<T>(sum);
            }
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * Threads + lane) * E;
        if (at >= a.width) continue;
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const f32x4 u = {gain[c][i], gain[c][i + 1], gain[c][i + 2], gain[c][i + 3]};
            const f32x4 v = {bias[c][i], bias[c][i + 1], bias[c][i + 2], bias[c][i + 3]};
            const f32x4 sum[2] = {Held ? held[0][(c * E + i) / 4][lane] : u, Held ? held[1][(c * E + i) / 4][lane] : v};
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                if (!alone) *reinterpret_cast<f32x4 *>(out + which * a.width + at + i) = sum[which];
                else if (to[which])
#pragma unroll
                    for (int e = 0; e < 4; ++e) to[which][at + i + e] = static_cast<T>(sum[which][e]);
            }
        }
    }
}

// The workgroups' records of 16 Q columns of dw (blockIdx.y = 0) or db: 64 sums over every 64th record, then these in
// order.
template <typename T, int Q>
__global__ __launch_bounds__(1024) void layer_norm_columns_kernel(const LayerNormArgs a)
{
    typedef float vec __attribute__((ext_vector_type(Q)));
    __shared__ float part[64][16 * Q + 1];
    T *const to = static_cast<T *>(blockIdx.y ? a.db : a.dw);
    if (!to) return;
    const int in = threadIdx.x % 16 * Q, first = blockIdx.x * 16 * Q, slice = threadIdx.x / 16;
    vec sum = {};
    if (first + in < a.width) {
        const float *p = a.partials + blockIdx.y * a.width + first + in;
#pragma unroll 4
        for (int b = slice; b < a.blocks; b += 64) sum += *reinterpret_cast<const vec *>(p + static_cast<long long>(b) * 2 * a.width);
    }
#pragma unroll
    for (int i = 0; i < Q; ++i) part[slice][in + i] = sum[i];
    __syncthreads();
    if (threadIdx.x < 16 * Q && first + threadIdx.x < a.width) {
        float all = part[0][threadIdx.x];
#pragma unroll 8
        for (int i = 1; i < 64; ++i) all += part[i][threadIdx.x];
        to[first + threadIdx.x] = static_cast<T>(all);
    }
}

template <typename T, int Threads, int C>
hipError_t enqueue(const LayerNormArgs &a, bool backward, hipStream_t stream)
{
    constexpr int Groups = kBlock<Threads> / Threads;
    if (!backward)
        return launch(layer_norm_kernel<T, Threads, C>, dim3(static_cast<unsigned>(std::min((a.rows + Groups - 1) / Groups, kNormBlocks))),
                      dim3(kBlock<Threads>), 0, stream, a);
    hipError_t e = hipSuccess;
    if (a.blocks) e = launch(layer_norm_backward_kernel<T, Threads, C>, dim3(a.blocks), dim3(kBackwardBlock<Threads>), 0, stream, a);
    if (e != hipSuccess || (!a.dw && !a.db) || a.blocks == 1) return e;
    // One column a thread or four: wide rows' records are more than a few loads of 4 bytes a thread bring, narrow ones leave too few
    // workgroups of four.  Backward, bf16, us, one and four: 8192 x 264 9.4 and 9.7, 520 12.2 and 12.5, 1024 14.9 and 14.8, 1600 20.0
    // and 20.0; 4096 x 2040 16.8 and 16.2, 2048 16.5 and 16.5, 3000 21.2 and 20.3; 2047 x 8192 27.6 and 24.7, 300 x 8192 20.7 and 16.6.
    if (a.width < 2048) return launch(layer_norm_columns_kernel<T, 1>, dim3((a.width + 15) / 16, a.db ? 2 : 1), dim3(1024), 0, stream, a);
    return launch(layer_norm_columns_kernel<T, 4>, dim3((a.width + 63) / 64, a.db ? 2 : 1), dim3(1024), 0, stream, a);
}

template <typename T>
hipError_t dispatch(const LayerNormArgs &a, bool backward, hipStream_t stream)
{
    constexpr int C = 16 / kVector<T>;                      // 16 values a lane
    const int threads = layer_norm_threads(a.width);
    // Half as many values a lane where they hold the row, so that no lane of 16 or 64 is without any at half the width.  Measured,
    // 8 values and 16, forward and backward, us: 65536 x 64 bf16 7.8 and 8.2, 12.1 and 14.1, x 128 8.9 and 9.2, 14.8 and 15.9; 8192 x 264
    // 5.5 and 5.7, 9.4 and 10.4, x 512 6.0 and 6.1, 10.2 and 11.2; 16384 x 512 fp32 12.6 and 12.7, 20.7 and 21.6.
    if (threads == 16)
        return a.width <= 128 ? enqueue<T, 16, C / 2>(a, backward, stream) : enqueue<T, 16, C>(a, backward, stream);
    if (threads == 64)
        return a.width <= 512 ? enqueue<T, 64, C / 2>(a, backward, stream) : enqueue<T, 64, C>(a, backward, stream);
    if (threads == 128) return enqueue<T, 128, C>(a, backward, stream);
    if (threads == 256) return enqueue<T, 256, C>(a, backward, stream);
    if (threads == 512) return enqueue<T, 512, C>(a, backward, stream);
    return enqueue<T, 1024, C>(a, backward, stream);
}

}  // namespace

hipError_t launch_layer_norm(const LayerNormArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? dispatch<__bf16>(a, false, stream) : dispatch<float>(a, false, stream);
}

hipError_t launch_layer_norm_backward(const LayerNormArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? dispatch<__bf16>(a, true, stream) : dispatch<float>(a, true, stream);
}

}  // namespace eager
