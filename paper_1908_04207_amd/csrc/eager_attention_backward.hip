// Gradients of causal attention over packed sequences.
//
//   P = exp(scale Q K^T - lse),  dP = dO V^T,  delta = rowsum(dO * O),  dS = P * (dP - delta)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Two kernels, each with sums of its own in registers, so that no sum depends on the order of
// workgroups: queries_kernel goes over the keys for a tile of queries (dQ, and delta on the way),
// keys_kernel over the queries for a tile of keys (dK, dV).  Both form P and dP again from the
// inputs, transposed to each other, so that the lane's side is the side that is summed for.
#include "eager_packed.h"

namespace eager {
namespace {

constexpr int kRows = 128;           // queries (keys) of a workgroup: 32 a wavefront
constexpr int kTile = 64;            // keys (queries) of a tile

template <typename T, int DP>
__global__ __launch_bounds__(256) void queries_kernel(const AttentionArgs a)
{
    constexpr int Chunks = DP * sizeof(T) / 16, TileBytes = kTile * Chunks * 16, Steps = DP / 16;
    __shared__ __align__(1024) char tiles[2][2][TileBytes];
    T *const type = nullptr;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % a.q_heads;
    const Tile t = find_tile<kRows>(a.cu, a.sequences, static_cast<int>(a.tokens),
                                    (gridDim.x - 1 - blockIdx.x) / a.q_heads);
    if (t.first >= t.end) return;
    if (t.segment == 0 || t.segment == a.sequences + 1) {
        clear_rows<T, kRows>(a.dq, head, t.first, t.end, a.dim);
        return;
    }
    const int kv_head = head / (a.q_heads / a.kv_heads);
    const int wave_row = t.first + 32 * wave, row = wave_row + (lane & 31);
    const bool there = row < t.end;
    const T *q_row = static_cast<const T *>(a.q.data) + static_cast<long long>(row) * a.q.row + head * a.q.head;
    const T *do_row = static_cast<const T *>(a.dout.data) + static_cast<long long>(row) * a.dout.row + head * a.dout.head;
    const T *o_row = static_cast<const T *>(a.out.data) + static_cast<long long>(row) * a.out.row + head * a.out.head;
    typename Operand<T>::frag q[Steps], g[Steps];
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < Steps; ++s) {
        q[s] = row_operand(q_row, s, lane, a.dim, there);
        g[s] = row_operand(do_row, s, lane, a.dim, there);
        const typename Operand<T>::frag o = row_operand(o_row, s, lane, a.dim, there);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = fmaf(static_cast<float>(g[s][j]), static_cast<float>(o[j]), delta);
    }
    delta += __shfl_xor(delta, 32, 64);
    float lse = 0.0f;
    if (there) {
        lse = a.lse[head * a.tokens + row] * kLog2e;
        if (lane < 32) a.delta[head * a.tokens + row] = delta;
    }

    const char *k_base = reinterpret_cast<const char *>(static_cast<const T *>(a.k.data) + kv_head * a.k.head);
    const char *v_base = reinterpret_cast<const char *>(static_cast<const T *>(a.v.data) + kv_head * a.v.head);
    const long long k_stride = a.k.row * sizeof(T), v_stride = a.v.row * sizeof(T);
    const int chunks = a.dim * sizeof(T) / 16;
    auto stage = [&](int key0, int buf) {
        stage_rows<kTile, Chunks, 4>(tiles[buf][0], k_base + key0 * k_stride, k_stride, t.end - key0, chunks, wave, lane);
        stage_rows<kTile, Chunks, 4>(tiles[buf][1], v_base + key0 * v_stride, v_stride, t.end - key0, chunks, wave, lane);
    };

    const float c = a.scale * kLog2e;
    const int last = min(t.end, t.first + kRows);
    f32x16 dq[DP / 32] = {};
    stage(t.begin, 0);
    for (int key0 = t.begin, buf = 0; key0 < last; key0 += kTile, buf ^= 1) {
        wait_loads();
        __syncthreads();
        if (key0 + kTile < last) stage(key0 + kTile, buf ^ 1);
        const bool diagonal = key0 + kTile - 1 > wave_row;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (key0 + 32 * b >= wave_row + 32) continue;
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int i = 0; i < Steps; ++i) {
                s = mma(read_rows<Chunks>(tiles[buf][0], 32 * b, i, lane, type), q[i], s);
                dp = mma(read_rows<Chunks>(tiles[buf][1], 32 * b, i, lane, type), g[i], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float p = exp2_fast(fmaf(s[i], c, -lse));
                if (diagonal && key0 + 32 * b + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) > row) p = 0.0f;
                s[i] = p * (dp[i] - delta);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const typename Operand<T>::frag ds = as_operand<T>(s, h);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
                    dq[d] = mma(read_columns<Chunks>(tiles[buf][0], 32 * d, 32 * b + 16 * h, 4, 8, lane, type), ds, dq[d]);
            }
        }
    }
    if (there) {
        T *y = static_cast<T *>(a.dq.data) + static_cast<long long>(row) * a.dq.row + head * a.dq.head;
        store_row<T, DP>(y, dq, a.scale, lane, a.dim);
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void keys_kernel(const AttentionArgs a)
{
    constexpr int Chunks = DP * sizeof(T) / 16, TileBytes = kTile * Chunks * 16, Steps = DP / 16;
    __shared__ __align__(1024) char tiles[2][2][TileBytes];
    __shared__ __align__(1024) float rows[2][2][kTile];
    T *const type = nullptr;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv_head = blockIdx.x % a.kv_heads, group = a.q_heads / a.kv_heads;
    const Tile t = find_tile<kRows>(a.cu, a.sequences, static_cast<int>(a.tokens), blockIdx.x / a.kv_heads);
    if (t.first >= t.end) return;
    if (t.segment == 0 || t.segment == a.sequences + 1) {
        clear_rows<T, kRows>(a.dk, kv_head, t.first, t.end, a.dim);
        clear_rows<T, kRows>(a.dv, kv_head, t.first, t.end, a.dim);
        return;
    }
    const int wave_key = t.first + 32 * wave, key = wave_key + (lane & 31);
    const bool there = key < t.end;
    const T *k_row = static_cast<const T *>(a.k.data) + static_cast<long long>(key) * a.k.row + kv_head * a.k.head;
    const T *v_row = static_cast<const T *>(a.v.data) + static_cast<long long>(key) * a.v.row + kv_head * a.v.head;
    typename Operand<T>::frag k[Steps], v[Steps];
#pragma unroll
    for (int s = 0; s < Steps; ++s) {
        k[s] = row_operand(k_row, s, lane, a.dim, there);
        v[s] = row_operand(v_row, s, lane, a.dim, there);
    }
    const long long q_stride = a.q.row * sizeof(T), g_stride = a.dout.row * sizeof(T);
    const int chunks = a.dim * sizeof(T) / 16;
    const int first_row = t.first;                      // a multiple of kTile rows from the sequence's first
    const int tiles_a_head = (t.end - first_row + kTile - 1) / kTile;
    auto stage = [&](int n, int buf) {
        const int head = kv_head * group + n / tiles_a_head, row0 = first_row + n % tiles_a_head * kTile;
        const char *q = reinterpret_cast<const char *>(static_cast<const T *>(a.q.data) + head * a.q.head) + row0 * q_stride;
        const char *g = reinterpret_cast<const char *>(static_cast<const T *>(a.dout.data) + head * a.dout.head) + row0 * g_stride;
        stage_rows<kTile, Chunks, 4>(tiles[buf][0], q, q_stride, t.end - row0, chunks, wave, lane);
        stage_rows<kTile, Chunks, 4>(tiles[buf][1], g, g_stride, t.end - row0, chunks, wave, lane);
        // rows beyond the sequence: zeros, with which P = 1, but dO and dP - delta are zeros too
        const float *per_row = (wave & 1 ? a.delta : a.lse) + head * a.tokens + row0;
        if (wave < 2)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(per_row, min(kTile, t.end - row0) * 4),
                                                     (__attribute__((address_space(3))) void *)(rows[buf][wave]), 4,
                                                     lane * 4, 0, 0, 0);
    };

    const float c = a.scale * kLog2e;
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    const int count = group * tiles_a_head;
    stage(0, 0);
    for (int n = 0, buf = 0; n < count; ++n, buf ^= 1) {
        const int row0 = first_row + n % tiles_a_head * kTile;
        wait_loads();
        __syncthreads();
        if (n + 1 < count) stage(n + 1, buf ^ 1);
        const bool diagonal = row0 < wave_key + 31;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (row0 + 32 * b + 31 < wave_key) continue;        // all rows come before the wavefront's keys
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int i = 0; i < Steps; ++i) {
                s = mma(read_rows<Chunks>(tiles[buf][0], 32 * b, i, lane, type), k[i], s);
                dp = mma(read_rows<Chunks>(tiles[buf][1], 32 * b, i, lane, type), v[i], dp);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = 32 * b + 8 * r + 4 * (lane >> 5);
                const f32x4 lse = *reinterpret_cast<const f32x4 *>(&rows[buf][0][at]);
                const f32x4 delta = *reinterpret_cast<const f32x4 *>(&rows[buf][1][at]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float p = exp2_fast(fmaf(s[4 * r + i], c, -lse[i] * kLog2e));
                    if (diagonal && key > row0 + at + i) p = 0.0f;
                    s[4 * r + i] = p;
                    dp[4 * r + i] = p * (dp[4 * r + i] - delta[i]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const typename Operand<T>::frag p = as_operand<T>(s, h), ds = as_operand<T>(dp, h);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    dv[d] = mma(read_columns<Chunks>(tiles[buf][1], 32 * d, 32 * b + 16 * h, 4, 8, lane, type), p, dv[d]);
                    dk[d] = mma(read_columns<Chunks>(tiles[buf][0], 32 * d, 32 * b + 16 * h, 4, 8, lane, type), ds, dk[d]);
                }
            }
        }
    }
    if (there) {
        T *yk = static_cast<T *>(a.dk.data) + static_cast<long long>(key) * a.dk.row + kv_head * a.dk.head;
        T *yv = static_cast<T *>(a.dv.data) + static_cast<long long>(key) * a.dv.row + kv_head * a.dv.head;
        store_row<T, DP>(yk, dk, a.scale, lane, a.dim);
        store_row<T, DP>(yv, dv, 1.0f, lane, a.dim);
    }
}

template <typename T, int DP>
void enqueue(const AttentionArgs &a, hipStream_t stream)
{
    const long long tiles = tile_numbers(a.tokens, a.sequences, kRows);
    hipLaunchKernelGGL((queries_kernel<T, DP>), dim3(static_cast<unsigned>(tiles * a.q_heads)), dim3(256), 0, stream, a);
    hipLaunchKernelGGL((keys_kernel<T, DP>), dim3(static_cast<unsigned>(tiles * a.kv_heads)), dim3(256), 0, stream, a);
}

}  // namespace

long long attention_workspace_bytes(long long tokens, int q_heads)
{
    return (tokens * q_heads * 4 + 15) / 16 * 16;
}

hipError_t launch_attention_backward(const AttentionArgs &a, bool bf16, hipStream_t stream)
{
    if (bf16 && a.dim <= 64) enqueue<__bf16, 64>(a, stream);
    else if (bf16) enqueue<__bf16, 128>(a, stream);
    else if (a.dim <= 64) enqueue<float, 64>(a, stream);
    else enqueue<float, 128>(a, stream);
    return hipGetLastError();
}

}  // namespace eager
