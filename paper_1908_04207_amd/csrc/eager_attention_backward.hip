// Gradients of causal attention over packed sequences.
//
//   P = exp(scale Q K^T - lse),  dP = dO V^T,  delta = rowsum(dO * O),  dS = P * (dP - delta)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Two kinds of workgroups, each with sums of its own in registers, so that no sum depends on their
// order: queries() goes over the keys for a tile of queries (dQ, and delta on the way),
// keys() over the queries for a tile of keys (dK, dV).  Both form P and dP again from the
// inputs, transposed to each other, so that the lane's side is the side that is summed for: 7
// products of 2 D operations an allowed pair where the formulas have 5.  Heads that share keys are
// summed by `parts` workgroups in fp32 and joined in the parts' order.  Batches of little work have
// both in one launch (gradients_kernel), the rows' delta then from a launch before it.
//
// With bf16 inputs P and dS are rounded to bf16 for the second products, whose other sides are bf16:
// the error is that of the formula's own operands.  Sums are fp32, and so are P and dS with fp32 inputs.
//
// Bound, heads of 64: what is open in the chain S -> P -> dP -> dS of a tile, with three wavefronts a SIMD in the queries' kernel and
// two in the keys' (vector instructions take 53 and 37 % of a unit's clocks, matrix instructions 35 and 33 %, 25 heads of
// 64) and, in short sequences, the last key tile's chain of all its queries.  Heads of 128 and fp32: one
// wavefront a SIMD in the keys' kernel (bf16 316 registers: two accumulators of 128 x 32), so waits of a
// tile's loads and of that chain are not covered by another wavefront; in fp32 with heads of 128 it keeps 132 bytes a
// lane in scratch memory.
// Measured: bf16, 16 heads (4 of keys) of 64, 16 sequences, 8192 tokens: 43 us dq, 49 us dk and dv, 12 us
// parts; 25 heads of 64, 8 sequences of 1024: 68 and 90 us (589 and 597 TFLOP/s, masked pairs not counted); 8
// heads (2) of 128, one of 16384: 833 and 1364 us (990 and 806 TFLOP/s); fp32, 16 heads (8) of 64, 9 sequences,
// 4099 tokens: 108 and 125 us.
//
// Slower, same sizes: both halves of a tile side by side with heads of 128 (registers spill: 4.8 ms), two tiles of queries
// a workgroup (dq 84 us instead of 52 in the first).
#include "eager_launch.h"
#include "eager_packed.h"

namespace eager {
namespace {

constexpr int kRows = kAttentionRows;        // queries (keys) of a workgroup: 32 a wavefront
constexpr int kTile = 64;            // keys (queries) of a tile
// How many halves of a tile are unrolled: with long heads two of them side by side do not fit the registers.
template <typename T, int DP> constexpr int kHalves = DP * sizeof(T) > 128 ? 1 : 2;

// Arrays of their own, so that the compiler knows a load into one apart from a read of another.
#define EAGER_TILES __shared__ __align__(1024) char tile0[kTile * DP * sizeof(T)]; \
                    __shared__ __align__(1024) char tile1[kTile * DP * sizeof(T)]; \
                    __shared__ __align__(1024) char tile2[kTile * DP * sizeof(T)]; \
                    __shared__ __align__(1024) char tile3[kTile * DP * sizeof(T)]
#define EAGER_ROWS  __shared__ __align__(1024) float rows0[2][kTile]; \
                    __shared__ __align__(1024) float rows1[2][kTile]

// dq of 128 rows of a head, id.  write: also leaves what keys() begins its sums with, for every row.
template <typename T, int DP>
__device__ __forceinline__ void queries(const AttentionArgs &a, int id, bool write, char *k_tile0, char *v_tile0, char *k_tile1, char *v_tile1)
{
    constexpr int Chunks = DP * sizeof(T) / 16, Steps = DP / 16;
    T *const type = nullptr;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = id % a.q_heads;
    const Tile t = find_tile<kRows>(a.cu, a.sequences, static_cast<int>(a.tokens), id / a.q_heads, false);
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
    decltype(operand(typename Operand<T>::frag())) q[Steps], g[Steps];
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < Steps; ++s) {
        const typename Operand<T>::frag x = row_operand(do_row, s, lane, a.dim, there), o = row_operand(o_row, s, lane, a.dim, there);
        q[s] = operand(row_operand(q_row, s, lane, a.dim, there));
        g[s] = operand(x);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = fmaf(static_cast<float>(x[j]), static_cast<float>(o[j]), delta);
    }
    delta = both_sum(delta);
    float lse = 0.0f;
    if (there) {
        lse = a.lse[head * a.tokens + row];
        if (lane < 32 && write) {
            a.delta[head * a.tokens + row] = -delta;
            a.start[head * a.tokens + row] = -lse / a.scale;
        }
        lse *= kLog2e;
    }

    const char *k_base = reinterpret_cast<const char *>(static_cast<const T *>(a.k.data) + kv_head * a.k.head);
    const char *v_base = reinterpret_cast<const char *>(static_cast<const T *>(a.v.data) + kv_head * a.v.head);
    const long long k_stride = a.k.row * sizeof(T), v_stride = a.v.row * sizeof(T);
    const int chunks = a.dim * sizeof(T) / 16;
    auto stage = [&](int key0, char *k_tile, char *v_tile) {
        stage_rows<kTile, Chunks, 4>(k_tile, k_base + key0 * k_stride, k_stride, t.end - key0, chunks, wave, lane);
        stage_rows<kTile, Chunks, 4>(v_tile, v_base + key0 * v_stride, v_stride, t.end - key0, chunks, wave, lane);
    };

    const float c = a.scale * kLog2e;
    const int last = min(t.end, t.first + kRows);
    f32x16 dq[DP / 32] = {};
    auto tile = [&](int key0, char *k_tile, char *v_tile, char *next_k, char *next_v) {
        wait_loads();
        __syncthreads();
        stage(key0 + kTile, next_k, next_v);            // beyond the sequence: zeros
#pragma unroll kHalves<T, DP>
        for (int b = 0; b < 2; ++b) {
            if (key0 + 32 * b >= wave_row + 32) continue;
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int i = 0; i < Steps; ++i) {
                s = mma(operand(read_rows<Chunks>(k_tile, 32 * b, i, lane, type)), q[i], s);
                dp = mma(operand(read_rows<Chunks>(v_tile, 32 * b, i, lane, type)), g[i], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = exp2_fast(fmaf(s[i], c, -lse));
            if (key0 + 32 * b + 31 > wave_row) {
                const int seen = row - key0 - 32 * b - 4 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (8 * (i >> 2) + (i & 3) > seen) s[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] *= dp[i] - delta;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto ds = operand(as_operand<T>(s, h));
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
                    dq[d] = mma(operand(read_columns<Chunks>(k_tile, 32 * d, 32 * b + 16 * h, 4, 8, lane, type)), ds, dq[d]);
            }
        }
    };
    stage(t.begin, k_tile0, v_tile0);
    for (int key0 = t.begin; key0 < last; key0 += 2 * kTile) {
        tile(key0, k_tile0, v_tile0, k_tile1, v_tile1);
        tile(key0 + kTile, k_tile1, v_tile1, k_tile0, v_tile0);
    }
    wait_loads();
    if (there) {
        T *y = static_cast<T *>(a.dq.data) + static_cast<long long>(row) * a.dq.row + head * a.dq.head;
        store_row<T, DP>(y, dq, a.scale, lane, a.dim);
    }
}

// The query heads that share a key head fall into `parts` parts, each with workgroups of its own:
// with few keys and heads there would be too few of them, and those of the first keys, which have
// the most queries, would run alone at the end.  With more than one part the sums of each go to the
// workspace in fp32 and parts_kernel adds them.
template <typename T, int DP>
__device__ __forceinline__ void keys(const AttentionArgs &a, int id, char *q_tile0, char *g_tile0, char *q_tile1, char *g_tile1,
                                     float (*rows0)[kTile], float (*rows1)[kTile])
{
    constexpr int Chunks = DP * sizeof(T) / 16, Steps = DP / 16;
    T *const type = nullptr;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shared = id % (a.kv_heads * a.parts), kv_head = shared / a.parts, part = shared % a.parts;
    const int heads = a.q_heads / a.kv_heads / a.parts;
    const Tile t = find_tile<kRows>(a.cu, a.sequences, static_cast<int>(a.tokens), id / (a.kv_heads * a.parts), true);
    if (t.first >= t.end) return;
    // where the sums go: [part][k, v][kv head][token][dim]
    float *const sums = a.sums + (static_cast<long long>(part) * 2 * a.kv_heads + kv_head) * a.tokens * a.dim;
    const long long to_v = static_cast<long long>(a.kv_heads) * a.tokens * a.dim;
    if (t.segment == 0 || t.segment == a.sequences + 1) {
        if (a.parts == 1) {
            clear_rows<T, kRows>(a.dk, kv_head, t.first, t.end, a.dim);
            clear_rows<T, kRows>(a.dv, kv_head, t.first, t.end, a.dim);
        } else {
            const Heads y = {sums, a.dim, 0}, z = {sums + to_v, a.dim, 0};
            clear_rows<float, kRows>(y, 0, t.first, t.end, a.dim);
            clear_rows<float, kRows>(z, 0, t.first, t.end, a.dim);
        }
        return;
    }
    const int wave_key = t.first + 32 * wave, key = wave_key + (lane & 31);
    const bool there = key < t.end;
    const T *k_row = static_cast<const T *>(a.k.data) + static_cast<long long>(key) * a.k.row + kv_head * a.k.head;
    const T *v_row = static_cast<const T *>(a.v.data) + static_cast<long long>(key) * a.v.row + kv_head * a.v.head;
    decltype(operand(typename Operand<T>::frag())) k[Steps], v[Steps];
#pragma unroll
    for (int s = 0; s < Steps; ++s) {
        k[s] = operand(row_operand(k_row, s, lane, a.dim, there));
        v[s] = operand(row_operand(v_row, s, lane, a.dim, there));
    }
    const long long q_stride = a.q.row * sizeof(T), g_stride = a.dout.row * sizeof(T);
    const int chunks = a.dim * sizeof(T) / 16;
    // tiles of queries of one head after the other
    int next_head = (kv_head * a.parts + part) * heads, next_row = t.first;
    const int last_head = next_head + heads;
    auto stage = [&](char *q_tile, char *g_tile, float (*rows)[kTile]) {
        const int left = next_head < last_head ? t.end - next_row : 0;
        const int head = min(next_head, last_head - 1);
        const char *q = reinterpret_cast<const char *>(static_cast<const T *>(a.q.data) + head * a.q.head) + next_row * q_stride;
        const char *g = reinterpret_cast<const char *>(static_cast<const T *>(a.dout.data) + head * a.dout.head) + next_row * g_stride;
        stage_rows<kTile, Chunks, 4>(q_tile, q, q_stride, left, chunks, wave, lane);
        stage_rows<kTile, Chunks, 4>(g_tile, g, g_stride, left, chunks, wave, lane);
        // -lse / scale and -delta; rows beyond the sequence: zeros, with which P = 1, but dO and dP - delta are zeros too
        const float *per_row = (wave & 1 ? a.delta : a.start) + head * a.tokens + next_row;
        if (wave < 2)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(per_row, min(kTile, left) * 4),
                                                     (__attribute__((address_space(3))) void *)(rows[wave]), 4,
                                                     lane * 4, 0, 0, 0);
        next_row += kTile;
        if (next_row >= t.end) {
            next_row = t.first;
            ++next_head;
        }
    };

    const float c = a.scale * kLog2e;
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    const int tiles_a_head = (t.end - t.first + kTile - 1) / kTile, count = heads * tiles_a_head;
    int row0 = t.first;
    auto tile = [&](char *q_tile, char *g_tile, float (*rows)[kTile], char *next_q, char *next_g, float (*next_rows)[kTile]) {
        wait_loads();
        __syncthreads();
        stage(next_q, next_g, next_rows);
#pragma unroll kHalves<T, DP>
        for (int b = 0; b < 2; ++b) {
            if (row0 + 32 * b + 31 < wave_key) continue;        // all queries come before the wavefront's keys
            // the sums begin with -lse / scale and -delta: P = exp(scale s), dS = P dp
            f32x16 s, dp;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = 32 * b + 8 * r + 4 * (lane >> 5);
                const f32x4 x = *reinterpret_cast<const f32x4 *>(&rows[0][at]), y = *reinterpret_cast<const f32x4 *>(&rows[1][at]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * r + i] = x[i], dp[4 * r + i] = y[i];
            }
#pragma unroll
            for (int i = 0; i < Steps; ++i) {
                s = mma(operand(read_rows<Chunks>(q_tile, 32 * b, i, lane, type)), k[i], s);
                dp = mma(operand(read_rows<Chunks>(g_tile, 32 * b, i, lane, type)), v[i], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = exp2_fast(s[i] * c);
            if (row0 + 32 * b < wave_key + 31) {
                const int seen = key - row0 - 32 * b - 4 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (8 * (i >> 2) + (i & 3) < seen) s[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) dp[i] *= s[i];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto p = operand(as_operand<T>(s, h)), ds = operand(as_operand<T>(dp, h));
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    dv[d] = mma(operand(read_columns<Chunks>(g_tile, 32 * d, 32 * b + 16 * h, 4, 8, lane, type)), p, dv[d]);
                    dk[d] = mma(operand(read_columns<Chunks>(q_tile, 32 * d, 32 * b + 16 * h, 4, 8, lane, type)), ds, dk[d]);
                }
            }
        }
        row0 += kTile;
        if (row0 >= t.end) row0 = t.first;
    };
    stage(q_tile0, g_tile0, rows0);
    int n = 0;
    for (; n + 1 < count; n += 2) {
        tile(q_tile0, g_tile0, rows0, q_tile1, g_tile1, rows1);
        tile(q_tile1, g_tile1, rows1, q_tile0, g_tile0, rows0);
    }
    if (n < count) tile(q_tile0, g_tile0, rows0, q_tile1, g_tile1, rows1);
    wait_loads();
    if (!there) return;
    if (a.parts == 1) {
        T *yk = static_cast<T *>(a.dk.data) + static_cast<long long>(key) * a.dk.row + kv_head * a.dk.head;
        T *yv = static_cast<T *>(a.dv.data) + static_cast<long long>(key) * a.dv.row + kv_head * a.dv.head;
        store_row<T, DP>(yk, dk, a.scale, lane, a.dim);
        store_row<T, DP>(yv, dv, 1.0f, lane, a.dim);
    } else {
        store_row<float, DP>(sums + static_cast<long long>(key) * a.dim, dk, a.scale, lane, a.dim);
        store_row<float, DP>(sums + to_v + static_cast<long long>(key) * a.dim, dv, 1.0f, lane, a.dim);
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1) void queries_kernel(const AttentionArgs a)
{
    EAGER_TILES;
    queries<T, DP>(a, blockIdx.x, true, tile0, tile1, tile2, tile3);
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 128 ? 2 : 1) void keys_kernel(const AttentionArgs a)
{
    EAGER_TILES;
    EAGER_ROWS;
    keys<T, DP>(a, blockIdx.x, tile0, tile1, tile2, tile3, rows0, rows1);
}

// Both in one launch, after rows_kernel has left what keys() wants of every row.
template <typename T, int DP>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 128 ? 2 : 1) void gradients_kernel(const AttentionArgs a, int of_keys)
{
    EAGER_TILES;
    EAGER_ROWS;
    const int id = blockIdx.x;
    if (id < of_keys) keys<T, DP>(a, id, tile0, tile1, tile2, tile3, rows0, rows1);
    else queries<T, DP>(a, id - of_keys, false, tile0, tile1, tile2, tile3);
}

// delta and lse of 32 rows of a head a wavefront, added in the order of queries()
template <typename T, int DP>
__global__ __launch_bounds__(256) void rows_kernel(const AttentionArgs a)
{
    const int lane = threadIdx.x & 63, head = blockIdx.x % a.q_heads;
    const long long row = static_cast<long long>(blockIdx.x / a.q_heads) * kRows + 32 * (threadIdx.x >> 6) + (lane & 31);
    const bool there = row < a.tokens;
    const T *do_row = static_cast<const T *>(a.dout.data) + row * a.dout.row + head * a.dout.head;
    const T *o_row = static_cast<const T *>(a.out.data) + row * a.out.row + head * a.out.head;
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const typename Operand<T>::frag g = row_operand(do_row, s, lane, a.dim, there), o = row_operand(o_row, s, lane, a.dim, there);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = fmaf(static_cast<float>(g[j]), static_cast<float>(o[j]), delta);
    }
    delta = both_sum(delta);
    if (there && lane < 32) {
        a.delta[head * a.tokens + row] = -delta;
        a.start[head * a.tokens + row] = -a.lse[head * a.tokens + row] / a.scale;
    }
}

// dk (blockIdx.y = 0) and dv (1) from the parts' sums, four values a thread, in the parts' order
template <typename T>
__global__ __launch_bounds__(256) void parts_kernel(const AttentionArgs a)
{
    const Heads &y = blockIdx.y ? a.dv : a.dk;
    const int quads = a.dim / 4;
    const long long of_head = a.tokens * quads, all = a.kv_heads * of_head;
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= all) return;
    const f32x4 *sums = reinterpret_cast<const f32x4 *>(a.sums) + blockIdx.y * all + i;
    f32x4 x = *sums;
    for (int part = 1; part < a.parts; ++part) x += sums[part * 2 * all];
    const long long head = i / of_head, in = i - head * of_head, token = in / quads;
    T *row = static_cast<T *>(y.data) + token * y.row + head * y.head;
    *reinterpret_cast<typename Operand<T>::quad *>(row + (in - token * quads) * 4) = to_quad(x, static_cast<T *>(nullptr));
}

template <typename T, int DP>
hipError_t enqueue(const AttentionArgs &a, hipStream_t stream)
{
    hipError_t e;
    const long long tiles = tile_numbers(a.tokens, a.sequences, kRows);
    const unsigned of_queries = static_cast<unsigned>(tiles * a.q_heads), of_keys = static_cast<unsigned>(tiles * a.kv_heads * a.parts);
    if (attention_together(tiles * a.q_heads, DP)) {
        const long long blocks = (a.tokens + kRows - 1) / kRows * a.q_heads;
        e = launch(rows_kernel<T, DP>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
        if (e == hipSuccess)
            e = launch(gradients_kernel<T, DP>, dim3(of_keys + of_queries), dim3(256), 0, stream, a, static_cast<int>(of_keys));
    } else {
        e = launch(queries_kernel<T, DP>, dim3(of_queries), dim3(256), 0, stream, a);
        if (e == hipSuccess) e = launch(keys_kernel<T, DP>, dim3(of_keys), dim3(256), 0, stream, a);
    }
    if (e != hipSuccess || a.parts == 1) return e;
    const long long quads = a.tokens * a.kv_heads * (a.dim / 4);
    return launch(parts_kernel<T>, dim3(static_cast<unsigned>((quads + 255) / 256), 2), dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_attention_backward(const AttentionArgs &a, bool bf16, hipStream_t stream)
{
    if (bf16) return a.dim <= 64 ? enqueue<__bf16, 64>(a, stream) : enqueue<__bf16, 128>(a, stream);
    return a.dim <= 64 ? enqueue<float, 64>(a, stream) : enqueue<float, 128>(a, stream);
}

}  // namespace eager
