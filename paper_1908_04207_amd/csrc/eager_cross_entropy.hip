// Output projection and softmax cross entropy over the vocabulary, and their gradients.
//
//   l = x w^T,  lse = log sum exp(l),  loss = lse - l[target]
//   dl = dloss (exp(l - lse) - onehot(target)),  dx = dl w,  dw = dl^T x
//
// Forward: one product whose tiles leave the maximum and the sum of their part of the vocabulary
// for every row, then a small kernel over these.  Backward, for one piece of the vocabulary after
// the other: the piece's logits again, turned into dl in the product's epilogue and kept in the
// workspace; dx += dl w in fp32 sums (one per slice of the piece); dw = dl^T x of the piece.
//
// All products are one kernel.  Operand A is the side whose index runs within a lane's results
// (vocabulary for the logits, width for the gradients), B the side that the lane counts, so that
// softmax statistics stay within a lane and results are stored four values at a time.
#include "eager_matrix.h"
#include "eager_model.h"

namespace eager {
namespace {

// One side of a product: element (row, k).  Rows hold consecutive k, or (Columns) k rows hold
// consecutive rows.
struct Side {
    const void *data;
    long long stride;        // elements
    long long rows;
    long long k;             // values of k that are there; from here on k reads as zero
};

struct Product {
    Side a, b;
    int tiles_a, tiles_b, slices;
    int steps;               // k tiles of a slice

    // what becomes of it
    void *out;               // [b row][a row]
    long long out_stride;
    int accumulate;
    float2 *stats;           // [a tile][b row]: maximum, sum
    float *right;            // logit of the target
    const long long *target;
    const float *lse, *dloss;
    long long first;         // vocabulary index of a row 0
    int live;                // rows of a that are vocabulary (the rest is padding)
    int vocab;
};

enum Epilogue { kStats, kDlogits, kSums, kResult };

// Bytes of a tile: Rows * 128 whatever the layout (kDepth values of k are 128 bytes)
template <typename T> constexpr int kDepth = 128 / sizeof(T);

template <typename T, int Rows, bool Columns, int Waves>
__device__ __forceinline__ void stage_side(char *tile, const Side &s, long long row0, long long k0,
                                           int wave, int lane)
{
    constexpr int E = 16 / sizeof(T);
    const char *data = static_cast<const char *>(s.data);
    if (!Columns) {
        stage_rows<Rows, 8, Waves>(tile, data + (row0 * s.stride + k0) * sizeof(T), s.stride * sizeof(T),
                                   static_cast<int>(min(s.rows - row0, static_cast<long long>(Rows))),
                                   static_cast<int>(min((s.k - k0) / E, 8ll)), wave, lane);
    } else {
        constexpr int Chunks = Rows / E;
        const int rows_left = static_cast<int>(min(s.k - k0, static_cast<long long>(kDepth<T>)));
        const int chunks_left = static_cast<int>(min((s.rows - row0) / E, static_cast<long long>(Chunks)));
        const char *base = data + (k0 * s.stride + row0) * sizeof(T);
        const long long stride = s.stride * sizeof(T);
        const unsigned bytes = rows_left <= 0 || chunks_left <= 0 ? 0u
            : static_cast<unsigned>((rows_left - 1) * stride + chunks_left * 16);
        const __amdgpu_buffer_rsrc_t r = buffer(base, bytes);
#pragma unroll
        for (int i = 0; i < Rows * 8 / 64 / Waves; ++i) {
            const int piece = i * Waves + wave, id = piece * 64 + lane;
            const int row = id / Chunks, chunk = (id % Chunks) ^ (sizeof(T) == 2 ? (row & 3) << 2 : 0);
            load_lds16(r, tile + piece * 1024,
                       chunk < chunks_left ? static_cast<unsigned>(row * static_cast<unsigned>(stride)) + chunk * 16 : kOutside);
        }
    }
}

template <typename T, int Rows, bool Columns>
__device__ __forceinline__ typename Operand<T>::frag read_side(const char *tile, int row0, int step, int lane)
{
    if (!Columns) return read_rows<8>(tile, row0, step, lane, static_cast<T *>(nullptr));
    return read_columns<Rows * sizeof(T) / 16, sizeof(T) == 2 ? 2 : 31>(tile, row0, 16 * step, 8, 4, lane, static_cast<T *>(nullptr));
}

template <typename T, int BM, int BN, int WM, int WN, bool ColumnsA, bool ColumnsB, int Epi>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(const Product p)
{
    constexpr int Waves = WM * WN, MI = BM / WM / 32, NI = BN / WN / 32, Steps = kDepth<T> / 16;
    __shared__ __align__(1024) char tiles[2][(BM + BN) * 128];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile_b = blockIdx.x % p.tiles_b, rest = blockIdx.x / p.tiles_b;
    const int tile_a = rest % p.tiles_a, slice = rest / p.tiles_a;
    const long long a0 = static_cast<long long>(tile_a) * BM, b0 = static_cast<long long>(tile_b) * BN;
    const int wave_a = wave % WM * (BM / WM), wave_b = wave / WM * (BN / WN);
    const long long k_first = static_cast<long long>(slice) * p.steps * kDepth<T>;
    const long long k_last = min(max(p.a.k, p.b.k), k_first + static_cast<long long>(p.steps) * kDepth<T>);
    auto stage = [&](long long k0, int buf) {
        stage_side<T, BM, ColumnsA, Waves>(tiles[buf], p.a, a0, k0, wave, lane);
        stage_side<T, BN, ColumnsB, Waves>(tiles[buf] + BM * 128, p.b, b0, k0, wave, lane);
    };
    f32x16 c[MI][NI] = {};
    if (k_first < k_last) stage(k_first, 0);
    int buf = 0;
    for (long long k0 = k_first; k0 < k_last; k0 += kDepth<T>, buf ^= 1) {
        wait_loads();
        __syncthreads();
        if (k0 + kDepth<T> < k_last) stage(k0 + kDepth<T>, buf ^ 1);
#pragma unroll
        for (int s = 0; s < Steps; ++s) {
            typename Operand<T>::frag a[MI], b[NI];
#pragma unroll
            for (int i = 0; i < MI; ++i) a[i] = read_side<T, BM, ColumnsA>(tiles[buf], wave_a + 32 * i, s, lane);
#pragma unroll
            for (int j = 0; j < NI; ++j) b[j] = read_side<T, BN, ColumnsB>(tiles[buf] + BM * 128, wave_b + 32 * j, s, lane);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) c[i][j] = mma(a[i], b[j], c[i][j]);
        }
    }

    const int half = lane >> 5;
    if (Epi == kStats) {
        __syncthreads();
        float2 *parts = reinterpret_cast<float2 *>(tiles[0]);          // [WM][BN]
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const long long row = b0 + wave_b + 32 * j + (lane & 31);
            const long long target = row < p.b.rows ? p.target[row] : -1;
            float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const long long v = a0 + wave_a + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3);
                    if (v >= p.live) c[i][j][r] = -__builtin_inff();
                    else if (v == target) p.right[row] = c[i][j][r];
                    top = fmaxf(top, c[i][j][r]);
                }
            const float base = top == -__builtin_inff() ? 0.0f : top * kLog2e;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += exp2_fast(fmaf(c[i][j][r], kLog2e, -base));
            const float other = __shfl_xor(top, 32, 64), other_sum = __shfl_xor(sum, 32, 64);
            const float both = fmaxf(top, other);
            const float at = both == -__builtin_inff() ? 0.0f : both;
            sum = sum * exp2_fast((top - at) * kLog2e) + other_sum * exp2_fast((other - at) * kLog2e);
            if (half == 0) parts[wave % WM * BN + wave_b + 32 * j + lane] = make_float2(both, sum);
        }
        __syncthreads();
        for (int n = threadIdx.x; n < BN; n += 64 * Waves) {
            float2 all = parts[n];
#pragma unroll
            for (int i = 1; i < WM; ++i) {
                const float2 q = parts[i * BN + n];
                const float both = fmaxf(all.x, q.x), at = both == -__builtin_inff() ? 0.0f : both;
                all = make_float2(both, all.y * exp2_fast((all.x - at) * kLog2e) + q.y * exp2_fast((q.x - at) * kLog2e));
            }
            if (b0 + n < p.b.rows) p.stats[tile_a * p.b.rows + b0 + n] = all;
        }
        return;
    }
    typedef typename Operand<T>::quad quad;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const long long row = b0 + wave_b + 32 * j + (lane & 31);
        long long target = -1;
        float lse = 0.0f, g = 0.0f;
        if (Epi == kDlogits && row < p.b.rows) {
            target = p.target[row];
            lse = p.lse[row] * kLog2e;
            g = target < 0 ? 0.0f : target >= p.vocab ? __builtin_nanf("") : p.dloss[row];
            target -= p.first;
        }
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const long long at = a0 + wave_a + 32 * i + 8 * r + 4 * half;
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = c[i][j][4 * r + e];
                if (Epi == kDlogits) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float q = exp2_fast(fmaf(x[e], kLog2e, -lse)) - (at + e == target ? 1.0f : 0.0f);
                        x[e] = g == 0.0f || at + e >= p.live ? 0.0f : g * q;
                    }
                    *reinterpret_cast<quad *>(static_cast<T *>(p.out) + row * p.out_stride + at) = to_quad(x, static_cast<T *>(nullptr));
                } else if (row < (Epi == kResult ? p.live : p.b.rows) && at < p.a.rows) {
                    if (Epi == kSums) {
                        f32x4 *y = reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + (slice * p.b.rows + row) * p.out_stride + at);
                        if (p.accumulate) x += *y;
                        *y = x;
                    } else {
                        *reinterpret_cast<quad *>(static_cast<T *>(p.out) + row * p.out_stride + at) = to_quad(x, static_cast<T *>(nullptr));
                    }
                }
            }
    }
}

// loss and lse of 64 rows from the tiles' statistics: four wavefronts share the tiles
__global__ __launch_bounds__(256) void rows_kernel(const float2 *stats, const float *right, const long long *target,
                                                   float *loss, float *lse, long long rows, int tiles, int vocab)
{
    __shared__ float2 part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = static_cast<long long>(blockIdx.x) * 64 + lane;
    float top = -__builtin_inff(), sum = 0.0f;
    if (row < rows)
        for (int t = wave; t < tiles; t += 4) {
            const float2 q = stats[t * rows + row];
            const float both = fmaxf(top, q.x), at = both == -__builtin_inff() ? 0.0f : both;
            sum = sum * exp2_fast((top - at) * kLog2e) + q.y * exp2_fast((q.x - at) * kLog2e);
            top = both;
        }
    part[wave][lane] = make_float2(top, sum);
    __syncthreads();
    if (wave || row >= rows) return;
    for (int i = 1; i < 4; ++i) {
        const float2 q = part[i][lane];
        const float both = fmaxf(top, q.x), at = both == -__builtin_inff() ? 0.0f : both;
        sum = sum * exp2_fast((top - at) * kLog2e) + q.y * exp2_fast((q.x - at) * kLog2e);
        top = both;
    }
    const float all = fmaf(log2_fast(sum), kLn2, top);
    const long long t = target[row];
    lse[row] = all;
    loss[row] = t < 0 ? 0.0f : t >= vocab ? __builtin_nanf("") : all - right[row];
}

// dx from the slices' sums
template <typename T>
__global__ __launch_bounds__(256) void sums_kernel(const float *sums, T *dx, long long stride, long long rows, int width, int slices)
{
    const int quads = width / 4;
    const long long n = rows * quads, i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= n) return;
    f32x4 x = *reinterpret_cast<const f32x4 *>(sums + i * 4);
    for (int s = 1; s < slices; ++s) x += *reinterpret_cast<const f32x4 *>(sums + (s * n + i) * 4);
    *reinterpret_cast<typename Operand<T>::quad *>(dx + i / quads * stride + i % quads * 4) = to_quad(x, static_cast<T *>(nullptr));
}

constexpr int kTileA = 128, kTileB = 128;

long long round_up(long long x, long long to) { return (x + to - 1) / to * to; }

template <typename T, bool ColumnsA, bool ColumnsB, int Epi>
void multiply(Product p, hipStream_t stream)
{
    p.tiles_a = static_cast<int>(round_up(p.a.rows, kTileA) / kTileA);
    p.tiles_b = static_cast<int>(round_up(p.b.rows, kTileB) / kTileB);
    const long long steps = round_up(p.a.k > p.b.k ? p.a.k : p.b.k, kDepth<T>) / kDepth<T>;
    p.steps = static_cast<int>(round_up(steps, p.slices) / p.slices);
    const unsigned grid = static_cast<unsigned>(static_cast<long long>(p.tiles_a) * p.tiles_b * p.slices);
    hipLaunchKernelGGL((product_kernel<T, kTileA, kTileB, 2, 2, ColumnsA, ColumnsB, Epi>), dim3(grid), dim3(256), 0, stream, p);
}

// Vocabulary rows of a piece and slices of dx for a workspace of so many bytes (at most what
// cross_entropy_workspace_bytes asks for); 0 if it is too small.
struct Pieces {
    long long rows_padded, piece;
    int slices;
};

long long piece_of(long long rows, int vocab, int bytes)
{
    const long long rows_padded = round_up(rows > 0 ? rows : 1, kTileB), all = round_up(vocab, kTileA);
    const long long fit = (1ll << 28) / bytes / rows_padded / kTileA * kTileA;
    return fit < kTileA ? kTileA : fit < all ? fit : all;
}

template <typename T>
hipError_t forward(const CrossEntropyArgs &a, hipStream_t stream)
{
    Product p = {};
    p.a = {a.w, a.w_stride, a.vocab, a.width};
    p.b = {a.x, a.x_stride, a.rows, a.width};
    p.slices = 1;
    p.live = a.vocab;
    p.target = a.target;
    const long long tiles = round_up(a.vocab, kTileA) / kTileA;
    p.stats = reinterpret_cast<float2 *>(a.workspace);
    p.right = reinterpret_cast<float *>(p.stats + tiles * a.rows);
    multiply<T, false, false, kStats>(p, stream);
    hipLaunchKernelGGL(rows_kernel, dim3(static_cast<unsigned>((a.rows + 63) / 64)), dim3(256), 0, stream, p.stats, p.right,
                       a.target, a.loss, a.lse, a.rows, static_cast<int>(tiles), a.vocab);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const CrossEntropyArgs &a, hipStream_t stream)
{
    const long long rows_padded = round_up(a.rows, kTileB), piece = piece_of(a.rows, a.vocab, sizeof(T));
    const T *w = static_cast<const T *>(a.w);
    T *dl = reinterpret_cast<T *>(a.workspace);
    float *sums = reinterpret_cast<float *>(a.workspace + rows_padded * piece * sizeof(T));
    const int slices = 1;
    for (long long first = 0; first < a.vocab; first += piece) {
        const int live = static_cast<int>(a.vocab - first < piece ? a.vocab - first : piece);
        const long long padded = round_up(live, kTileA);
        Product p = {};
        if (a.rows) {
            p.a = {w + first * a.w_stride, a.w_stride, live, a.width};
            p.b = {a.x, a.x_stride, a.rows, a.width};
            p.vocab = a.vocab;
            p.slices = 1;
            p.first = first;
            p.live = live;
            p.target = a.target;
            p.lse = a.lse;
            p.dloss = a.dloss;
            p.out = dl;
            p.out_stride = padded;
            multiply<T, false, false, kDlogits>(p, stream);
        }
        if (a.dx && a.rows) {
            p = {};
            // dl is zero from `live` to `padded`, so its last chunk may be read whole
            p.a = {w + first * a.w_stride, a.w_stride, a.width, live};
            p.b = {dl, padded, a.rows, round_up(live, 16 / sizeof(T))};
            p.slices = slices;
            p.out = sums;
            p.out_stride = a.width;
            p.accumulate = first > 0;
            multiply<T, true, false, kSums>(p, stream);
        }
        if (a.dw) {
            p = {};
            p.a = {a.x, a.x_stride, a.width, a.rows};
            p.b = {dl, padded, padded, a.rows};
            p.slices = 1;
            p.live = live;
            p.out = static_cast<T *>(a.dw) + first * a.w_stride;
            p.out_stride = a.w_stride;
            multiply<T, true, true, kResult>(p, stream);
        }
    }
    if (a.dx && a.rows)
        hipLaunchKernelGGL((sums_kernel<T>), dim3(static_cast<unsigned>((a.rows * (a.width / 4) + 255) / 256)), dim3(256), 0, stream,
                           sums, static_cast<T *>(a.dx), a.x_stride, a.rows, a.width, slices);
    return hipGetLastError();
}

}  // namespace

long long cross_entropy_workspace_bytes(long long rows, int width, int vocab, bool bf16, bool backward)
{
    if (!backward) return round_up(rows * (round_up(vocab, kTileA) / kTileA * 8 + 4), 16) + 16;
    const int bytes = bf16 ? 2 : 4;
    return round_up(rows, kTileB) * piece_of(rows, vocab, bytes) * bytes + rows * width * 4 + 16;
}

hipError_t launch_cross_entropy(const CrossEntropyArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? forward<__bf16>(a, stream) : forward<float>(a, stream);
}

hipError_t launch_cross_entropy_backward(const CrossEntropyArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? backward<__bf16>(a, stream) : backward<float>(a, stream);
}

}  // namespace eager
