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
//
// Statistics and the sums of dx and dw are fp32; dl is rounded to the inputs' type, since it is the operand of
// two products whose other side has that type.  fp32 products are six bf16 ones of operands cut into three bf16
// pieces of 8 bits each: a bf16 instruction has 16 times the rate of the fp32 one, so six cost less than one.
//
// Bound by the matrix instructions, busy 54 to 58 % of the time; what they wait for is the barrier between
// tiles and, in the last round, tiles that do not fill the card.  Measured (rows x width x vocabulary): 4096 x 1024 x 50257
// bf16 forward 457 us (923 TFLOP/s), backward with a tenth of the rows masked: dl 439 us and 6 for the targets' entries, dx and dw
// 815 us (931 TFLOP/s of the rows that count); 8191 x 1600 x 50257 forward 1157 us (1139 TFLOP/s), two pieces of dl 602 and of dx and dw 1306 us
// (957 with 5 % masked); fp32 1019 x 1024 x 50257: 639, 652, 1176 us (164 TFLOP/s forward, 160 dx and dw; 36 to 56 bytes a
// lane in scratch memory with tiles of 256 x 256); 61 x 1024 x 50257
// forward 19.4 us, 5.3 TB/s of the projection.
//
// Slower: the compiler's own order of matrix instructions and reads (10 to 15 %, see spread()), 4 wavefronts of 256 x 256
// (8 %), wavefronts of raised priority (no effect).
#include "eager_distillation.h"
#include "eager_gather.h"
#include "eager_joined.h"
#include "eager_launch.h"
#include "eager_matrix.h"
#include "eager_model.h"
#include "eager_model_rules.h"

#include <type_traits>

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
    int steps, all_steps;    // k tiles of a slice, of the product

    // what becomes of it
    void *out;               // [b row][a row]
    long long out_stride;
    int accumulate;
    float2 *stats;           // [a tile][b row]: maximum (as a power of two), sum
    float *right;            // logit of the target
    const long long *target;
    const float *lse, *dloss;
    float scale;             // of the logits in exponents of two: log2(e) / temperature
    long long first;         // vocabulary index of a row 0
    int live;                // rows of a that are vocabulary (the rest is padding)
    int vocab;
    int whole;               // one tile of a holds the vocabulary
    float *others;           // [a tile][b row]: sums of p without the target's, or NULL
    const int *counted;      // device: rows of x that count (gather_kernel), or NULL: all of them
    int counted_k;           // they are k, not the rows of b
    long long low;           // bytes from dl to what its rounding left, where that is kept
    const float *common;     // factor that dl leaves out and its products put in
};

// kKept: kStats, and the logits too.  kShared: kDlogits without the factor p.common.  kParted: kDlogits in two pieces, what
// rounding leaves of each in the second
enum Epilogue { kStats, kKept, kDlogits, kShared, kParted, kSums, kResult };
// dl as the gradients' products find it
enum Form { kPlain, kFactored, kTwice };

constexpr bool gives_statistics(int epilogue) { return epilogue == kStats || epilogue == kKept; }
constexpr bool gives_dlogits(int epilogue) { return epilogue == kDlogits || epilogue == kShared || epilogue == kParted; }

// A tile of one side has Rows * 128 bytes whatever the layout: kDepth values of k are 128 bytes.
template <typename T> constexpr int kDepth = 128 / sizeof(T);

// Tile after tile of one side into shared memory.  A lane's chunk is the same in each of its
// loads, whose rows are row_step bytes apart; what lies beyond the operand reads as zeros.
template <typename T, int Rows, bool Columns, int Waves>
struct Source {
    static constexpr int E = 16 / sizeof(T), Chunks = Columns ? Rows / E : 8, Loads = Rows / 8 / Waves;
    static_assert(Rows % (8 * Waves) == 0 && (Waves * 64 / Chunks % 4 == 0 || sizeof(T) == 4), "whole loads");
    const char *base;
    long long bytes, advance;
    unsigned offset, row_step;
    int chunk, chunks_left, wave;

    __device__ __forceinline__ Source(const Side &s, long long row0, long long k0, int wave, int lane) : wave(wave)
    {
        const long long stride = s.stride * sizeof(T);
        const int id = wave * 64 + lane, row = id / Chunks;
        row_step = static_cast<unsigned>(Waves * 64 / Chunks * stride);
        if (Columns) {
            base = static_cast<const char *>(s.data) + k0 * stride + row0 * sizeof(T);
            const long long there = min((s.rows - row0) / E, static_cast<long long>(Chunks));
            bytes = (s.k - k0 - 1) * stride + there * 16;
            advance = kDepth<T> * stride;
            chunk = (id % Chunks) ^ (sizeof(T) == 2 ? (row & 3) << 2 : 0);
            offset = chunk < there ? static_cast<unsigned>(row * stride) + chunk * 16 : kOutside;
        } else {
            base = static_cast<const char *>(s.data) + row0 * stride + k0 * sizeof(T);
            bytes = (min(s.rows - row0, static_cast<long long>(Rows)) - 1) * stride + (s.k - k0) * sizeof(T);
            advance = 128;
            chunk = (id % 8) ^ exchange<8>(row);
            chunks_left = static_cast<int>((s.k - k0) / E);
            offset = static_cast<unsigned>(row * stride) + chunk * 16;
        }
    }

    // the next tile; zeros instead where !live
    __device__ __forceinline__ void load(char *tile, bool live)
    {
        const __amdgpu_buffer_rsrc_t r = buffer(base, covered(live ? bytes : 0));
        const unsigned at = Columns || chunk < chunks_left ? offset : kOutside;
#pragma unroll
        for (int i = 0; i < Loads; ++i) load_lds16(r, tile + (i * Waves + wave) * 1024, at + i * row_step);
        base += advance;
        bytes -= advance;
        if (!Columns) chunks_left -= 8;
    }

    // from the first of the last `tiles` on once more, `far` bytes away
    __device__ __forceinline__ void again(int tiles, long long far)
    {
        base += far - tiles * advance;
        bytes += tiles * advance;
        if (!Columns) chunks_left += 8 * tiles;
    }
};

template <typename T, int Rows, bool Columns>
__device__ __forceinline__ typename Operand<T>::frag read_side(const char *tile, int row0, int step, int lane)
{
    if constexpr (!Columns) return read_rows<8>(tile, row0, step, lane, static_cast<T *>(nullptr));
    else return read_columns<Rows * sizeof(T) / 16, sizeof(T) == 2 ? 2 : kNoExchange>(tile, row0, 16 * step, 8, 4, lane, static_cast<T *>(nullptr));
}

// Workgroups id, id + 8, ... run on the same chiplet (one second-level cache): which of `all` pieces of work
// workgroup `id` takes, so that each chiplet has a contiguous share.
__device__ __forceinline__ int in_order(int id, int all)
{
    const int chiplet = id & 7, share = all >> 3, rest = all & 7;
    return chiplet * share + min(chiplet, rest) + (id >> 3);
}

// Tile n: 8 tiles of b are gone through for every tile of a.
__device__ __forceinline__ void place(int n, int tiles_a, int tiles_b, int &tile_a, int &tile_b)
{
    constexpr int Group = 8;
    const int group = n / (Group * tiles_a), first = group * Group, width = min(Group, tiles_b - first);
    const int in = n - group * Group * tiles_a;
    tile_b = first + in % width;
    tile_a = in / width;
}

// One workgroup computes BM x BN results with WM x WN wavefronts.  Two tiles in shared memory take
// turns: while one is multiplied, the next is on its way into the other.  A step's operands are
// read while the step before is multiplied, the first step's of a tile during the last one of the
// tile before, so the barrier between tiles stands in the shadow of matrix instructions.
template <typename T, typename Shape, bool ColumnsA, bool ColumnsB, int Epi, int Form = kPlain>
__device__ __forceinline__ void product(const Product &p, int tile_a, int tile_b, int slice, char *tile0, char *tile1)
{
    constexpr int BM = Shape::A, BN = Shape::B, WM = Shape::WavesA, WN = Shape::WavesB;
    constexpr int Waves = WM * WN, MI = BM / WM / 32, NI = BN / WN / 32, Steps = kDepth<T> / 16;
    typedef typename Operand<T>::frag frag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long a0 = static_cast<long long>(tile_a) * BM, b0 = static_cast<long long>(tile_b) * BN;
    const int wave_a = wave % WM * (BM / WM), wave_b = wave / WM * (BN / WN);
    Side a_side = p.a, b_side = p.b;
    int all_steps = p.all_steps;
    if (!gives_statistics(Epi)) {
        const int counted = *p.counted;
        if (p.counted_k) {
            a_side.k = b_side.k = counted;
            all_steps = (counted + kDepth<T> - 1) / kDepth<T>;
        } else {
            b_side.rows = counted;
            if (b0 >= counted) return;
        }
    }
    const int first = slice * p.steps;
    const int once = max(0, min(p.steps, all_steps - first)), count = Form == kTwice ? 2 * once : once;
    const long long k0 = static_cast<long long>(first) * kDepth<T>;
    Source<T, BM, ColumnsA, Waves> side_a(a_side, a0, k0, wave, lane);
    Source<T, BN, ColumnsB, Waves> side_b(b_side, b0, k0, wave, lane);
    auto stage = [&](char *tile, int t) {
        if (Form == kTwice && t == once) {                             // b's second pieces
            side_a.again(once, 0);
            side_b.again(once, p.low);
        }
        side_a.load(tile, t < count);
        side_b.load(tile + BM * 128, t < count);
    };
    f32x16 c[MI][NI] = {};
    frag a[2][MI], b[2][NI];
    auto read = [&](const char *tile, int step, int set) {
#pragma unroll
        for (int i = 0; i < MI; ++i) a[set][i] = read_side<T, BM, ColumnsA>(tile, wave_a + 32 * i, step, lane);
#pragma unroll
        for (int j = 0; j < NI; ++j) b[set][j] = read_side<T, BN, ColumnsB>(tile + BM * 128, wave_b + 32 * j, step, lane);
    };
    // of a step: reads of shared memory, among the first three quarters of its matrix instructions, and loads, among all (spread)
    constexpr int Reads = MI * (ColumnsA ? 2 : 1) + NI * (ColumnsB ? 2 : 1), Products = MI * NI;
    constexpr int Loads = (BM + BN) / 8 / Waves;
    auto body = [&](char *here, char *next, int t) {
#pragma unroll
        for (int s = 0; s < Steps; ++s) {
            if (s + 1 < Steps) {
                read(here, s + 1, (s + 1) & 1);
            } else {
                wait_loads();
                __syncthreads();
                stage(here, t + 2);
                read(next, 0, 0);
            }
            decltype(operand(frag())) right[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) right[j] = operand(b[s & 1][j]);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const auto left = operand(a[s & 1][i]);
#pragma unroll
                for (int j = 0; j < NI; ++j) c[i][j] = mma(left, right[j], c[i][j]);
            }
            if constexpr (sizeof(T) == 2) {
                if (s + 1 < Steps) spread<Products, Reads, 0>();
                else spread<Products, Reads, Loads>();
            }
        }
    };
    static_assert(Steps % 2 == 0, "a tile ends with the operand registers it began with");
    stage(tile0, 0);
    wait_loads();
    __syncthreads();
    stage(tile1, 1);
    read(tile0, 0, 0);
    int t = 0;
    for (; t + 1 < count; t += 2) {
        body(tile0, tile1, t);
        body(tile1, tile0, t + 1);
    }
    if (t < count) body(tile0, tile1, t);
    // the last step has asked for zeros beyond the product, in either tile: every wavefront's are there
    // before an epilogue writes into the tiles
    wait_loads();
    __syncthreads();

    const int half = lane >> 5;
    if (gives_statistics(Epi)) {
        if (Epi == kKept) {
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const long long row = b0 + wave_b + 32 * j + (lane & 31), from = a0 + wave_a + 4 * half;
                float *const to = static_cast<float *>(p.out) + row * p.out_stride + from;
                const int left = row < p.b.rows ? static_cast<int>(min(p.live - from, static_cast<long long>(BM))) : 0;
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        f32x4 x;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = c[i][j][4 * r + e];
                        if (32 * i + 8 * r < left) *reinterpret_cast<f32x4 *>(to + 32 * i + 8 * r) = x;
                    }
            }
        }
        float2 *parts = reinterpret_cast<float2 *>(tile0);             // [WM][BN]
        const int live = static_cast<int>(min(p.live - a0, static_cast<long long>(BM))) - wave_a - 4 * half;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const long long row = b0 + wave_b + 32 * j + (lane & 31);
            const long long target = Epi == kStats && row < p.b.rows ? p.target[row] : -1;
            // the target's place among the lane's results, if it has it
            const long long from = target - a0 - wave_a - 4 * half;
            const int at = from >= 0 && from < min(live, 32 * MI) ? static_cast<int>(from) : -1;
            float top = -__builtin_inff(), sum = 0.0f, right = 0.0f;
            // few wavefronts hold a target or the end of the vocabulary
            if (__any(at >= 0)) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * i + 8 * (r >> 2) + (r & 3) == at) right = c[i][j][r];
                if (at >= 0 && (at & 4) == 0) p.right[row] = right;
            }
            auto reduce = [&](auto whole) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (whole || 32 * i + 8 * (r >> 2) + (r & 3) < live) top = fmaxf(top, c[i][j][r]);
                // in powers of two from here on: what rounding leaves of top * scale stays in the exponents
                top *= p.scale;
                const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float e = exp2_fast(fmaf(c[i][j][r], p.scale, -base));
                        if (whole || 32 * i + 8 * (r >> 2) + (r & 3) < live) sum += e;
                    }
            };
            if (__all(live >= 32 * MI)) reduce(std::true_type());
            else reduce(std::false_type());
            const float other = __shfl_xor(top, 32, 64), other_sum = __shfl_xor(sum, 32, 64);
            const float both = fmaxf(top, other);
            const float zero = both == -__builtin_inff() ? 0.0f : both;
            sum = sum * exp2_fast(top - zero) + other_sum * exp2_fast(other - zero);
            if (half == 0) parts[wave % WM * BN + wave_b + 32 * j + lane] = make_float2(both, sum);
        }
        __syncthreads();
        for (int n = threadIdx.x; n < BN; n += 64 * Waves) {
            float2 all = parts[n];
#pragma unroll
            for (int i = 1; i < WM; ++i) {
                const float2 q = parts[i * BN + n];
                const float both = fmaxf(all.x, q.x), zero = both == -__builtin_inff() ? 0.0f : both;
                all = make_float2(both, all.y * exp2_fast(all.x - zero) + q.y * exp2_fast(q.x - zero));
            }
            if (b0 + n < p.b.rows) p.stats[tile_a * p.b.rows + b0 + n] = all;
        }
        return;
    }
    typedef typename Operand<T>::quad quad;
    T *const type = nullptr;
    // bf16 results cross shared memory, so that stores are whole cache lines; a row of BM results is
    // BM / 8 chunks, exchanged among themselves against bank conflicts
    constexpr bool Across = sizeof(T) == 2 && Epi != kSums;
    constexpr int RowChunks = BM / 8, RowsOfTile0 = (BM + BN) * 128 / (BM * 2);
    static_assert(!Across || BN <= 2 * RowsOfTile0, "results fit the tiles");
    auto place_of = [&](int row, int chunk) {
        char *tile = row < RowsOfTile0 ? tile0 + row * BM * 2 : tile1 + (row - RowsOfTile0) * BM * 2;
        return tile + (chunk ^ (row & (RowChunks - 1) & 31)) * 16;
    };
    const int live = static_cast<int>(min(p.live - a0, static_cast<long long>(BM)));
    const long long rows = Epi == kResult ? p.live : b_side.rows;
    if constexpr (gives_dlogits(Epi)) {
        float g[NI], others[NI], scale[NI];
        int target[NI];
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const long long row = b0 + wave_b + 32 * j + (lane & 31);
            float lse = __builtin_inff();               // rows that there are not: zeros
            g[j] = 0.0f, others[j] = -1.0f, scale[j] = 1.0f, target[j] = -1;
            if (row < rows) {
                const long long v = p.target[row], from = v - p.first - a0;
                lse = p.lse[row] * kLog2e;
                g[j] = v >= p.vocab ? __builtin_nanf("") : p.dloss[row];
                if (Epi == kShared) g[j] /= *p.common;
                target[j] = from >= wave_a && from < wave_a + 32 * MI ? static_cast<int>(from) : -1;
            }
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) c[i][j][r] = exp2_fast(fmaf(c[i][j][r], p.scale, -lse));
            if (__any(live < wave_a + 32 * MI)) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (wave_a + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3) >= live) c[i][j][r] = 0.0f;
            }
        }
        // 1 - p of the target as the sum of the others: lse in fp32 is up to 2^-24 of itself off, too much for rows
        // whose p is close to 1.  With the whole vocabulary in one tile p is normalised anew as well; with more tiles
        // each leaves its sum and targets_kernel puts the target's entry in.
        if (p.others) {
            float *parts = reinterpret_cast<float *>(tile0);           // [WM][BN]
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                float sum = 0.0f;
                if (__any(target[j] >= 0)) {
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            sum += wave_a + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3) == target[j] ? 0.0f : c[i][j][r];
                } else {
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum += c[i][j][r];
                }
                sum += __shfl_xor(sum, 32, 64);
                if (half == 0) parts[wave % WM * BN + wave_b + 32 * j + lane] = sum;
            }
            __syncthreads();
            for (int n = threadIdx.x; n < BN && b0 + n < rows; n += 64 * Waves) {
                float all = 0.0f;
#pragma unroll
                for (int i = 0; i < WM; ++i) all += parts[i * BN + n];
                p.others[tile_a * p.b.rows + b0 + n] = all;
            }
            __syncthreads();
        } else if (p.whole) {
            float2 *parts = reinterpret_cast<float2 *>(tile0);         // [WM][BN]: others, target
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                float sum = 0.0f, its = 0.0f;
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool hit = wave_a + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3) == target[j];
                        sum += hit ? 0.0f : c[i][j][r];
                        its += hit ? c[i][j][r] : 0.0f;
                    }
                sum += __shfl_xor(sum, 32, 64);
                its += __shfl_xor(its, 32, 64);
                if (half == 0) parts[wave % WM * BN + wave_b + 32 * j + lane] = make_float2(sum, its);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                float2 all = {};
#pragma unroll
                for (int i = 0; i < WM; ++i) {
                    const float2 q = parts[i * BN + wave_b + 32 * j + (lane & 31)];
                    all.x += q.x, all.y += q.y;
                }
                others[j] = -all.x;
                scale[j] = 1.0f / (all.x + all.y);
                if (g[j] == 0.0f) scale[j] = 0.0f;      // rows that there are not
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            if (__any(target[j] >= 0)) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (wave_a + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3) == target[j])
                            c[i][j][r] = p.whole ? others[j] : c[i][j][r] - 1.0f;
            }
            const float by = g[j] * scale[j];
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) c[i][j][r] *= by;
        }
    }
    if (Epi == kResult && Form == kFactored) {
        const float by = *p.common;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i) c[i][j] *= by;
    }
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int in_b = wave_b + 32 * j + (lane & 31);
        const long long row = b0 + in_b;
        const long long from = a0 + wave_a + 4 * half;
        const int limit = gives_dlogits(Epi) ? BM : row < rows ? static_cast<int>(min(p.a.rows - from, static_cast<long long>(BM))) : 0;
        float *const sums = static_cast<float *>(p.out) + (slice * p.b.rows + row) * p.out_stride + from;
        T *const out = static_cast<T *>(p.out) + row * p.out_stride + from;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = 32 * i + 8 * r;
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = c[i][j][4 * r + e];
                if (Across) {
                    *reinterpret_cast<quad *>(place_of(in_b, (wave_a + at) >> 3) + 8 * half) = to_quad(x, type);
                } else if (at < limit) {
                    if (Epi == kSums) {
                        if (p.accumulate) x += *reinterpret_cast<const f32x4 *>(sums + at);
                        *reinterpret_cast<f32x4 *>(sums + at) = x;
                    } else {
                        *reinterpret_cast<quad *>(out + at) = to_quad(x, type);
                    }
                }
            }
    }
    auto store_across = [&](char *to) {
        __syncthreads();
#pragma unroll 4
        for (int id = threadIdx.x; id < BN * RowChunks; id += 64 * Waves) {
            const int in_b = id / RowChunks, chunk = id % RowChunks;
            const long long row = b0 + in_b, at = a0 + chunk * 8;
            if (gives_dlogits(Epi) || (row < rows && at < p.a.rows))
                *reinterpret_cast<bf16x8 *>(reinterpret_cast<T *>(to) + row * p.out_stride + at) =
                    *reinterpret_cast<const bf16x8 *>(place_of(in_b, chunk));
        }
    };
    if (Across) store_across(static_cast<char *>(p.out));
    if constexpr (Epi == kParted) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int in_b = wave_b + 32 * j + (lane & 31);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    f32x4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = c[i][j][4 * r + e];
                    x -= __builtin_convertvector(to_quad(x, type), f32x4);
                    *reinterpret_cast<quad *>(place_of(in_b, (wave_a + 32 * i + 8 * r) >> 3) + 8 * half) = to_quad(x, type);
                }
        }
        store_across(static_cast<char *>(p.out) + p.low);
    }
}

// Two arrays, so that the compiler knows a load into one apart from a read of the other.
#define EAGER_TILES __shared__ __align__(1024) char tile0[(Shape::A + Shape::B) * 128]; \
                    __shared__ __align__(1024) char tile1[(Shape::A + Shape::B) * 128]

// Large tiles are one to a compute unit, and a last round of a few takes as long as a full one: up to kUnits / 4
// tiles of it are cut in four, so that every unit has a quarter.
template <typename T, typename Shape, int Epi>
__global__ __launch_bounds__(Shape::Threads) void logits_kernel(const Product p)
{
    EAGER_TILES;
    const int rows = gives_statistics(Epi) ? static_cast<int>(p.b.rows) : *p.counted, tiles_b = (rows + Shape::B - 1) / Shape::B;
    const int all = p.tiles_a * tiles_b;
    int id = blockIdx.x, tile_a, tile_b;
    if constexpr (Shape::Quartered) {
        const int last = all % kUnits <= kUnits / 4 ? all % kUnits : 0, full = all - last;
        if (id >= full) {
            id -= full;
            if (id >= 4 * last) return;
            const int n = in_order(id, 4 * last);
            place(full + n / 4, p.tiles_a, tiles_b, tile_a, tile_b);
            product<T, Quarter, false, false, Epi>(p, tile_a, 4 * tile_b + n % 4, 0, tile0, tile1);
            return;
        }
        place(in_order(id, full), p.tiles_a, tiles_b, tile_a, tile_b);
    } else {
        if (id >= all) return;
        place(in_order(id, all), p.tiles_a, tiles_b, tile_a, tile_b);
    }
    product<T, Shape, false, false, Epi>(p, tile_a, tile_b, 0, tile0, tile1);
}

// The tile of workgroup `id` of a product in slices.
template <typename T, typename Shape, bool ColumnsB, int Epi, int Form>
__device__ __forceinline__ void gradient(const Product &p, int id, char *tile0, char *tile1)
{
    const int all = p.tiles_a * p.tiles_b, slice = id / all;
    int tile_a, tile_b;
    place(in_order(id - slice * all, all), p.tiles_a, p.tiles_b, tile_a, tile_b);
    product<T, Shape, true, ColumnsB, Epi, Form>(p, tile_a, tile_b, slice, tile0, tile1);
}

// dw and dx of a piece in one launch: what one leaves idle in its last round the other fills.
// SumsOfDw: dw in slices of the rows, as sums in the workspace.
template <typename T, typename Shape, bool SumsOfDw, int Form>
__global__ __launch_bounds__(Shape::Threads) void gradients_kernel(const Product dw, const Product dx, int dw_tiles)
{
    EAGER_TILES;
    const int id = blockIdx.x;
    if (id < dw_tiles) gradient<T, Shape, true, SumsOfDw ? kSums : kResult, Form>(dw, id, tile0, tile1);
    else gradient<T, Shape, false, kSums, Form>(dx, id - dw_tiles, tile0, tile1);
}

// loss and lse of 16 rows from the tiles' statistics: 64 threads a row share the tiles, four loads of each under way at
// a time.  Bound by the latency of the loads and the launch: 61 rows of 393 tiles 4.1 us, 4096 of 197 4.9 (64 rows a workgroup: 6.0 and 5.5)
__global__ __launch_bounds__(1024) void rows_kernel(const float2 *stats, const float *right, const long long *target,
                                                    float *loss, float *lse, long long rows, int tiles, int vocab)
{
    __shared__ float2 part[16][kJoined];
    const float2 all = joined_statistics(stats, rows, tiles, part);
    const float top = all.x, sum = all.y;
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + threadIdx.x;
    if (threadIdx.x >= kJoined || row >= rows) return;
    // the largest logit is not added to the logarithm where the loss takes one away again
    const float log_sum = log1pf(sum - 1.0f);
    const long long t = target[row];
    lse[row] = fmaf(top, kLn2, log_sum);
    loss[row] = t < 0 ? 0.0f : t >= vocab ? __builtin_nanf("") : fmaf(fmaf(-right[row], kLog2e, top), kLn2, log_sum);
}

// The rows that count in the backward pass - those with a target and a weight - side by side: the
// products leave the others out, whatever stands in them.  Bound by one copy of x; 4096 x 1024 in bf16 7.4 us, and with
// a tenth of the targets masked the products have a tenth less to do.
__device__ __forceinline__ bool counts(const Gather &g, long long row) { return (g.target[row] >= 0) & (g.dloss[row] != 0.0f); }

// kGathered rows a workgroup
template <typename T>
__global__ __launch_bounds__(1024) void gather_kernel(const Gather g)
{
    __shared__ int sums[16], place[kGathered];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long first = static_cast<long long>(blockIdx.x) * kGathered;
    int before = 0;
    if (!g.before) {
#pragma unroll 8
        for (long long row = threadIdx.x; row < first; row += 1024) before += counts(g, row);
        for (int m = 1; m < 64; m *= 2) before += __shfl_xor(before, m, 64);
        if (lane == 0) sums[wave] = before;
    }
    __syncthreads();
    if (wave == 0) {
        before = g.before ? g.before[blockIdx.x] : 0;
        if (!g.before)
            for (int w = 0; w < 16; ++w) before += sums[w];
        const long long row = first + lane;
        const bool mine = lane < kGathered && row < g.rows;
        place_rows(g, first, before, mine ? g.target[row] : -1, place);
    }
    __syncthreads();
    move_rows<T>(g, first, place);
}

// `before` of many rows, by one workgroup: 1024 times kGathered rows at a time
__global__ __launch_bounds__(1024) void before_kernel(const Gather g, int *before)
{
    __shared__ int sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long blocks = (g.rows + kGathered - 1) / kGathered;
    int base = 0;
    for (long long b0 = 0; b0 < blocks; b0 += 1024) {
        const long long first = (b0 + threadIdx.x) * kGathered;
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kGathered; ++i)
            if (first + i < g.rows) mine += counts(g, first + i);
        int upto = mine;
        for (int m = 1; m < 64; m *= 2) {
            const int other = __shfl_up(upto, m, 64);
            if (lane >= m) upto += other;
        }
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int start = base;
        for (int w = 0; w < wave; ++w) start += sums[w];
        if (b0 + threadIdx.x < blocks) before[b0 + threadIdx.x] = start + upto - mine;
        for (int w = 0; w < 16; ++w) base += sums[w];
        __syncthreads();
    }
}

// The targets' entries of dl, 16 rows a workgroup: minus the others' sum, 64 threads a row.  Only where that is the smaller of
// the two: all p are off by lse's rounding relative to themselves, so p - 1 is the better one for a small p.  Bound by the latency of
// the loads and the launch: 4096 rows of 197 tiles 6.0 us, 1019 5.2 us; of a small
// backward pass (64 x 256 x 1009 in bf16 23.6 us, 500 x 512 x 3000 35.8) the sums and this launch are 2 and 3.5 us.
template <typename T>
__global__ __launch_bounds__(1024) void targets_kernel(const Product p, T *dl)
{
    __shared__ float part[16][kJoined];
    const int rows = *p.counted;
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + threadIdx.x % kJoined;
    const float sum = joined_sums(p.others, row < rows ? row : -1, p.b.rows, p.tiles_a, part);
    if (threadIdx.x >= kJoined || row >= rows) return;
    const long long v = p.target[row];
    if (v < p.vocab && sum < 0.5f) dl[row * p.out_stride + v] = static_cast<T>(-sum * p.dloss[row]);
}

// dx (and dw) from the slices' sums, four values a thread
struct Sums {
    const float *sums;       // [slices][rows_padded][width]
    const int *place;        // per row of `out`: its row in the sums, -1: zeros; NULL: the same
    void *out;
    long long stride, rows, rows_padded;
    int slices;
    const float *common;     // factor
};
template <typename T, bool Factored>
__global__ __launch_bounds__(256) void sums_kernel(const Sums dx, const Sums dw, int width)
{
    const Sums &s = blockIdx.y ? dw : dx;
    const int quads = width / 4;
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= s.rows * quads) return;
    const long long row = i / quads, at = (i - row * quads) * 4, place = s.place ? s.place[row] : row;
    f32x4 x = {};
    if (place >= 0) {
        const f32x4 *from = reinterpret_cast<const f32x4 *>(s.sums + place * width + at);
        x = *from;
#pragma unroll 4
        for (int n = 1; n < s.slices; ++n) x += from[n * s.rows_padded * quads];
        if (Factored) x *= *s.common;
    }
    *reinterpret_cast<typename Operand<T>::quad *>(static_cast<T *>(s.out) + row * s.stride + at) = to_quad(x, static_cast<T *>(nullptr));
}

// Tiles of a product, and their number.
template <typename T>
int lay_out(Product &p, int shape)
{
    p.tiles_a = static_cast<int>(round_up(p.a.rows, kSides[shape][0]) / kSides[shape][0]);
    p.tiles_b = static_cast<int>(round_up(p.b.rows, kSides[shape][1]) / kSides[shape][1]);
    p.all_steps = static_cast<int>(round_up(std::max(p.a.k, p.b.k), kDepth<T>) / kDepth<T>);
    p.steps = (p.all_steps + p.slices - 1) / p.slices;
    return p.tiles_a * p.tiles_b * p.slices;
}

template <typename T, int Epi>
hipError_t launch_logits(Product &p, int shape, hipStream_t stream)
{
    const int tiles = lay_out<T>(p, shape);
    const dim3 grid(shape == kLarge ? std::min(4 * tiles, tiles + 3 * (kUnits / 4)) : tiles);
    if (shape == kLarge) return launch(logits_kernel<T, Large, Epi>, grid, dim3(Large::Threads), 0, stream, p);
    if (shape == kMedium) return launch(logits_kernel<T, Medium, Epi>, grid, dim3(Medium::Threads), 0, stream, p);
    return launch(logits_kernel<T, Narrow, Epi>, grid, dim3(Narrow::Threads), 0, stream, p);
}

template <typename T, int Form>
hipError_t launch_gradients(const Cut &c, const Product &dw, const Product &dx, int dw_tiles, dim3 grid, hipStream_t stream)
{
    if (c.gradients == kLarge)
        return launch(gradients_kernel<T, Large, false, Form>, grid, dim3(Large::Threads), 0, stream, dw, dx, dw_tiles);
    return launch(c.dw_slices > 1 ? gradients_kernel<T, Medium, true, Form> : gradients_kernel<T, Medium, false, Form>, grid,
                  dim3(Medium::Threads), 0, stream, dw, dx, dw_tiles);
}

template <typename T>
hipError_t forward(const CrossEntropyArgs &a, hipStream_t stream)
{
    const bool taught = a.teacher.index;
    const int shape = logits_shape(a.rows, a.width, a.vocab, sizeof(T), taught);
    const bool kept = taught && keeps_logits(a.rows, a.width, a.vocab, a.teacher.entries, sizeof(T));
    const long long own = taught ? teacher_bytes(a.rows, a.vocab, kept) : 0;
    // a teacher's favourite takes the target's place, or the logits are kept and the entries' taken from them
    long long *const favourite = reinterpret_cast<long long *>(a.workspace);
    if (taught && !kept) {
        const hipError_t e = launch_picked(a, favourite, sizeof(T) == 2, stream);
        if (e != hipSuccess) return e;
    }
    const long long tiles = round_up(a.vocab, kSides[shape][0]) / kSides[shape][0];
    Product p = {};
    p.a = {a.w, a.w_stride, a.vocab, a.width};
    p.b = {a.x, a.x_stride, a.rows, a.width};
    p.slices = 1;
    p.live = a.vocab;
    p.scale = taught ? kLog2e / a.teacher.temperature : kLog2e;
    p.target = taught ? favourite : a.target;
    p.out = a.workspace;
    p.out_stride = round_up(a.vocab, 4);
    p.stats = reinterpret_cast<float2 *>(a.workspace + own);
    p.right = reinterpret_cast<float *>(p.stats + tiles * a.rows);
    const hipError_t e = kept ? launch_logits<T, kKept>(p, shape, stream) : launch_logits<T, kStats>(p, shape, stream);
    if (e != hipSuccess) return e;
    if (taught) {
        const Tiled t = {p.stats, p.right, favourite, static_cast<const float *>(p.out), p.out_stride, static_cast<int>(tiles), p.scale};
        return launch_divergence(a, t, kept, stream);
    }
    const float2 *stats = p.stats;
    const float *right = p.right;
    return launch(rows_kernel, dim3(static_cast<unsigned>((a.rows + kJoined - 1) / kJoined)), dim3(1024), 0, stream, stats, right,
                  a.target, a.loss, a.lse, a.rows, static_cast<int>(tiles), a.vocab);
}

template <typename T>
hipError_t backward(const CrossEntropyArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    constexpr bool Rounded = sizeof(T) == 2;
    const bool taught = a.teacher.index;
    const Form form = !taught || !Rounded ? kPlain : dlogits_pieces(a.rows, a.width, a.vocab, sizeof(T)) == 2 ? kTwice : kFactored;
    const Cut c = cut_of(a.rows, a.width, a.vocab, sizeof(T), taught, form == kTwice ? 2 : 1);
    const Layout l = layout_of(c, a.rows, a.width, sizeof(T));
    const long long low = l.end + teacher_target_bytes(a.rows) - l.dl;       // behind the favourites
    const T *w = static_cast<const T *>(a.w);
    T *dl = reinterpret_cast<T *>(a.workspace + l.dl), *x = reinterpret_cast<T *>(a.workspace + l.x);
    float *sums = reinterpret_cast<float *>(a.workspace + l.dx_sums), *dw_sums = reinterpret_cast<float *>(a.workspace + l.dw_sums);
    int *counted = reinterpret_cast<int *>(a.workspace + l.counted), *place = reinterpret_cast<int *>(a.workspace + l.place);
    float *const common = form == kFactored ? reinterpret_cast<float *>(counted + 4) : nullptr;
    Sums of_dx = {}, of_dw = {};
    const float scale = taught ? kLog2e / a.teacher.temperature : kLog2e;
    const bool few = taught && a.rows && a.rows <= kFewTaught;
    const long long *target = a.target;
    if (taught) {
        long long *const favourite = reinterpret_cast<long long *>(a.workspace + l.end);
        if (a.rows && !few) e = launch_favourites(a, favourite, stream);
        target = favourite;
    }
    Gather g = {a.x, target, a.lse, a.dloss, a.rows, a.x_stride, a.width, taught ? 1.0f / a.teacher.temperature : 1.0f, nullptr, x,
                reinterpret_cast<long long *>(a.workspace + l.target), reinterpret_cast<float *>(a.workspace + l.lse),
                reinterpret_cast<float *>(a.workspace + l.dloss), place, counted, common};
    if (e == hipSuccess && a.rows > kCountedByEach) {
        int *before = reinterpret_cast<int *>(a.workspace + l.before);
        e = launch(before_kernel, dim3(1), dim3(1024), 0, stream, g, before);
        g.before = before;
    }
    // (without rows one workgroup says that none count)
    if (few)
        e = launch_taught_rows(a, g, sizeof(T) == 2, stream);
    else if (e == hipSuccess)
        e = launch(gather_kernel<T>, dim3(static_cast<unsigned>(std::max((a.rows + kGathered - 1) / kGathered, 1ll))), dim3(1024), 0,
                   stream, g);
    for (long long first = 0; e == hipSuccess && first < a.vocab; first += c.piece) {
        const int live = static_cast<int>(std::min<long long>(a.vocab - first, c.piece));
        const long long padded = round_up(live, kSides[c.logits][0]);
        if (a.rows) {
            Product p = {};
            p.a = {w + first * a.w_stride, a.w_stride, live, a.width};
            p.b = {x, a.width, a.rows, a.width};
            p.slices = 1;
            p.first = first;
            p.live = live;
            p.vocab = a.vocab;
            p.scale = scale;
            p.whole = !taught && a.vocab <= kSides[c.logits][0];
            p.target = g.target_out;
            p.lse = g.lse_out;
            p.dloss = g.dloss_out;
            p.counted = counted;
            p.out = dl;
            p.out_stride = padded;
            p.others = c.pieces == 1 && !p.whole ? reinterpret_cast<float *>(a.workspace + l.others) : nullptr;
            p.low = form == kTwice ? low : 0;
            p.common = common;
            if (form == kTwice) e = launch_logits<T, Rounded ? kParted : kDlogits>(p, c.logits, stream);
            else if (form == kFactored) e = launch_logits<T, Rounded ? kShared : kDlogits>(p, c.logits, stream);
            else e = launch_logits<T, kDlogits>(p, c.logits, stream);
            if (e == hipSuccess && taught) {
                const Entries n = {place, g.target_out, g.lse_out, g.dloss_out, common, p.others, p.tiles_a, dl, p.low, padded, first, live, scale};
                e = launch_entries(a, n, sizeof(T) == 2, stream);
            } else if (e == hipSuccess && p.others)
                e = launch(targets_kernel<T>, dim3(static_cast<unsigned>((a.rows + kJoined - 1) / kJoined)), dim3(1024), 0, stream, p, dl);
            if (e != hipSuccess) return e;
        }
        Product dx = {}, dw = {};
        int dx_tiles = 0, dw_tiles = 0;
        if (a.dx && a.rows) {
            // dl is zero from `live` to `padded`, so its last chunk may be read whole
            dx.a = {w + first * a.w_stride, a.w_stride, a.width, live};
            dx.b = {dl, padded, a.rows, round_up(live, 16 / sizeof(T))};
            dx.counted = counted;
            dx.low = low;
            dx.slices = c.dx_slices;
            dx.out = sums;
            dx.out_stride = a.width;
            dx.accumulate = first > 0;
            dx_tiles = lay_out<T>(dx, c.gradients);
        }
        if (a.dw) {
            dw.a = {x, a.width, a.width, a.rows};
            dw.counted = counted;
            dw.low = low;
            dw.common = common;
            dw.counted_k = 1;
            dw.b = {dl, padded, padded, a.rows};
            dw.slices = c.dw_slices;
            dw.live = live;
            dw.out = c.dw_slices > 1 ? dw_sums : static_cast<void *>(static_cast<T *>(a.dw) + first * a.w_stride);
            dw.out_stride = c.dw_slices > 1 ? a.width : a.w_stride;
            dw_tiles = lay_out<T>(dw, c.gradients);
            of_dw.rows_padded = padded;
        }
        const dim3 grid(dx_tiles + dw_tiles);
        if (!(dx_tiles + dw_tiles)) continue;
        if (form == kTwice) e = launch_gradients<T, Rounded ? kTwice : kPlain>(c, dw, dx, dw_tiles, grid, stream);
        else if (form == kFactored) e = launch_gradients<T, Rounded ? kFactored : kPlain>(c, dw, dx, dw_tiles, grid, stream);
        else e = launch_gradients<T, kPlain>(c, dw, dx, dw_tiles, grid, stream);
    }
    if (e != hipSuccess) return e;
    if (a.dx && a.rows) of_dx = {sums, place, a.dx, a.x_stride, a.rows, a.rows, c.dx_slices, common};
    if (a.dw && c.dw_slices > 1) of_dw = {dw_sums, nullptr, a.dw, a.w_stride, a.vocab, of_dw.rows_padded, c.dw_slices, common};
    const long long quads = std::max(of_dx.rows, of_dw.rows) * (a.width / 4);
    if (!quads) return hipSuccess;
    return launch(form == kFactored ? sums_kernel<T, Rounded> : sums_kernel<T, false>, dim3(static_cast<unsigned>((quads + 255) / 256), of_dw.rows ? 2 : 1), dim3(256), 0, stream, of_dx,
                  of_dw, a.width);
}

}  // namespace

hipError_t launch_cross_entropy(const CrossEntropyArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? forward<__bf16>(a, stream) : forward<float>(a, stream);
}

hipError_t launch_cross_entropy_backward(const CrossEntropyArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? backward<__bf16>(a, stream) : backward<float>(a, stream);
}

}  // namespace eager
