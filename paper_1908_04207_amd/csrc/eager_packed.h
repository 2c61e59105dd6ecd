// Tiles of a packed batch: which rows a workgroup has, found from the sequences' bounds in device
// memory, so that no call waits for lengths.
//
// The rows fall into sequences + 2 segments: those before the first sequence, the sequences, those
// after the last.  Together they have at most tokens / Rows + sequences + 2 tiles, and as many
// workgroups (a head) look for theirs.  Under a causal mask a tile's work grows along its sequence (for keys:
// towards its front), so up to 64 segments, a lane each, are gone through by work: the n-th tile is found from
// F(j) = sum over segments of max(0, tiles - j), the number of tiles of work j or more.  More segments than lanes go by
// number: segment i, which begins at row e_i, has the tiles from e_i / Rows + i on; as
// floor(a + b) >= floor(a) + floor(b), they suffice for its rows, and the numbers ascend.
//
// Measured, 8192 tokens, 16 heads (4 of keys) of 64, bf16, by work and by number, forward / backward in us: 8 sequences, the
// longest of 2709 tokens, 51 / 143 and 67 / 183; 16 (1590) 32.5 / 102 and 37 / 103; 32 (1080) 27.8 / 91 and 28.8 / 88; 62 (541) 26.1 / 91.5 and
// 25.3 / 86; 62 (1155) 33 / 108 and 36.6 / 109.5.  Beyond 62 a long sequence among short ones costs that tenth: 63 (1130) 37 / 112.
#pragma once

#include "eager_matrix.h"
#include "eager_model.h"
#include "eager_model_rules.h"

namespace eager {

struct Tile {
    int segment;             // 0 and sequences + 1: rows of no sequence
    int begin, end;          // rows of the segment
    int first;               // first row of the tile; none if it is not below `end`
};

__device__ __forceinline__ int segment_start(const int *cu, int sequences, int tokens, int i)
{
    const int bound = cu[min(max(i - 1, 0), sequences)];
    return i == 0 ? 0 : i > sequences + 1 ? tokens : min(max(bound, 0), tokens);
}

// Up to 64 segments: a lane a segment, one trip to memory; then a lane a value of j.
template <int Rows>
__device__ __forceinline__ Tile find_by_work(const int *cu, int sequences, int tokens, int number, bool from_back)
{
    const int lane = threadIdx.x & 63;
    const int begin = segment_start(cu, sequences, tokens, lane), next = segment_start(cu, sequences, tokens, lane + 1);
    const int tiles = lane < sequences + 2 ? (max(next - begin, 0) + Rows - 1) / Rows : 0;
    int most = tiles;
    for (int m = 1; m < 64; m *= 2) most = max(most, __shfl_xor(most, m, 64));
    most = __builtin_amdgcn_readfirstlane(most);
    // the largest j with F(j) > number, from the end of [lo, lo + count) that is left
    int lo = 0, count = most + 1, rest = 0;
    for (;;) {
        const int step = (count + 63) >> 6, j = lo + lane * step;
        int f = 0, after = 0;                           // F(j), F(j + 1)
        for (int s = 0; s < sequences + 2; ++s) {
            const int n = __builtin_amdgcn_readlane(tiles, s);
            f += max(n - j, 0);
            after += max(n - j - 1, 0);
        }
        const int k = __popcll(__ballot(lane * step < count && f > number)) - 1;
        if (k < 0) {                                    // there are fewer tiles
            Tile t = {};
            return t;
        }
        lo += k * step;
        if (step == 1) {
            rest = number - __builtin_amdgcn_readlane(after, k);
            break;
        }
        count = min(step, count - k * step);
    }
    // of the segments with more than lo tiles, the one with `rest` of them in front of it
    unsigned long long mask = __ballot(tiles > lo);
    for (; rest > 0; --rest) mask &= mask - 1;
    const int s = __ffsll(static_cast<long long>(mask)) - 1;
    Tile t;
    t.segment = s;
    t.begin = __builtin_amdgcn_readlane(begin, s);
    t.end = max(t.begin, __builtin_amdgcn_readlane(next, s));
    t.first = t.begin + (from_back ? __builtin_amdgcn_readlane(tiles, s) - 1 - lo : lo) * Rows;
    return t;
}

// More: 64 candidates at a time.  The last step's candidates are the bounds.
template <int Rows>
__device__ __forceinline__ Tile find_by_number(const int *cu, int sequences, int tokens, int number)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, count = sequences + 2;
    Tile t;
    for (;;) {
        const int step = (count + 63) >> 6;
        const int i = lo + lane * step;
        const int start = segment_start(cu, sequences, tokens, i), next = segment_start(cu, sequences, tokens, i + 1);
        const bool below = lane * step < count && start / Rows + i <= number;
        const int k = max(__popcll(__ballot(below)) - 1, 0);
        lo += k * step;
        if (step == 1) {
            t.begin = __builtin_amdgcn_readlane(start, k);
            t.end = max(t.begin, __builtin_amdgcn_readlane(next, k));
            break;
        }
        count = min(step, count - k * step);
    }
    t.segment = __builtin_amdgcn_readfirstlane(lo);
    const long long first = t.begin + static_cast<long long>(number - (t.begin / Rows + t.segment)) * Rows;
    t.first = static_cast<int>(min(max(first, static_cast<long long>(t.begin)), static_cast<long long>(t.end)));
    return t;
}

// Every wavefront searches for itself.  from_back: the first tiles of a segment have the most work.
template <int Rows>
__device__ __forceinline__ Tile find_tile(const int *cu, int sequences, int tokens, int number, bool from_back)
{
    return sequences <= 62 ? find_by_work<Rows>(cu, sequences, tokens, number, from_back)
                           : find_by_number<Rows>(cu, sequences, tokens, number);
}

// The larger of, and the sum over, a lane and the one 32 away.
__device__ __forceinline__ void both_halves(float &x, float &y)
{
    const unsigned a = __builtin_bit_cast(unsigned, x);
    const auto p = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const unsigned low = p[0], high = p[1];     // a cast of p[1] itself would give p[0]
    x = __builtin_bit_cast(float, low);
    y = __builtin_bit_cast(float, high);
}
__device__ __forceinline__ float both_max(float x)
{
    float y;
    both_halves(x, y);
    return __builtin_elementwise_maximum(x, y);
}
__device__ __forceinline__ float both_sum(float x)
{
    float y;
    both_halves(x, y);
    return x + y;
}

// A lane's operand of one row straight from global memory, k step `step`; zeros where !there and
// beyond the head's dim elements.
__device__ __forceinline__ bf16x8 row_operand(const __bf16 *row, int step, int lane, int dim, bool there)
{
    const int at = 16 * step + 8 * (lane >> 5);
    bf16x8 f = {};
    if (there && at < dim) f = *reinterpret_cast<const bf16x8 *>(row + at);
    return f;
}
__device__ __forceinline__ f32x8 row_operand(const float *row, int step, int lane, int dim, bool there)
{
    const int at = 16 * step + 8 * (lane >> 5);
    f32x8 f = {};
    if (there && at < dim) {
        const f32x4 a = *reinterpret_cast<const f32x4 *>(row + at), b = *reinterpret_cast<const f32x4 *>(row + at + 4);
        f = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return f;
}

// A lane's column of a 32-column, DP-row result to its row of an output, times `factor`.
template <typename T, int DP>
__device__ __forceinline__ void store_row(T *row, const f32x16 (&acc)[DP / 32], float factor, int lane, int dim)
{
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int at = 32 * b + 8 * r + 4 * (lane >> 5);
            f32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = acc[b][4 * r + i] * factor;
            if (at < dim) *reinterpret_cast<typename Operand<T>::quad *>(row + at) = to_quad(x, static_cast<T *>(nullptr));
        }
}

// Zeros for the rows [first, first + Rows) below `end` of one head.
template <typename T, int Rows>
__device__ __forceinline__ void clear_rows(const Heads &y, int head, int first, int end, int dim)
{
    const int quads = dim / 4, rows = min(Rows, end - first);
    for (int i = threadIdx.x; i < rows * quads; i += blockDim.x) {
        T *row = static_cast<T *>(y.data) + static_cast<long long>(first + i / quads) * y.row + head * y.head;
        *reinterpret_cast<typename Operand<T>::quad *>(row + i % quads * 4) = to_quad(f32x4{0, 0, 0, 0}, static_cast<T *>(nullptr));
    }
}

}  // namespace eager
