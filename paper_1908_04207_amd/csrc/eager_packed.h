// Tiles of a packed batch: which rows a workgroup has, found from the sequences' bounds in device
// memory, so that no call waits for lengths.
//
// The rows fall into sequences + 2 segments: those before the first sequence, the sequences, those
// after the last.  Segment i, which begins at row e_i, has the tiles from e_i / Rows + i on: as
// floor(a + b) >= floor(a) + floor(b), they suffice for its rows, and the numbers ascend, so a
// search finds a tile's segment.  At most tokens / Rows + sequences + 2 numbers are in use.
#pragma once

#include "eager_matrix.h"
#include "eager_model.h"

namespace eager {

struct Tile {
    int segment;             // 0 and sequences + 1: rows of no sequence
    int begin, end;          // rows of the segment
    int first;               // first row of the tile; none if it is not below `end`
};

__device__ __forceinline__ int segment_start(const int *cu, int sequences, int tokens, int i)
{
    if (i == 0) return 0;
    if (i > sequences + 1) return tokens;
    return min(max(cu[i - 1], 0), tokens);
}

// Every wavefront searches for itself, 64 candidates at a time.
template <int Rows>
__device__ __forceinline__ Tile find_tile(const int *cu, int sequences, int tokens, int number)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, count = sequences + 2;
    while (count > 1) {
        const int step = (count + 63) >> 6;
        const int i = lo + lane * step;
        const bool below = lane * step < count && segment_start(cu, sequences, tokens, i) / Rows + i <= number;
        const int k = max(__popcll(__ballot(below)) - 1, 0);
        lo += k * step;
        count = min(step, count - k * step);
    }
    Tile t;
    t.segment = __builtin_amdgcn_readfirstlane(lo);
    t.begin = __builtin_amdgcn_readfirstlane(segment_start(cu, sequences, tokens, lo));
    t.end = __builtin_amdgcn_readfirstlane(max(t.begin, segment_start(cu, sequences, tokens, lo + 1)));
    const long long first = t.begin + static_cast<long long>(number - (t.begin / Rows + lo)) * Rows;
    t.first = __builtin_amdgcn_readfirstlane(static_cast<int>(min(max(first, 0ll), static_cast<long long>(t.end))));
    return t;
}

inline long long tile_numbers(long long tokens, int sequences, int rows) { return tokens / rows + sequences + 2; }

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
