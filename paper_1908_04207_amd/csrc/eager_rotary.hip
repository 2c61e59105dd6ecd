// Rotation of query and key heads by position, and the table of its cosines and sines.
//
//   of a pair (a, b):  a' = a cos - b sin,  b' = b cos + a sin;  gradients: the same with -sin
//
// Pairs are i and i + half or 2 i and 2 i + 1 of the first 2 half elements of a head, the others are copied.  A thread
// holds the cosines and sines of its place in a head and takes that place in several heads of its token, so that
// their loads are under way together and the table is read once for them.
//
// Bound by memory, every array once.  Measured: 20011 tokens of 50 heads of 64 in fp32 (256 MB an array) 98 us (5.2 TB/s); 8192
// of 20 heads of 64 in bf16, half of each turned, pairs side by side (21 MB, which the last cache holds) 10.0 us, 12.1 with the
// copied places in a branch of their own; 61 tokens 4 us, a launch.  The table: 131072 positions of 64 pairs (67 MB) 14 to 17 us,
// vector instructions in 64 bits busy two thirds of that beside the stores.
#include "eager_launch.h"
#include "eager_model.h"
#include "eager_model_rules.h"
#include "eager_vector.h"

namespace eager {
namespace {

template <typename T, int V> struct Piece;
template <> struct Piece<__bf16, 8> { typedef bf16x8 type; };
template <> struct Piece<__bf16, 4> { typedef bf16x4 type; };
template <> struct Piece<float, 4> { typedef f32x4 type; };

// Places of a head: `turned` of them with V elements and their partners (Interleaved: V elements, partners among them),
// then those of as many elements that are copied.  A wavefront has places of both kinds; they differ in what becomes of
// the loaded values alone.
template <typename T, int V, bool Interleaved>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a, int places, int turned)
{
    typedef typename Piece<T, V>::type vec;
    constexpr int N = Interleaved ? V / 2 : V;              // pairs a place
    constexpr int Pieces = Interleaved ? 1 : 2;
    typedef float angles __attribute__((ext_vector_type(N)));
    typedef angles placed __attribute__((aligned(N < 4 ? 4 * N : 16)));      // tables are on 16 bytes
    const int units = (a.groups[0] + a.groups[1]) * places;
    const int tokens = units < 256 ? 256 / units : 1;       // of a workgroup
    const int mine = units < 256 ? threadIdx.x / units : 0;
    if (mine >= tokens) return;
    for (long long token = static_cast<long long>(blockIdx.x) * tokens + mine; token < a.tokens;
         token += static_cast<long long>(gridDim.x) * tokens) {
        const int pos = a.positions[token];
        for (int unit = threadIdx.x - mine * units; unit < units; unit += 256) {
            int group = unit / places;
            const int place = unit - group * places;
            const bool which = group >= a.groups[0], turns = place < turned;
            if (which) group -= a.groups[0];
            const int moved = which ? a.moved[1] : a.moved[0];
            const int first = turns ? place * V : 2 * a.half + (place - turned) * Pieces * V, second = first + (turns ? a.half : V);
            if (first >= moved) continue;
            const bool both = Pieces == 2 && second < moved;
            // A thread's heads lie side by side, or where pairs are halves apart as many on as there are groups, so that the
            // short pieces of neighbouring threads lie beside each other.  Measured, side by side and apart, us: halves, bf16,
            // 52083 tokens of 12 heads of 80 53.0 and 47.5, 14568 of 143 of 24 57.5 and 51.9; interleaved, fp32, 19531 of 20 of 64
            // 47.9 and 50.0.
            const int apart = Interleaved ? 1 : which ? a.groups[1] : a.groups[0], h0 = Interleaved ? group * kTurnedHeads : group;
            const int left = (which ? a.heads[1] : a.heads[0]) - h0;
            const Heads from = which ? a.x[1] : a.x[0], to = which ? a.y[1] : a.y[0];
            const T *x = static_cast<const T *>(from.data) + token * from.row + h0 * from.head;
            T *y = static_cast<T *>(to.data) + token * to.row + h0 * to.head;
            const long long x_step = apart * from.head, y_step = apart * to.head;
            vec p[kTurnedHeads], q[kTurnedHeads];
#pragma unroll
            for (int h = 0; h < kTurnedHeads; ++h)
                if (h * apart < left) {
                    p[h] = *reinterpret_cast<const vec *>(x + h * x_step + first);
                    if (both) q[h] = *reinterpret_cast<const vec *>(x + h * x_step + second);
                }
            if (turns) {
                const bool known = pos >= 0 && pos < a.table_rows;
                const long long o = static_cast<long long>(known ? pos : 0) * a.half + place * N;
                angles c = *reinterpret_cast<const placed *>(a.cos_table + o);
                angles s = *reinterpret_cast<const placed *>(a.sin_table + o);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    c[i] = known ? c[i] : __builtin_nanf("");
                    s[i] *= a.sign;
                }
#pragma unroll
                for (int h = 0; h < kTurnedHeads; ++h) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float u = static_cast<float>(Interleaved ? p[h][2 * i] : p[h][i]);
                        const float v = static_cast<float>(Interleaved ? p[h][2 * i + 1] : q[h][i]);
                        const T left = static_cast<T>(fmaf(u, c[i], -(v * s[i]))), right = static_cast<T>(fmaf(v, c[i], u * s[i]));
                        if (Interleaved) p[h][2 * i] = left, p[h][2 * i + 1] = right;
                        else p[h][i] = left, q[h][i] = right;
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < kTurnedHeads; ++h)
                if (h * apart < left) {
                    *reinterpret_cast<vec *>(y + h * y_step + first) = p[h];
                    if (both) *reinterpret_cast<vec *>(y + h * y_step + second) = q[h];
                }
        }
    }
}

template <typename T, int V, bool Interleaved>
hipError_t enqueue(const RotaryArgs &a, hipStream_t stream)
{
    const int turned = a.half / (Interleaved ? V / 2 : V);
    const int most = std::max(a.moved[0], a.moved[1]);
    const int places = turned + (most - 2 * a.half + (Interleaved ? V : 2 * V) - 1) / (Interleaved ? V : 2 * V);
    const int units = (a.groups[0] + a.groups[1]) * places, tokens = units < 256 ? 256 / units : 1;
    return launch(rotary_kernel<T, V, Interleaved>, dim3(static_cast<unsigned>(std::min((a.tokens + tokens - 1) / tokens, kMostBlocks))),
                  dim3(256), 0, stream, a, places, turned);
}

// Four pairs of a position a thread.  The angle in quarter turns, in 64 bits; what is beyond the nearest whole number
// of them, at most an eighth of a turn, goes into the series of sine and cosine up to x^11 and x^10, which leave out
// less than 7e-12 and 2e-10 (pi/4 to the 13th and 12th over the factorials), a hundredth of a rounding of the result.
__global__ __launch_bounds__(256) void rotary_table_kernel(const TableArgs a)
{
    const int quads = a.half / 4, rows = 256 / quads;       // positions of a workgroup
    const int mine = threadIdx.x / quads, first = (threadIdx.x - mine * quads) * 4;
    if (mine >= rows) return;
    double quarters_of[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) quarters_of[i] = a.quarters[first + i];
    for (long long pos = static_cast<long long>(blockIdx.x) * rows + mine; pos < a.positions; pos += static_cast<long long>(gridDim.x) * rows) {
        f32x4 c, s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (adding 1.5 2^52 leaves the nearest whole number in the last bits)
            const double quarters = static_cast<double>(pos) * quarters_of[i], shifted = quarters + 0x1.8p52;
            const int n = __double2loint(shifted) & 3;
            const double x = (quarters - (shifted - 0x1.8p52)) * 1.5707963267948966, x2 = x * x;
            double sine = fma(x2, -1.0 / 39916800, 1.0 / 362880), cosine = fma(x2, -1.0 / 3628800, 1.0 / 40320);
            sine = fma(x2, sine, -1.0 / 5040), cosine = fma(x2, cosine, -1.0 / 720);
            sine = fma(x2, sine, 1.0 / 120), cosine = fma(x2, cosine, 1.0 / 24);
            sine = fma(x2, sine, -1.0 / 6), cosine = fma(x2, cosine, -0.5);
            sine = fma(x2 * x, sine, x), cosine = fma(x2, cosine, 1.0);
            const double along = n & 1 ? sine : cosine, across = n & 1 ? cosine : sine;
            c[i] = static_cast<float>((n == 1 || n == 2 ? -along : along) * a.magnitude);
            s[i] = static_cast<float>((n & 2 ? -across : across) * a.magnitude);
        }
        *reinterpret_cast<f32x4 *>(a.cos_table + pos * a.half + first) = c;
        *reinterpret_cast<f32x4 *>(a.sin_table + pos * a.half + first) = s;
    }
}

}  // namespace

// Places of 16 bytes; in bf16 halves that are no multiple of 8 take 8 bytes (4 pairs), as 16 would pass their end: 8192 tokens
// of 20 heads of 64, 24 of them turned, 11.7 us.
hipError_t launch_rotary(const RotaryArgs &a, bool bf16, bool interleaved, hipStream_t stream)
{
    if (!bf16) return interleaved ? enqueue<float, 4, true>(a, stream) : enqueue<float, 4, false>(a, stream);
    if (interleaved) return enqueue<__bf16, 8, true>(a, stream);
    return a.half % 8 == 0 ? enqueue<__bf16, 8, false>(a, stream) : enqueue<__bf16, 4, false>(a, stream);
}

hipError_t launch_rotary_table(const TableArgs &a, hipStream_t stream)
{
    const int rows = 256 / (a.half / 4);
    return launch(rotary_table_kernel, dim3(static_cast<unsigned>(std::min((a.positions + rows - 1) / rows, kTableBlocks))), dim3(256), 0,
                  stream, a);
}

}  // namespace eager
