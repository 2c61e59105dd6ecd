// Causal attention over packed sequences, forward.
//
//   s_ij = scale <q_i, k_j>,  m_i = max s_i,  l_i = sum exp(s_ij - m_i),  out_i = sum exp(s_ij - m_i) v_j / l_i
//
// One pass over the keys with the running maximum and sum of every row.  The products are formed
// transposed, S^T = K Q^T and O^T = V^T P^T: a lane then holds scores of one row only, so maximum
// and sum are taken in registers (one exchange between the halves of a wavefront), the rescaling
// of O is one factor a lane, and P^T is the second product's operand as it stands.  P is rounded to
// bf16 for that product where the inputs are (a matrix instruction takes both sides in one type); its sum l is taken
// in fp32 before the rounding, so that lse is that of the scores, and the weights that are applied add up to one
// within P's roundings.
//
// Tiles of keys come by loads that write shared memory directly, one tile ahead, and tiles of queries
// with the most keys first: a workgroup's time is its number of key tiles.
//
// Bound, heads of 64: the vector instructions of the softmax (an exponential of 16 clocks per 64 scores and about 4 more
// instructions each), 75 % of a unit's clocks with 25 heads beside 32 % of matrix instructions, and what is open between a tile's
// steps, which wait for each other (barrier, scores, maximum, exponentials, second product); with short
// sequences the longest row's chain of them: 0.87 us a tile of keys and 3.2 us of start and end (16 sequences: 68 and
// 26 %).  Heads of 128: matrix instructions 56 %, vector instructions 56 %.
// Measured: bf16, 16 heads (4 of keys) of 64: 113 tokens 6.2 us, 16 sequences of 8192 tokens 31 us; 25 heads of 64, 8
// sequences of 1024: 50 us (532 TFLOP/s, masked pairs not counted); 8 heads (2) of 128, one sequence of 16384: 588 us
// (935 TFLOP/s); fp32, 16 heads (8) of 64, 9 sequences, 4099 tokens: 78 us.
//
// Slower, 16 sequences and 8 x 1024 of the above: two groups of wavefronts that share a row's keys and join their
// statistics (39 and 62 us against 31 and 52), two tiles of queries a workgroup (43 and 61).
#include "eager_launch.h"
#include "eager_packed.h"

namespace eager {
namespace {

constexpr int kRows = kAttentionRows;        // query rows of a workgroup: 32 a wavefront
constexpr int kKeys = 64;            // keys of a tile

template <typename T, int DP>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1) void attention_kernel(const AttentionArgs a)
{
    constexpr int Chunks = DP * sizeof(T) / 16, TileBytes = kKeys * Chunks * 16, Steps = DP / 16;
    // arrays of their own, so that the compiler knows a load into one apart from a read of another
    __shared__ __align__(1024) char k_tile0[TileBytes];
    __shared__ __align__(1024) char v_tile0[TileBytes];
    __shared__ __align__(1024) char k_tile1[TileBytes];
    __shared__ __align__(1024) char v_tile1[TileBytes];
    T *const type = nullptr;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % a.q_heads;
    const Tile t = find_tile<kRows>(a.cu, a.sequences, static_cast<int>(a.tokens),
                                    blockIdx.x / a.q_heads, false);
    if (t.first >= t.end) return;
    if (t.segment == 0 || t.segment == a.sequences + 1) {
        clear_rows<T, kRows>(a.out, head, t.first, t.end, a.dim);
        for (int i = threadIdx.x; i < min(kRows, t.end - t.first); i += 256)
            a.lse[head * a.tokens + t.first + i] = -__builtin_inff();
        return;
    }
    const int kv_head = head / (a.q_heads / a.kv_heads);
    const int wave_row = t.first + 32 * wave, row = wave_row + (lane & 31);
    const T *q_row = static_cast<const T *>(a.q.data) + static_cast<long long>(row) * a.q.row + head * a.q.head;
    decltype(operand(typename Operand<T>::frag())) q[Steps];
#pragma unroll
    for (int s = 0; s < Steps; ++s) q[s] = operand(row_operand(q_row, s, lane, a.dim, row < t.end));

    const char *k_base = reinterpret_cast<const char *>(static_cast<const T *>(a.k.data) + kv_head * a.k.head);
    const char *v_base = reinterpret_cast<const char *>(static_cast<const T *>(a.v.data) + kv_head * a.v.head);
    const long long k_stride = a.k.row * sizeof(T), v_stride = a.v.row * sizeof(T);
    const int chunks = a.dim * sizeof(T) / 16;
    auto stage = [&](int key0, char *k_tile, char *v_tile) {
        stage_rows<kKeys, Chunks, 4>(k_tile, k_base + key0 * k_stride, k_stride, t.end - key0, chunks, wave, lane);
        stage_rows<kKeys, Chunks, 4>(v_tile, v_base + key0 * v_stride, v_stride, t.end - key0, chunks, wave, lane);
    };

    const float c = a.scale * kLog2e;
    const int last = min(t.end, t.first + kRows);       // no key from here on is seen
    f32x16 o[DP / 32] = {};
    float top = -__builtin_inff(), sum = 0.0f;
    auto tile = [&](int key0, char *k_tile, char *v_tile, char *next_k, char *next_v) {
        wait_loads();
        __syncthreads();
        stage(key0 + kKeys, next_k, next_v);            // beyond the sequence: zeros
        if (key0 >= wave_row + 32) return;              // every key is later than the wavefront's rows
        f32x16 s[2] = {};
#pragma unroll
        for (int i = 0; i < Steps; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[b] = mma(operand(read_rows<Chunks>(k_tile, 32 * b, i, lane, type)), q[i], s[b]);
        if (key0 + kKeys - 1 > wave_row) {
            const int seen = row - key0 - 4 * (lane >> 5);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * b + 8 * (i >> 2) + (i & 3) > seen) s[b][i] = -__builtin_inff();
        }
        // (a NaN among the scores stays: its row becomes NaN)
        float best = top;
#pragma unroll
        for (int i = 0; i < 16; ++i) best = __builtin_elementwise_maximum(best, __builtin_elementwise_maximum(s[0][i], s[1][i]));
        best = both_max(best);
        const float base = best == -__builtin_inff() ? 0.0f : best * c;
        if (__any(best != top)) {                       // a new maximum: rare after the first tiles
            // from the rounded reference that the sums have: exactly 1 for the rows whose maximum stays
            const float keep = exp2_fast(top * c - base);
            top = best;
            sum *= keep;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= keep;
        }
        float add[2] = {};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = exp2_fast(fmaf(s[b][i], c, -base));
                add[b] += s[b][i];
            }
        sum += add[0] + add[1];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto p = operand(as_operand<T>(s[b], h));
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
                    o[d] = mma(operand(read_columns<Chunks>(v_tile, 32 * d, 32 * b + 16 * h, 4, 8, lane, type)), p, o[d]);
            }
    };
    stage(t.begin, k_tile0, v_tile0);
    for (int key0 = t.begin; key0 < last; key0 += 2 * kKeys) {
        tile(key0, k_tile0, v_tile0, k_tile1, v_tile1);
        tile(key0 + kKeys, k_tile1, v_tile1, k_tile0, v_tile0);
    }
    wait_loads();
    sum = both_sum(sum);
    if (row < t.end) {
        T *out = static_cast<T *>(a.out.data) + static_cast<long long>(row) * a.out.row + head * a.out.head;
        store_row<T, DP>(out, o, 1.0f / sum, lane, a.dim);
        // what rounding the reference top * c has left is in the sum, and taken out of its logarithm
        const float left = top == -__builtin_inff() ? 0.0f : fmaf(top, c, -(top * c));
        if (lane < 32) a.lse[head * a.tokens + row] = fmaf(top, a.scale, (log2_fast(sum) - left) * kLn2);
    }
}

template <typename T>
hipError_t enqueue(const AttentionArgs &a, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(tile_numbers(a.tokens, a.sequences, kRows) * a.q_heads));
    return launch(a.dim <= 64 ? attention_kernel<T, 64> : attention_kernel<T, 128>, grid, dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_attention(const AttentionArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? enqueue<__bf16>(a, stream) : enqueue<float>(a, stream);
}

}  // namespace eager
