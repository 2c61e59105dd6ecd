// The divergence of a student's softmax from a teacher's, known by the top logits of each row, and its gradients of
// logits at those entries.
//
//   q = softmax(t / temperature) over the entries, p = softmax(l / temperature) over the vocabulary, l = x w^T
//   loss = sum q (log q - log p),  dl = dloss / temperature (p - q)
//
// The products are those of the cross entropy, with the word that the teacher favours in the target's place: tiles
// leave statistics forward, dl without q backward.  What is left for here: the student's logits of the entries, one
// dot product each, in the forward pass; the losses; and the entries' dl, which replace what the tiles wrote there,
// as p - q is to be rounded and not p.
//
// Differences are formed where they keep their digits: log p from a logit's distance to the row's largest, and the
// favourite's p - q, where p is beyond a half, from the sums of the others' q and p.
#include "eager_distillation.h"
#include "eager_joined.h"
#include "eager_launch.h"
#include "eager_model_rules.h"
#include "eager_vector.h"

namespace eager {
namespace {

constexpr int kEntries = 256, kOfLane = kEntries / 64;

__device__ __forceinline__ bool counts(long long index, float logit) { return (index >= 0) & (logit != -__builtin_inff()); }

// A row's entries, kOfLane a lane of a wavefront.
struct List {
    long long index[kOfLane];
    float logit[kOfLane];
    bool used[kOfLane];

    __device__ __forceinline__ List(const TeacherArgs &t, long long row, int lane)
    {
#pragma unroll
        for (int j = 0; j < kOfLane; ++j) {
            const int k = 64 * j + lane;
            index[j] = k < t.entries ? t.index[row * t.entries + k] : -1;
            logit[j] = k < t.entries ? t.logits[row * t.entries + k] : 0.0f;
            used[j] = counts(index[j], logit[j]);
        }
    }

    __device__ __forceinline__ float top() const
    {
        float t = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < kOfLane; ++j) t = used[j] ? fmaxf(t, logit[j]) : t;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) t = fmaxf(t, __shfl_xor(t, m, 64));
        return t;
    }

    // the word of the largest logit (the first of equal ones; any where none is a number), -1: no entry counts, vocab: an
    // index is beyond it
    __device__ __forceinline__ long long favourite(int vocab, int lane) const
    {
        const float t = top();
        long long word = -1;
        int at = 1 << 30;
        bool beyond = false;
#pragma unroll
        for (int j = 0; j < kOfLane; ++j) {
            if (!used[j]) continue;
            beyond |= index[j] >= vocab;
            const int rank = 64 * j + lane + (logit[j] == t ? 0 : 1 << 20);
            if (rank < at) at = rank, word = index[j];
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int other = __shfl_xor(at, m, 64);
            const long long its = __shfl_xor(word, m, 64);
            if (other < at) at = other, word = its;
        }
        return __any(beyond) ? vocab : word;
    }
};

// Four sums over a wavefront at once: after two steps a lane holds a quarter of the lanes' sum of one of them.
// Sum i is in the lanes whose last two bits are i.
__device__ __forceinline__ float four_sums(const float (&x)[4], int lane)
{
    const bool odd = lane & 1, upper = lane & 2;
    const float a = (odd ? x[1] : x[0]) + __shfl_xor(odd ? x[0] : x[1], 1, 64);
    const float b = (odd ? x[3] : x[2]) + __shfl_xor(odd ? x[2] : x[3], 1, 64);
    float c = (upper ? b : a) + __shfl_xor(upper ? a : b, 2, 64);
#pragma unroll
    for (int m = 4; m < 64; m *= 2) c += __shfl_xor(c, m, 64);
    return c;
}

// One row a workgroup, four entries a wavefront at a time.
template <typename T>
__global__ __launch_bounds__(256) void picked_kernel(const CrossEntropyArgs a, long long *favourite)
{
    constexpr int E = kVector<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), entries = a.teacher.entries;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        if (wave == 0) {
            const long long word = List(a.teacher, row, lane).favourite(a.vocab, lane);
            if (lane == 0) favourite[row] = word;
        }
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        for (int e0 = 4 * wave; e0 < entries; e0 += 16) {
            const T *w[4];
            float sum[4] = {};
            long long mine = -1;
            bool used = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = min(e0 + j, entries - 1);
                const long long index = a.teacher.index[row * entries + k];
                const bool there = counts(index, a.teacher.logits[row * entries + k]);
                if ((lane & 3) == j) mine = index, used = there;
                w[j] = static_cast<const T *>(a.w) + (there && index < a.vocab ? index : 0) * a.w_stride;
            }
            for (int at = lane * E; at < a.width; at += 64 * E) {
                const auto u = load16(x + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const auto v = load16(w[j] + at);
#pragma unroll
                    for (int i = 0; i < E; ++i) sum[j] = fmaf(static_cast<float>(u[i]), static_cast<float>(v[i]), sum[j]);
                }
            }
            const float all = four_sums(sum, lane);
            if (lane < 4 && e0 + lane < entries)
                a.teacher.picked[row * entries + e0 + lane] = !used ? 0.0f : mine < a.vocab ? all : __builtin_nanf("");
        }
    }
}

// Four rows a workgroup.
__global__ __launch_bounds__(256) void favourites_kernel(const CrossEntropyArgs a, long long *favourite)
{
    const int lane = threadIdx.x & 63;
    for (long long row = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6); row < a.rows; row += 4ll * gridDim.x) {
        const long long word = List(a.teacher, row, lane).favourite(a.vocab, lane);
        if (lane == 0) favourite[row] = word;
    }
}

// kJoined rows a workgroup: their statistics, then a wavefront for each row's entries.
__global__ __launch_bounds__(1024) void divergence_kernel(const CrossEntropyArgs a, const float2 *stats, const float *right,
                                                          const long long *favourite, int tiles, float scale)
{
    __shared__ float2 part[16][kJoined];
    __shared__ float tops[kJoined], logs[kJoined];
    const float2 all = joined_statistics(stats, a.rows, tiles, part);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x < kJoined) {
        const long long row = static_cast<long long>(blockIdx.x) * kJoined + threadIdx.x;
        const float log_sum = log1pf(all.y - 1.0f);
        tops[threadIdx.x] = all.x, logs[threadIdx.x] = log_sum;
        if (row < a.rows) a.lse[row] = fmaf(all.x, kLn2, log_sum);
    }
    __syncthreads();
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + wave;
    if (row >= a.rows) return;
    const long long word = favourite[row];
    if (word < 0 || word >= a.vocab) {
        if (lane == 0) a.loss[row] = word < 0 ? 0.0f : __builtin_nanf("");
        return;
    }
    const List list(a.teacher, row, lane);
    const float top = list.top(), its = right[row];
    float sum = 0.0f, e[kOfLane], distance[kOfLane], loss = 0.0f;
#pragma unroll
    for (int j = 0; j < kOfLane; ++j) {
        // logarithms to base two, of q without its sum
        distance[j] = list.used[j] ? (list.logit[j] - top) * scale : 0.0f;
        e[j] = list.used[j] ? exp2_fast(distance[j]) : 0.0f;
        sum += e[j];
    }
    sum = lanes_sum<64>(sum);
    const float log_q = log1pf(sum - 1.0f);
#pragma unroll
    for (int j = 0; j < kOfLane; ++j) {
        if (!list.used[j]) continue;
        const float l = list.index[j] == word ? its : a.teacher.picked[row * a.teacher.entries + 64 * j + lane];
        const float apart = distance[j] - fmaf(l, scale, -tops[wave]);
        const float term = e[j] / sum * (fmaf(apart, kLn2, logs[wave]) - log_q);
        loss += e[j] == 0.0f ? 0.0f : term;
    }
    loss = lanes_sum<64>(loss);
    if (lane == 0) a.loss[row] = loss;
}

// kJoined rows a workgroup, a wavefront for each row's entries.
template <typename T>
__global__ __launch_bounds__(1024) void entries_kernel(const CrossEntropyArgs a, const Entries n)
{
    __shared__ float part[16][kJoined], apart[kJoined];
    __shared__ int words[kJoined][kEntries];
    __shared__ float shares[kJoined][kEntries];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (n.others) {
        const long long row = static_cast<long long>(blockIdx.x) * kJoined + threadIdx.x % kJoined;
        const float sum = joined_sums(n.others, row < a.rows ? n.place[row] : -1, a.rows, n.tiles, part);
        if (threadIdx.x < kJoined) apart[threadIdx.x] = sum;
        __syncthreads();
    }
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + wave;
    const int place = row < a.rows ? n.place[row] : -1;
    if (place < 0) return;
    const long long word = n.favourite[place];
    if (word >= a.vocab) return;                         // the tiles wrote NaN
    const List list(a.teacher, row, lane);
    const float top = list.top();
    float sum = 0.0f, q[kOfLane];
#pragma unroll
    for (int j = 0; j < kOfLane; ++j) {
        q[j] = list.used[j] ? exp2_fast((list.logit[j] - top) * n.scale) : 0.0f;
        sum += q[j];
    }
    sum = lanes_sum<64>(sum);
    float rest = 0.0f;                                   // of q, without the favourite's
#pragma unroll
    for (int j = 0; j < kOfLane; ++j) {
        const int k = 64 * j + lane;
        q[j] /= sum;
        if (list.used[j] && list.index[j] != word) rest += q[j];
        words[wave][k] = list.used[j] ? static_cast<int>(list.index[j]) : -1;
        shares[wave][k] = q[j];
    }
    rest = lanes_sum<64>(rest);
    __builtin_amdgcn_wave_barrier();
    const float lse = n.lse[place] * kLog2e, by = n.dloss[place];
#pragma unroll
    for (int j = 0; j < kOfLane; ++j) {
        const int k = 64 * j + lane;
        if (!list.used[j] || list.index[j] < n.first || list.index[j] >= n.first + n.live) continue;
        // a word that stands in several entries is written by the first of them
        float share = 0.0f;
        bool first = true;
        for (int i = 0; i < a.teacher.entries; ++i) {
            const bool same = words[wave][i] == list.index[j];
            share += same ? shares[wave][i] : 0.0f;
            first &= !(same && i < k);
        }
        if (!first) continue;
        float d = exp2_fast(fmaf(a.teacher.picked[row * a.teacher.entries + k], n.scale, -lse)) - share;
        if (n.others && list.index[j] == word && apart[wave] < 0.5f) d = rest - apart[wave];
        static_cast<T *>(n.dl)[place * n.stride + list.index[j] - n.first] = static_cast<T>(d * by);
    }
}

unsigned workgroups(long long rows, int each) { return static_cast<unsigned>(std::min((rows + each - 1) / each, kMostBlocks)); }

}  // namespace

hipError_t launch_picked(const CrossEntropyArgs &a, long long *favourite, bool bf16, hipStream_t stream)
{
    return launch(bf16 ? picked_kernel<__bf16> : picked_kernel<float>, dim3(workgroups(a.rows, 1)), dim3(256), 0, stream, a, favourite);
}

hipError_t launch_favourites(const CrossEntropyArgs &a, long long *favourite, hipStream_t stream)
{
    return launch(favourites_kernel, dim3(workgroups(a.rows, 4)), dim3(256), 0, stream, a, favourite);
}

hipError_t launch_divergence(const CrossEntropyArgs &a, const float2 *stats, const float *right, const long long *favourite,
                             int tiles, float scale, hipStream_t stream)
{
    return launch(divergence_kernel, dim3(static_cast<unsigned>((a.rows + kJoined - 1) / kJoined)), dim3(1024), 0, stream, a, stats,
                  right, favourite, tiles, scale);
}

hipError_t launch_entries(const CrossEntropyArgs &a, const Entries &n, bool bf16, hipStream_t stream)
{
    return launch(bf16 ? entries_kernel<__bf16> : entries_kernel<float>, dim3(static_cast<unsigned>((a.rows + kJoined - 1) / kJoined)),
                  dim3(1024), 0, stream, a, n);
}

}  // namespace eager
