// The divergence of a student's softmax from a teacher's, known by the top logits of each row, and its gradients of
// logits at those entries.
//
//   q = softmax(t / temperature) over the entries, p = softmax(l / temperature) over the vocabulary, l = x w^T
//   loss = sum q (log q - log p),  dl = dloss / temperature (p - q)
//
// The products are those of the cross entropy, with the word that the teacher favours in the target's place: tiles
// leave statistics forward, dl without q backward.  What is left for here: the student's logits of the entries in the
// forward pass, one dot product each, or out of all logits where these are few enough to be kept (keeps_logits); the
// losses; and the entries' dl, which replace what the tiles wrote there, as p - q is to be rounded and not p.
//
// Bound by the products (see there).  Measured, us, 4096 x 1024 x 50257 in bf16 with 64 entries a row: picked logits 39 (435 MB of
// the projection's rows at 11 TB/s, most from second-level caches; 61 with fmaf for dot instructions and 64 lanes an entry), divergences 7, favourites 5,
// entries of dl 11.3, beside 910 of logits, twice, and 830 of dx and dw; 1019 rows in fp32 with 32 entries 16.5, 6.5, 5 and 7.1 beside
// 1305 and 1180; 64 x 512 x 1000 in bf16 with 256 entries: entries of dl 5.7 (20.8 where every entry was compared with every
// other of its row for repeated words), beside 22 and 7.
//
// dl beside bf16 inputs is bf16 itself, in two pieces for few rows (dlogits_pieces).  For more, what is rounded leaves out the
// digits of the first row's weight, which the products' sums are multiplied by: a mean gives every row the same weight, and
// rounded with it dl of all words that the student does not know yet (p - q near -1) would be off by the same part,
// up to 2^-8, and so would be the gradients; numbers just below 1 are rounded by 2^-9 at most.  (Rows of one to three entries:
// dx 0.0029 of its norm off before, 0.0021 since; no time.)
//
// Differences are formed where they keep their digits: log p from a logit's distance to the row's largest, and the
// favourite's p - q, where p is beyond a half, from the sums of the others' q and p.
#include "eager_distillation.h"
#include "eager_joined.h"
#include "eager_launch.h"
#include "eager_model_rules.h"
#include "eager_vector.h"

#include <type_traits>

namespace eager {
namespace {

constexpr int kEntries = 256;
constexpr int kPlaceBits = 13, kPlaces = 1 << kPlaceBits;    // of a row's words, to find equal ones
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
static_assert(kPlaces / 32 == 4 * 64, "four words of bits a lane");

__device__ __forceinline__ bool counts(long long index, float logit) { return (index >= 0) & (logit != -__builtin_inff()); }

// A row's entries, N a lane of a wavefront.
template <int N>
struct List {
    long long index[N];
    float logit[N];
    bool used[N];

    __device__ __forceinline__ List(const TeacherArgs &t, long long row, int lane)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
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
        for (int j = 0; j < N; ++j) t = used[j] ? fmaxf(t, logit[j]) : t;
        return wave_max(t);
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
        for (int j = 0; j < N; ++j) {
            if (!used[j]) continue;
            beyond |= index[j] >= vocab;
            const int rank = 64 * j + lane + (logit[j] == t ? 0 : 1 << 20);
            if (rank < at) at = rank, word = index[j];
        }
        // (ranks are whole numbers below 2^24 but for a missing one's, so fp32 holds them)
        const float best = -wave_max(-static_cast<float>(at));
        const unsigned long long who = __ballot(static_cast<float>(at) == best);
        word = __shfl(word, __builtin_ctzll(who), 64);
        return __any(beyond) ? vocab : word;
    }
};

__device__ __forceinline__ float dot(bf16x8 a, bf16x8 b, float c)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) c = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{a[i], a[i + 1]}, bf16x2{b[i], b[i + 1]}, c, false);
    return c;
}
__device__ __forceinline__ float dot(f32x4 a, f32x4 b, float c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = fmaf(a[i], b[i], c);
    return c;
}

// One row a workgroup.  Eight lanes take an entry, 128 bytes of its word's row at a time, so that rows of any width keep
// them busy and a load covers eight entries; a wavefront has two such sets of entries under way.
template <typename T, int N>
__global__ __launch_bounds__(256) void picked_kernel(const CrossEntropyArgs a, long long *favourite)
{
    constexpr int E = kVector<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), entries = a.teacher.entries;
    const int in = lane >> 3, first = (lane & 7) * E;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const List<N> list(a.teacher, row, lane);
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const bool there = list.used[b] && list.index[b] < a.vocab;
            const unsigned long long known = __ballot(there), used = __ballot(list.used[b]);
            const int word = there ? static_cast<int>(list.index[b]) : 0;
            const int at[2] = {8 * wave + in, 32 + 8 * wave + in};
            const T *w[2];
            float sum[2] = {};
#pragma unroll
            for (int j = 0; j < 2; ++j) w[j] = static_cast<const T *>(a.w) + __shfl(word, at[j], 64) * a.w_stride;
            const bool both = known >> (32 + 8 * wave) & 0xff;
            if (both) {
#pragma unroll 4
                for (int i = first; i < a.width; i += 8 * E) {
                    const auto u = load16(x + i);
#pragma unroll
                    for (int j = 0; j < 2; ++j) sum[j] = dot(u, load16(w[j] + i), sum[j]);
                }
            } else if (known >> (8 * wave) & 0xff) {
#pragma unroll 8
                for (int i = first; i < a.width; i += 8 * E) sum[0] = dot(load16(x + i), load16(w[0] + i), sum[0]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                sum[j] += moved<0xb1>(sum[j]);          // 1 0 3 2
                sum[j] += moved<0x4e>(sum[j]);          // 2 3 0 1
                sum[j] += moved<0x141>(sum[j]);         // 7 - i
                if (first == 0 && 64 * b + at[j] < entries)
                    a.teacher.picked[row * entries + 64 * b + at[j]] =
                        known >> at[j] & 1 ? sum[j] : used >> at[j] & 1 ? __builtin_nanf("") : 0.0f;
            }
        }
        if (wave == 3) {
            const long long word = list.favourite(a.vocab, lane);
            if (lane == 0) favourite[row] = word;
        }
    }
}

// Four rows a workgroup.
template <int N>
__global__ __launch_bounds__(256) void favourites_kernel(const CrossEntropyArgs a, long long *favourite)
{
    const int lane = threadIdx.x & 63;
    for (long long row = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6); row < a.rows; row += 4ll * gridDim.x) {
        const long long word = List<N>(a.teacher, row, lane).favourite(a.vocab, lane);
        if (lane == 0) favourite[row] = word;
    }
}

// Favourites and rows that count in one launch, kGathered rows a workgroup, a wavefront each; all of them look at the lists of
// the rows in front for whether these count.  The whole backward pass, us, beside two launches: 2 x 848 x 469 with 31 entries
// 29.3 for 30.6, 17 x 512 x 3000 with 128 35.4 for 37.1, 61 x 1024 x 50257 with 16 123.4 both; 128 x 512 x 1000 with 64 alike and
// with 256 56 for 51, so up to 64 rows.
template <typename T, int N>
__global__ __launch_bounds__(1024) void taught_rows_kernel(const CrossEntropyArgs a, const Gather g)
{
    __shared__ int sums[16], place[kGathered];
    __shared__ long long words[kGathered];
    static_assert(kGathered == 16, "a wavefront a row");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long first = static_cast<long long>(blockIdx.x) * kGathered;
    const long long word = List<N>(a.teacher, min(first + wave, a.rows - 1), lane).favourite(a.vocab, lane);
    int before = 0;
    for (long long row = wave; row < first; row += 16) {
        const List<N> list(a.teacher, row, lane);
        bool any = false;
#pragma unroll
        for (int j = 0; j < N; ++j) any |= list.used[j];
        before += __any(any) && g.dloss[row] != 0.0f;
    }
    if (lane == 0) words[wave] = word, sums[wave] = before;
    __syncthreads();
    if (wave == 0) {
        before = 0;
        for (int w = 0; w < 16; ++w) before += sums[w];
        place_rows(g, first, before, lane < kGathered ? words[lane] : -1, place);
    }
    __syncthreads();
    move_rows<T>(g, first, place);
}

// kJoined rows a workgroup: their statistics, then a wavefront for each row's entries (whose loads come first).
template <int N, bool Kept>
__global__ __launch_bounds__(1024) void divergence_kernel(const CrossEntropyArgs a, const Tiled t)
{
    __shared__ float2 part[16][kJoined];
    __shared__ float tops[kJoined], logs[kJoined];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + wave, there = min(row, a.rows - 1);
    const List<N> list(a.teacher, there, lane);
    const long long word = Kept ? list.favourite(a.vocab, lane) : t.favourite[there];
    const float right = Kept ? 0.0f : t.right[there];
    float l[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int k = 64 * j + lane;
        if (Kept) {
            const bool known = list.used[j] && list.index[j] < a.vocab;
            l[j] = known ? t.logits[there * t.stride + list.index[j]] : list.used[j] ? __builtin_nanf("") : 0.0f;
            if (row < a.rows && k < a.teacher.entries) a.teacher.picked[row * a.teacher.entries + k] = l[j];
        } else {
            l[j] = list.used[j] ? a.teacher.picked[there * a.teacher.entries + k] : 0.0f;
        }
    }
    const float2 all = joined_statistics(t.stats, a.rows, t.tiles, part);
    if (threadIdx.x < kJoined) {
        const long long mine = static_cast<long long>(blockIdx.x) * kJoined + threadIdx.x;
        const float log_sum = log1pf(all.y - 1.0f);
        tops[threadIdx.x] = all.x, logs[threadIdx.x] = log_sum;
        if (mine < a.rows) a.lse[mine] = fmaf(all.x, kLn2, log_sum);
    }
    __syncthreads();
    if (row >= a.rows) return;
    if (word < 0 || word >= a.vocab) {
        if (lane == 0) a.loss[row] = word < 0 ? 0.0f : __builtin_nanf("");
        return;
    }
    const float top = list.top();
    float sum = 0.0f, e[N], distance[N], loss = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        // logarithms to base two, of q without its sum
        distance[j] = list.used[j] ? (list.logit[j] - top) * t.scale : 0.0f;
        e[j] = list.used[j] ? exp2_fast(distance[j]) : 0.0f;
        sum += e[j];
    }
    sum = lanes_sum<64>(sum);
    const float log_q = log1pf(sum - 1.0f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (!list.used[j]) continue;
        // the favourite's logit is the tiles' own, as the row's largest is
        const float its = !Kept && list.index[j] == word ? right : l[j];
        const float apart = distance[j] - fmaf(its, t.scale, -tops[wave]);
        const float term = e[j] / sum * (fmaf(apart, kLn2, logs[wave]) - log_q);
        loss += e[j] == 0.0f ? 0.0f : term;
    }
    loss = lanes_sum<64>(loss);
    if (lane == 0) a.loss[row] = loss;
}

// kJoined rows a workgroup, a wavefront for each row's entries (whose loads come first).
template <typename T, int N>
__global__ __launch_bounds__(1024) void entries_kernel(const CrossEntropyArgs a, const Entries n)
{
    __shared__ float part[16][kJoined], apart[kJoined];
    __shared__ int words[kJoined][64 * N];
    __shared__ float shares[kJoined][64 * N];
    __shared__ __align__(16) unsigned seen[kJoined][kPlaces / 32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = static_cast<long long>(blockIdx.x) * kJoined + wave, there = min(row, a.rows - 1);
    const int place = row < a.rows ? n.place[there] : -1;
    const List<N> list(a.teacher, there, lane);
    float p[N];
#pragma unroll
    for (int j = 0; j < N; ++j) p[j] = list.used[j] ? a.teacher.picked[there * a.teacher.entries + 64 * j + lane] : 0.0f;
    const int known = max(place, 0);
    const long long word = n.favourite[known];
    const float lse = n.lse[known] * kLog2e, by = n.common ? n.dloss[known] / *n.common : n.dloss[known];
    if (n.others) {
        const long long mine = static_cast<long long>(blockIdx.x) * kJoined + threadIdx.x % kJoined;
        const float sum = joined_sums(n.others, mine < a.rows ? n.place[mine] : -1, a.rows, n.tiles, part);
        if (threadIdx.x < kJoined) apart[threadIdx.x] = sum;
        __syncthreads();
    }
    if (place < 0 || word >= a.vocab) return;            // (beyond the vocabulary: the tiles wrote NaN)
    const float top = list.top();
    float sum = 0.0f, q[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        q[j] = list.used[j] ? exp2_fast((list.logit[j] - top) * n.scale) : 0.0f;
        sum += q[j];
    }
    sum = lanes_sum<64>(sum);
    float rest = 0.0f;                                   // of q, without the favourite's
#pragma unroll
    for (int j = 0; j < N; ++j) {
        q[j] /= sum;
        if (list.used[j] && list.index[j] != word) rest += q[j];
    }
    rest = lanes_sum<64>(rest);
    // which entries find their word's bit set already; one of two equal words does, and few others
    reinterpret_cast<u32x4 *>(seen[wave])[lane] = u32x4{};
    __builtin_amdgcn_wave_barrier();
    unsigned met[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const unsigned at = static_cast<unsigned>(list.index[j]) * 0x9e3779b1u >> (32 - kPlaceBits);
        met[j] = list.used[j] ? atomicOr(&seen[wave][at >> 5], 1u << (at & 31)) >> (at & 31) & 1 : 0;
    }
    bool first[N], several = false;
    float share[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        for (unsigned long long left = __ballot(met[j]); left && !several; left &= left - 1) {
            const int its = __builtin_amdgcn_readlane(static_cast<int>(list.index[j]), __builtin_ctzll(left));
            int equal = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) equal += __popcll(__ballot(list.used[i] && static_cast<int>(list.index[i]) == its));
            several |= equal > 1;
        }
        first[j] = list.used[j] && list.index[j] >= n.first && list.index[j] < n.first + n.live;
        share[j] = q[j];
    }
    // a word that stands in several entries is written by the first of them, with all their shares
    if (several) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            words[wave][64 * j + lane] = list.used[j] ? static_cast<int>(list.index[j]) : -1;
            shares[wave][64 * j + lane] = q[j];
            share[j] = 0.0f;
        }
        __builtin_amdgcn_wave_barrier();
        for (int i = 0; i < a.teacher.entries; ++i) {
            const int word_i = words[wave][i];
            const float share_i = shares[wave][i];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool its = list.used[j] && word_i == static_cast<int>(list.index[j]);
                share[j] += its ? share_i : 0.0f;
                first[j] &= !(its && i < 64 * j + lane);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (!first[j]) continue;
        float d = exp2_fast(fmaf(p[j], n.scale, -lse)) - share[j];
        if (n.others && list.index[j] == word && apart[wave] < 0.5f) d = rest - apart[wave];
        T *const at = static_cast<T *>(n.dl) + place * n.stride + list.index[j] - n.first;
        *at = static_cast<T>(d * by);
        if (n.low) *reinterpret_cast<T *>(reinterpret_cast<char *>(at) + n.low) = static_cast<T>(d * by - static_cast<float>(static_cast<T>(d * by)));
    }
}

unsigned workgroups(long long rows, int each) { return static_cast<unsigned>(std::min((rows + each - 1) / each, kMostBlocks)); }

// Entries a lane: lists of up to 64, 128 and 256.
template <typename F>
hipError_t by_entries(int entries, const F &call)
{
    static_assert(kEntries == 256, "four entries a lane at most");
    if (entries <= 64) return call(std::integral_constant<int, 1>());
    if (entries <= 128) return call(std::integral_constant<int, 2>());
    return call(std::integral_constant<int, 4>());
}

}  // namespace

hipError_t launch_picked(const CrossEntropyArgs &a, long long *favourite, bool bf16, hipStream_t stream)
{
    return by_entries(a.teacher.entries, [&](auto n) {
        return launch(bf16 ? picked_kernel<__bf16, n> : picked_kernel<float, n>, dim3(workgroups(a.rows, 1)), dim3(256), 0, stream, a, favourite);
    });
}

hipError_t launch_favourites(const CrossEntropyArgs &a, long long *favourite, hipStream_t stream)
{
    return by_entries(a.teacher.entries, [&](auto n) {
        return launch(favourites_kernel<n>, dim3(workgroups(a.rows, 4)), dim3(256), 0, stream, a, favourite);
    });
}

hipError_t launch_taught_rows(const CrossEntropyArgs &a, const Gather &g, bool bf16, hipStream_t stream)
{
    return by_entries(a.teacher.entries, [&](auto n) {
        return launch(bf16 ? taught_rows_kernel<__bf16, n> : taught_rows_kernel<float, n>,
                      dim3(static_cast<unsigned>((a.rows + kGathered - 1) / kGathered)), dim3(1024), 0, stream, a, g);
    });
}

hipError_t launch_divergence(const CrossEntropyArgs &a, const Tiled &t, bool kept, hipStream_t stream)
{
    return by_entries(a.teacher.entries, [&](auto n) {
        return launch(kept ? divergence_kernel<n, true> : divergence_kernel<n, false>,
                      dim3(static_cast<unsigned>((a.rows + kJoined - 1) / kJoined)), dim3(1024), 0, stream, a, t);
    });
}

hipError_t launch_entries(const CrossEntropyArgs &a, const Entries &n, bool bf16, hipStream_t stream)
{
    return by_entries(a.teacher.entries, [&](auto each) {
        return launch(bf16 ? entries_kernel<__bf16, each> : entries_kernel<float, each>,
                      dim3(static_cast<unsigned>((a.rows + kJoined - 1) / kJoined)), dim3(1024), 0, stream, a, n);
    });
}

}  // namespace eager
