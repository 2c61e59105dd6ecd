// What the projection's products (eager_cross_entropy.hip) ask of distillation's own kernels (eager_distillation.hip).
#pragma once

#include "eager_gather.h"
#include "eager_model.h"

namespace eager {

// The backward pass's rows that count, and a piece of their gradients of logits.
struct Entries {
    const int *place;                // per row: its place among those that count, -1: none
    const long long *favourite;      // of a place, as lse and dloss (the latter over the temperature)
    const float *lse, *dloss;
    const float *common;             // factor that dl leaves out, or NULL
    const float *others;             // [tiles][rows]: sums of p without the favourite's, or NULL
    int tiles;
    void *dl;
    long long low;                   // bytes from dl to its second pieces, 0: there are none
    long long stride, first;         // first: word of dl's column 0
    int live;                        // words of the piece
    float scale;                     // log2(e) / temperature
};

// What there is for the losses: the tiles' statistics, and all logits or the favourites' as the tiles have them.
struct Tiled {
    const float2 *stats;             // [tiles][rows]
    const float *right;
    const long long *favourite;
    const float *logits;
    long long stride;                // of the logits
    int tiles;
    float scale;                     // log2(e) / temperature
};

// Student's logits of the entries, and the word that each row's teacher favours: -1 without an entry that counts, the
// vocabulary's size where an index is beyond it.
hipError_t launch_picked(const CrossEntropyArgs &a, long long *favourite, bool bf16, hipStream_t stream);
// The latter alone.
hipError_t launch_favourites(const CrossEntropyArgs &a, long long *favourite, hipStream_t stream);
// Of up to kFewTaught rows those that count, with the latter.
constexpr long long kFewTaught = 64;
hipError_t launch_taught_rows(const CrossEntropyArgs &a, const Gather &g, bool bf16, hipStream_t stream);
// Losses and log-sum-exps; kept: the entries' logits too, from all logits, else launch_picked was before.
hipError_t launch_divergence(const CrossEntropyArgs &a, const Tiled &t, bool kept, hipStream_t stream);
// The entries' gradients of logits in place of those of words that no list has.
hipError_t launch_entries(const CrossEntropyArgs &a, const Entries &n, bool bf16, hipStream_t stream);

}  // namespace eager
