// How the model operators' launches get their shape: plain host code, checked on the CPU.
#pragma once

#include <algorithm>

namespace eager {

inline long long round_up(long long x, long long to) { return (x + to - 1) / to * to; }

constexpr int kUnits = 256;      // compute units
constexpr long long kMostBlocks = 1 << 20;       // of a grid whose workgroups go on in steps of it (threads stay below 2^32)
// A quarter of a large tile takes this of its time (bound by shared memory: three reads for two matrix instructions).
// Measured, three rounds of tiles and 32 more, the 32 whole or in quarters: 2048 rows, width 1024, bf16 135 and 125 us; 1600
// 186 and 171; fp32 661 (of medium tiles) and 612, 1015 and 943.
constexpr double kQuarter = 0.45;

// A workgroup's tile, its wavefronts, and how many workgroups have a compute unit (by their shared memory).
template <int A_, int B_, int WavesA_, int WavesB_, int OfUnit_>
struct TileShape {
    static constexpr int A = A_, B = B_, WavesA = WavesA_, WavesB = WavesB_, Threads = 64 * WavesA * WavesB, OfUnit = OfUnit_;
    static constexpr bool Quartered = A == 256 && B == 256;
};
typedef TileShape<256, 256, 2, 4, 1> Large;
typedef TileShape<256, 64, 4, 2, 1> Quarter;             // of a large one: a last round that is not full
typedef TileShape<128, 128, 2, 2, 2> Medium;
typedef TileShape<128, 64, 4, 1, 3> Narrow;

// What a product costs in a shape of tiles: rounds of as many tiles as run at once, each a number of
// steps of k (128 bytes) and what filling and emptying takes, in microseconds.  Fitted to sweeps of all three; where they
// differ most (rows x width x vocabulary, bf16, forward, Large / Medium / Narrow, us): 1019 x 1024 x 50257 128 / 125 / 146,
// 61 x 1024 x 50257 35 / 27 / 25, 100 x 512 x 3000 21 / 16 / 13; backward, Large / Medium: 4000 x 800 x 500 126 / 77, and 42
// with dw in slices of the rows.
struct Cost {
    double step, rest;
};
template <typename Shape> Cost cost_of(int bytes);
template <> inline Cost cost_of<Large>(int bytes) { return bytes == 2 ? Cost{1.4, 13} : Cost{5.9, 13}; }
template <> inline Cost cost_of<Medium>(int bytes) { return bytes == 2 ? Cost{1.0, 9} : Cost{3.0, 9}; }
template <> inline Cost cost_of<Narrow>(int bytes) { return bytes == 2 ? Cost{0.9, 6} : Cost{2.5, 6}; }

template <typename Shape>
double rounds_of(long long tiles) { return static_cast<double>((tiles + 256 * Shape::OfUnit - 1) / (256 * Shape::OfUnit)); }

// Quarters of large tiles cost what they do behind full rounds; alone they are no better than whole ones, and distillation
// counts them so (bf16, forward and backward, us, large and narrow: 2 x 848 x 469 45.1 and 40.7, 300 x 512 x 3000 61.3 and 57.5,
// 2916 x 288 x 858 66.4 and 63.9).
template <typename Shape>
double logits_time(long long rows, int width, long long vocab, int bytes, bool taught)
{
    const Cost c = cost_of<Shape>(bytes);
    const long long tiles = round_up(rows, Shape::B) / Shape::B * (round_up(vocab, Shape::A) / Shape::A);
    const long long last = Shape::Quartered && (tiles >= kUnits || !taught) ? tiles % kUnits : 0;
    const double rounds = last && last <= kUnits / 4 ? static_cast<double>(tiles / kUnits) + kQuarter : rounds_of<Shape>(tiles);
    return rounds * (round_up(width, 128 / bytes) / (128 / bytes) * c.step + c.rest);
}

// dw and dx of a piece: their tiles follow each other, so only the last round is not full.  They are gone through so many
// times (two where dl is in two pieces).
template <typename Shape>
double gradients_time(long long rows, int width, long long live, int dw_slices, int dx_slices, int bytes, int times)
{
    const Cost c = cost_of<Shape>(bytes);
    const long long depth = 128 / bytes, tiles_w = round_up(width, Shape::A) / Shape::A;
    const double dw = ((rows + depth - 1) / depth + dw_slices - 1) / dw_slices * times * c.step + c.rest;
    const double dx = ((live + depth - 1) / depth + dx_slices - 1) / dx_slices * times * c.step + c.rest;
    const long long dw_tiles = tiles_w * (round_up(live, Shape::B) / Shape::B) * dw_slices;
    const long long dx_tiles = tiles_w * (round_up(rows, Shape::B) / Shape::B) * dx_slices;
    // a slice's sums are written, read and, from the second piece on, read again
    const double sums = (dx_slices * static_cast<double>(rows) + (dw_slices > 1 ? dw_slices * static_cast<double>(live) : 0)) * width * 12;
    return std::max((dw_tiles * dw + dx_tiles * dx) / (256 * Shape::OfUnit) + std::max(dw, dx) / 2, std::max(dw, dx)) + sums / 5e6;
}

// How the backward pass is cut: vocabulary rows of a piece; slices that are summed apart, of a
// piece for dx and, where there is one piece, of the rows for dw; the shapes of tiles.  The fastest cut by
// the above is taken among those whose dl fit 512 MiB; 4096 columns are taken of however many rows (1 GiB in fp32 for 65536).
enum { kLarge, kMedium, kNarrow };
struct Cut {
    long long rows_padded, piece;
    int dx_slices, dw_slices, logits, gradients;
    long long pieces;
};

inline int logits_shape(long long rows, int width, long long vocab, int bytes, bool taught = false)
{
    const double t[3] = {logits_time<Large>(rows, width, vocab, bytes, taught), logits_time<Medium>(rows, width, vocab, bytes, taught),
                         logits_time<Narrow>(rows, width, vocab, bytes, taught)};
    return static_cast<int>(std::min_element(t, t + 3) - t);
}

constexpr int kSides[3][2] = {{Large::A, Large::B}, {Medium::A, Medium::B}, {Narrow::A, Narrow::B}};

inline Cut cut_of(long long rows, int width, int vocab, int bytes, bool taught = false, int times = 1)
{
    const long long padded = round_up(std::max(rows, 1ll), 256);
    const long long fit = std::max(4096ll, (1ll << 29) / bytes / padded / 256 * 256);
    const long long fewest = (vocab + fit - 1) / fit;
    // (what is gone through twice takes more slices while all of them run at once: 61 x 128 x 50257 67 us with 32, 55 with
    // 64; 100 x 64 x 20000 40 with 64, 44 with 256)
    const long long at_once = 256 / (round_up(std::max(rows, 1ll), 128) / 128 * (round_up(width, 128) / 128));
    const int most = times > 1 ? static_cast<int>(std::clamp(at_once, 32ll, 64ll)) : 32;
    Cut best = {padded, 0, 1, 1, 0, 0, 0};
    double least = 0;
    for (long long n = fewest; n < fewest + 6; ++n) {
        const long long piece = round_up((vocab + n - 1) / n, 256), pieces = (vocab + piece - 1) / piece;
        const int shape = logits_shape(rows, width, piece, bytes, taught);
        const double logits = std::min({logits_time<Large>(rows, width, piece, bytes, taught), logits_time<Medium>(rows, width, piece, bytes, taught),
                                        logits_time<Narrow>(rows, width, piece, bytes, taught)});
        for (int dx = 1; dx <= most; dx *= 2)
            for (int dw = 1; dw <= (pieces > 1 ? 1 : 32); dw *= 2)
                for (int g = dw > 1 ? kMedium : kLarge; g <= kMedium; ++g) {
                    const double one = g == kLarge ? gradients_time<Large>(rows, width, piece, dw, dx, bytes, times)
                                                   : gradients_time<Medium>(rows, width, piece, dw, dx, bytes, times);
                    const double last = std::max(0.2, static_cast<double>(vocab - (pieces - 1) * piece) / piece);
                    const double cost = (logits + one) * (pieces > 1 ? pieces - 1 + last : 1);
                    if (!best.piece || cost < least) {
                        least = cost;
                        best = {padded, piece, dx, dw, shape, g, pieces};
                    }
                }
        if (piece == 256) break;
    }
    return best;
}

// Rows that one workgroup of gather_kernel moves, and up to how many rows each of them counts those in front of it
// itself; beyond, it would read more targets than it has data to move.
constexpr int kGathered = 16;
constexpr long long kCountedByEach = 16384;

// Where things are in the backward pass's workspace (bytes from its start).
struct Layout {
    long long dl, others, dx_sums, dw_sums, x, target, lse, dloss, place, before, counted, end;
};

inline Layout layout_of(const Cut &c, long long rows, int width, int bytes)
{
    long long at = 0;
    auto take = [&](long long n) {
        const long long here = at;
        at += round_up(n, 256);
        return here;
    };
    Layout l;
    l.dl = take(c.rows_padded * c.piece * bytes);
    l.others = take(c.pieces == 1 ? c.piece / 128 * rows * 4 : 0);       // a number a row and tile, of 128 at least
    l.dx_sums = take(c.dx_slices * rows * width * 4);
    l.dw_sums = take(c.dw_slices > 1 ? c.dw_slices * c.piece * width * 4 : 0);
    l.x = take(rows * width * bytes);
    l.target = take(rows * 8);
    l.lse = take(rows * 4);
    l.dloss = take(rows * 4);
    l.place = take(rows * 4);
    l.before = take((rows + kGathered - 1) / kGathered * 4);
    l.counted = take(32);        // the number, and the factor that weights have in common
    l.end = at;
    return l;
}

inline long long cross_entropy_workspace_bytes(long long rows, int width, int vocab, bool bf16, bool backward)
{
    if (!backward) return round_up(rows * (round_up(vocab, 128) / 128 * 8 + 4), 16) + 16;
    const int bytes = bf16 ? 2 : 4;
    return layout_of(cut_of(rows, width, vocab, bytes), rows, width, bytes).end;
}

// Distillation: the word that each row's teacher favours, in front of the forward pass's statistics and behind the backward
// pass's arrays.
inline long long teacher_target_bytes(long long rows) { return round_up(rows * 8, 256); }

// The forward pass: whether all logits are kept, in fp32, and the entries' taken from them, or these are formed before as
// dot products of their own.  Keeping them costs their bytes at 4 to 8 TB/s in the products' epilogue; forming them, a
// launch and the projection's rows at 10 to 20 TB/s.  Measured, us of the whole pass, formed and kept: 8191 x 1600 x 1000
// in bf16 with 64 entries 118 and 46; 300 x 512 x 3000 with 128 20.8 and 17.0; one row x 1024 x 50257 with one 28.6 and
// 25.8; 4096 x 1024 x 8192 with 64 109 and 99; 61 x 1024 x 50257 with 16 30.4 and 29.8; 4096 x 1024 x 50257 with 64 459 and
// 637, 1019 rows 131 and 169; 4096 x 328 x 8000 in fp32 with 4 146 and 155.
// 256 MiB of logits, in rows of whole quads, are the most that are kept, as this operator is for logits that are not to be stored.
inline bool keeps_logits(long long rows, int width, int vocab, int entries, int bytes)
{
    const double formed = 4 + static_cast<double>(rows) * entries * width * bytes / 12e6, kept = static_cast<double>(rows) * round_up(vocab, 4);
    return kept <= 1 << 26 && kept * 4 / 4e6 < formed;
}

// In front of the forward pass's arrays: the logits, or the favourites.
inline long long teacher_bytes(long long rows, int vocab, bool kept)
{
    return kept ? round_up(rows * round_up(vocab, 4) * 4, 256) : teacher_target_bytes(rows);
}

// The backward pass with bf16 inputs: whether dl goes into the products rounded to bf16, or in two pieces, the second what
// the first one's rounding left.  The roundings of many entries average, to 0.0024 of the gradients' norm beside 0.0017 of
// their own rounding; of few rows a few entries decide, and one in eight such batches had gradients 1.5 to 2.3 times as far
// off as their own rounding.  Two pieces leave that one alone.  The backward pass, one piece and two, us: 2 x 848 x 469 29.3 and
// 30.7; 159 x 312 x 330 29.4 and 31.6; 61 x 1024 x 50257 99 and 124; 500 x 1024 x 8192, which stays with one, 71 and 93.
inline int dlogits_pieces(long long rows, int width, int vocab, int bytes)
{
    return bytes == 2 && (rows <= 128 || static_cast<double>(rows) * width * vocab <= 1 << 29) ? 2 : 1;
}

inline long long distillation_workspace_bytes(long long rows, int width, int vocab, int entries, bool bf16, bool backward)
{
    const int bytes = bf16 ? 2 : 4;
    if (!backward)
        return teacher_bytes(rows, vocab, keeps_logits(rows, width, vocab, entries, bytes)) +
               cross_entropy_workspace_bytes(rows, width, vocab, bf16, false);
    const int pieces = dlogits_pieces(rows, width, vocab, bytes);
    const Cut c = cut_of(rows, width, vocab, bytes, true, pieces);
    return layout_of(c, rows, width, bytes).end + teacher_target_bytes(rows) + (pieces - 1) * c.rows_padded * c.piece * bytes;
}

// Heads a workgroup takes at a time: two a group of lanes with 4 lanes a head in the forward pass,
// four in the backward pass, which keeps sums from turn to turn (8192 tokens of 20 heads of 64 in bf16:
// forward 11.0 us, 12.6 with 256; backward 15.8 us, 20.6 with 128).
inline int norm_rope_tokens_per_block(int heads, bool backward)
{
    const int want = backward ? 256 : 128;
    return heads >= want ? 1 : want / heads;
}

// Workgroups of the backward pass: at most 1024, each with the same number of turns.
inline int norm_rope_blocks(long long tokens, int q_heads, int kv_heads)
{
    const int per = norm_rope_tokens_per_block(q_heads + kv_heads, true);
    const long long all = (tokens + per - 1) / per, rounds = (all + 1023) / 1024;
    return static_cast<int>(all ? (all + rounds - 1) / rounds : 0);
}

// Numbers of a packed batch's tiles (eager_packed.h), of kAttentionRows rows each in every attention kernel.
constexpr int kAttentionRows = 128;
inline long long tile_numbers(long long tokens, int sequences, int rows) { return tokens / rows + sequences + 2; }

// Of the keys' kernel in bf16 with heads of up to 64 two workgroups have a compute unit, 512 run at once (of its other forms one
// and 256), and about four rounds of them even out what a causal mask leaves to each.  Measured (16 heads of 64, 4 of keys, 16 sequences of 8192 tokens, bf16): 4 parts 50 us and
// 12 for their sums, 2 parts (of a limit of 600) 62 and 8.
inline int attention_parts(long long tokens, int q_heads, int kv_heads, int sequences)
{
    const int group = q_heads / kv_heads;
    const long long workgroups = tile_numbers(tokens, sequences, kAttentionRows) * kv_heads;
    int parts = 1;
    while (parts < group && workgroups * parts < 2048)
        do ++parts; while (group % parts);
    return parts;
}

// The backward pass: both its kernels in one launch (true), or dq's and then the keys'. One launch has both tails at once
// and runs one kernel's long rows beside the other's; two leave dq's kernel its own registers and so more wavefronts a
// SIMD. Measured, apart and in one launch, us, by dq's workgroups * dim (bf16 unless said): 1000 tokens as 1 sequence, 8
// heads of 128 (9216) 83 and 55; 4000 as 1, 16 of 64 (33792) 181 and 152; the same as 4 (36864) 65 and 60; 4000 as 4, 8 of 128 (36864) 90 and 68; 6000 as 2, 16 of 64 (49152) 160 and 164; 6000 as 12,
// 8 of 128 (59392) 73 and 76; 8192 as 16, 16 of 64 (81920) 80 and 85.
inline bool attention_together(long long workgroups, int dim) { return workgroups * dim <= 40960; }

inline long long attention_row_bytes(long long tokens, int q_heads) { return (tokens * q_heads * 4 + 15) / 16 * 16; }

inline long long attention_workspace_bytes(long long tokens, int q_heads, int kv_heads, int dim, int sequences)
{
    const int parts = attention_parts(tokens, q_heads, kv_heads, sequences);
    return 2 * attention_row_bytes(tokens, q_heads) + (parts > 1 ? parts * 2ll * kv_heads * tokens * dim * 4 : 0);
}

// Lanes that hold a row of a layer norm, 16 values each: 16 (four rows a wavefront), a wavefront or several.
constexpr int kNormWidth = 16384;
inline int layer_norm_threads(int width)
{
    if (width <= 256) return 16;
    int threads = 64;
    while (threads * 16 < width) threads *= 2;
    return threads;
}

// Workgroups of its forward pass, which go on in steps of them: as many as run at once.  Measured, 1024, 2048, 4096 of them and one
// for each of the rows' groups: 20011 x 1600 fp32 109, 102, 103, 105 us; 3000 x 8192 fp32 76.8, 76.7, 79.4, 80.6; 8192 x 1024 bf16 14.2,
// 13.3, 13.4, 13.3.
constexpr long long kNormBlocks = 2048;

// Threads of a workgroup of its backward pass (more where a row takes more), and workgroups: one a compute unit, each of
// which leaves 2 width sums.  Measured, both kernels, 256 and 512 workgroups: 8192 x 1024 bf16 19.1 and 23.6 us, 2047 x 8192
// 33.3 and 41.9, 20011 x 1600 fp32 102 and 105, 65536 x 64 bf16 15.0 and 14.0; 256 threads and 512 workgroups 19.3 us, 37.4, 113;
// 1024 threads spill (47.2, 88.3, 338).  Two rows under way instead of one: 19.4, 31.8 against 33.3, 104, and 3000 x 8192 fp32 97 against 87.
// Rows of up to four turns are gone through by one workgroup, which leaves the sums themselves and needs no second kernel: a
// call of 32 x 1024 bf16 7.3 us and 9.9 with one workgroup for 8 rows (on the GPU alone 7.8 and 7.5), 128 x 64 7.1 and 9.8 (5.7, 6.6),
// 16 x 1600 fp32 8.5 and 10.0 (9.5, 8.4); 64 x 1024 in eight turns 10.7 and 10.0 (11.6, 7.5).
constexpr int kNormBackwardBlock = 512;
inline int layer_norm_blocks(long long rows, int width)
{
    const int groups = std::max(kNormBackwardBlock / layer_norm_threads(width), 1);
    if (rows > 0 && rows <= 4 * groups) return 1;
    return static_cast<int>(std::min<long long>((rows + groups - 1) / groups, kUnits));
}

inline long long layer_norm_workspace_bytes(long long rows, int width)
{
    const int blocks = layer_norm_blocks(rows, width);
    return blocks > 1 ? blocks * 2ll * width * 4 : 0;
}

// Heads that one thread of a rotation takes one after the other, with the position's angles in its registers.  Measured, 1,
// 2, 4 and 5 of them, us: 8192 tokens of 16 + 4 heads of 64 in bf16, half of each rotated 13.5, 10.5, 10.4, 11.0; 20011 of 25 + 25
// in fp32 97, 101, 106, 106; 61 of 16 + 4 in bf16 3.8, 4.0, 4.6, 5.2; 16384 of 8 + 2 of 128 23.0, 18.8, 18.5, 19.6.
constexpr int kTurnedHeads = 2;

// Workgroups of its table, each with several positions: 131072 positions of 64 pairs 15.7 us, 17.7 with one each.
constexpr long long kTableBlocks = 2048;

}  // namespace eager
