// The rules that give the model operators' launches their shape (eager_model_rules.h), over their whole
// range on the CPU.  Built with sanitizers and run by tests/test_model_host.py.
#include "../../paper_1908_04207_amd/csrc/eager_model_rules.h"

#include <cstdio>
#include <cstdlib>

using namespace eager;

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

static unsigned long long state = 1;
static long long draw(long long low, long long high)       // roughly log-uniform
{
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    long long span = high;
    for (int i = (state >> 33) % 12; i > 0; --i) span /= 4;
    span = std::max(low + 1, span);
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    return low + static_cast<long long>((state >> 20) % static_cast<unsigned long long>(span - low + 1));
}

int main()
{
    for (int n = 0; n < 4000; ++n) {
        const long long rows = n % 50 == 0 ? 0 : draw(1, 1 << 21);
        const int width = static_cast<int>(8 * draw(1, 512)), vocab = static_cast<int>(draw(1, 300000));
        for (int bytes = 2; bytes <= 4; bytes += 2) {
            const Cut c = cut_of(rows, width, vocab, bytes);
            CHECK(c.piece > 0 && c.piece % 256 == 0 && c.rows_padded % 256 == 0 && c.rows_padded >= rows);
            CHECK(c.piece - 256 < vocab);                                   // no empty piece
            CHECK(c.dx_slices >= 1 && c.dx_slices <= 32 && c.dw_slices >= 1 && c.dw_slices <= 32);
            CHECK(c.dw_slices == 1 || (c.piece >= vocab && c.gradients == kMedium));
            CHECK(c.logits >= kLarge && c.logits <= kNarrow && (c.gradients == kLarge || c.gradients == kMedium));
            CHECK(c.piece <= 4096 || c.rows_padded * c.piece * bytes <= (1ll << 29));
            // a tile of dl is addressed within 2^31 bytes
            CHECK(c.piece * bytes * 256 < (1ll << 31));
            const Layout l = layout_of(c, rows, width, bytes);
            const long long at[] = {l.dl, l.dx_sums, l.dw_sums, l.x, l.target, l.lse, l.dloss, l.place, l.before, l.counted, l.end};
            const long long size[] = {c.rows_padded * c.piece * bytes, c.dx_slices * rows * width * 4,
                                      c.dw_slices > 1 ? c.dw_slices * c.piece * width * 4 : 0, rows * width * bytes, rows * 8,
                                      rows * 4, rows * 4, rows * 4, (rows + kGathered - 1) / kGathered * 4, 4};
            for (int i = 0; i < 10; ++i) CHECK(at[i] % 256 == 0 && at[i] + size[i] <= at[i + 1]);
            CHECK(cross_entropy_workspace_bytes(rows, width, vocab, bytes == 2, true) == l.end);
            // the forward pass's tiles, whatever their shape, have room for their statistics
            CHECK(cross_entropy_workspace_bytes(rows, width, vocab, bytes == 2, false) >=
                  rows * (round_up(vocab, kSides[logits_shape(std::max(rows, 1ll), width, vocab, bytes)][0]) /
                          kSides[logits_shape(std::max(rows, 1ll), width, vocab, bytes)][0] * 8 + 4));
        }
        const int kv = static_cast<int>(draw(1, 64)), group = static_cast<int>(draw(1, 32));
        const int parts = attention_parts(rows, kv * group, kv, static_cast<int>(draw(1, 5000)));
        CHECK(parts >= 1 && parts <= group && group % parts == 0);
        const int blocks = norm_rope_blocks(rows, kv * group, kv), per = norm_rope_tokens_per_block(kv * group + kv, true);
        CHECK(per >= 1 && blocks <= 1024 && (rows == 0) == (blocks == 0));
        if (rows) CHECK((rows + per - 1) / per >= blocks);
    }
    // every segment's tiles have numbers of their own: floor(e / rows) + i, whatever the lengths
    for (int n = 0; n < 2000; ++n) {
        long long begin = 0, used = -1;
        const int sequences = static_cast<int>(draw(1, 40));
        for (int i = 0; i < sequences + 2; ++i) {
            const long long len = draw(0, 700), first = begin / kAttentionRows + i;
            CHECK(first > used);
            if (len) used = first + (len - 1) / kAttentionRows;
            begin += len;
        }
        CHECK(used < tile_numbers(begin, sequences, kAttentionRows));
    }
    std::puts("ok");
    return 0;
}
