// The launch rules of layer norms and of distillation's workspaces, on the CPU.
#include "../../paper_1908_04207_amd/csrc/eager_model_rules.h"

#include <cstdio>
#include <cstdlib>

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)

int main()
{
    using namespace eager;
    for (int width = 8; width <= kNormWidth; width += 8) {
        const int threads = layer_norm_threads(width);
        // a power of two from 16 lanes to the largest workgroup, 16 values a lane
        CHECK(threads >= 16 && threads <= 1024 && (threads & (threads - 1)) == 0 && threads != 32);
        CHECK(threads * 16 >= width);
        // half as many values a lane where the kernel is launched so
        if (threads == 16 && width <= 128) CHECK(threads * 8 >= width);
        if (threads == 64 && width <= 512) CHECK(threads * 8 >= width);
        for (long long rows : {0ll, 1ll, 3ll, 4ll, 17ll, 511ll, 512ll, 513ll, 2047ll, 8192ll, 70000ll, (1ll << 31) - (1ll << 16)}) {
            const int blocks = layer_norm_blocks(rows, width);
            CHECK(blocks >= 0 && blocks <= 1024 && (blocks > 0) == (rows > 0) && blocks <= rows);
            // a workgroup alone leaves the sums themselves
            CHECK(layer_norm_workspace_bytes(rows, width) == (blocks > 1 ? blocks * 2ll * width * 4 : 0));
        }
    }
    for (long long rows : {0ll, 1ll, 255ll, 4096ll, 1ll << 25})
        for (int width : {8, 1024})
            for (int vocab : {1, 300, 50257})
                for (int bf16 = 0; bf16 < 2; ++bf16)
                    for (int backward = 0; backward < 2; ++backward) {
                        const long long own = teacher_target_bytes(rows);
                        CHECK(own >= rows * 8 && own % 256 == 0);
                        for (int entries : {1, 16, 256}) {
                            const bool kept = !backward && keeps_logits(rows, width, vocab, entries, bf16 ? 2 : 4);
                            const long long first = teacher_bytes(rows, vocab, kept);
                            // quads of every row's logits, in front of statistics on 256 bytes
                            if (kept) CHECK(first >= rows * ((vocab + 3) / 4 * 4) * 4 && first % 256 == 0 && rows * vocab <= 1 << 26);
                            const int bytes = bf16 ? 2 : 4, pieces = backward ? dlogits_pieces(rows, width, vocab, bytes) : 1;
                            long long rest = cross_entropy_workspace_bytes(rows, width, vocab, bf16, backward);
                            if (backward) {
                                // second pieces behind all else, in the same order as the first ones
                                const Cut c = cut_of(rows, width, vocab, bytes, true, pieces);
                                const Layout l = layout_of(c, rows, width, bytes);
                                CHECK(c.piece > 0 && l.others - l.dl >= c.rows_padded * c.piece * bytes && (bf16 || pieces == 1));
                                rest = l.end + (pieces - 1) * c.rows_padded * c.piece * 2;
                            }
                            CHECK(distillation_workspace_bytes(rows, width, vocab, entries, bf16, backward) == first + rest);
                        }
                    }
    std::puts("ok");
    return 0;
}
