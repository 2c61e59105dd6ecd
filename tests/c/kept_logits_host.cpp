// What a distillation's forward pass keeps of the student's logits stays within 256 MiB as it is laid out, on the CPU.
#include "../../paper_1908_04207_amd/csrc/eager_model_rules.h"

#include <cstdio>
#include <cstdlib>

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (rows %lld, vocab %d)\n", __LINE__, #x, rows, vocab); std::exit(1); } } while (0)

int main()
{
    using namespace eager;
    int kept_ones = 0;
    for (long long rows : {1ll, 2ll, 5ll, 61ll, 4096ll, 65536ll, (1ll << 20) - 3, 1ll << 22, 1ll << 23, 1ll << 24, (1ll << 24) + 1, (1ll << 25) - 1, 1ll << 25})
        for (int vocab : {1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 63, 64, 65, 1000, 1023, 1024, 1025, 16385, 50257, 1 << 20, 1 << 26, 1 << 30})
            for (int width : {8, 1024, 1 << 21})
                for (int entries : {1, 64, 256})
                    for (int bytes : {2, 4}) {
                        const bool kept = keeps_logits(rows, width, vocab, entries, bytes);
                        const long long all = rows * ((vocab + 3ll) / 4 * 4) * 4;
                        kept_ones += kept;
                        if (kept) CHECK(all <= 1ll << 28 && teacher_bytes(rows, vocab, kept) >= all && teacher_bytes(rows, vocab, kept) < all + 256);
                        // the workspace holds that beside the cross entropy's arrays and nothing else
                        CHECK(distillation_workspace_bytes(rows, width, vocab, entries, bytes == 2, false) ==
                              teacher_bytes(rows, vocab, kept) + cross_entropy_workspace_bytes(rows, width, vocab, bytes == 2, false));
                    }
    if (!kept_ones) return std::puts("none kept"), 1;
    std::puts("ok");
    return 0;
}
