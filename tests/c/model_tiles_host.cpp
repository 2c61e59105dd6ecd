// Where things lie in the tiles of the model operators' products (eager_tiles.h) and in a backward pass's workspace, and
// what the rules say of sizes that tests stand on (eager_model_rules.h), on the CPU with sanitizers.
// Run by tests/test_model_host.py.
#include "../../paper_1908_04207_amd/csrc/eager_model_rules.h"
#include "../../paper_1908_04207_amd/csrc/eager_tiles.h"

#include <cstdio>
#include <cstdlib>

using namespace eager;

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

// Every chunk of a row has a place of its own in that row.
template <int Chunks, int Shift>
static void places(int rows)
{
    for (volatile int row = 0; row < rows; row = row + 1) {
        bool used[Chunks] = {};
        for (int chunk = 0; chunk < Chunks; ++chunk) {
            const int at = chunk ^ exchange_of<Chunks, Shift>(row);
            CHECK(at >= 0 && at < Chunks && !used[at]);
            CHECK((row * Chunks + at) * 16 < 160 * 1024);
            used[at] = true;
        }
    }
}

int main()
{
    places<8, kOfRows>(256);             // rows of 128 bytes: vocabulary products, heads of 64 in bf16
    places<16, kOfRows>(64);             // heads of 64 in fp32, of 128 in bf16
    places<32, kOfRows>(64);             // heads of 128 in fp32
    places<32, 2>(64);                   // bf16 columns of 256 and 128 rows
    places<16, 2>(64);
    places<64, kNoExchange>(32);         // fp32 columns
    places<32, kNoExchange>(32);
    // a tile of 256 rows at the largest stride, as wide as the stride, fp32: its last bytes are covered, and the
    // offset that stands for none is not
    const long long stride = (1ll << 21) * 4, bytes = 255 * stride + stride;
    CHECK(covered(bytes) == static_cast<unsigned long long>(bytes));
    CHECK(covered(2 * bytes) <= kOutside && covered(1ll << 40) <= kOutside);
    CHECK(kOutside + 255ull * stride < (1ull << 32));                      // nor after the steps between its rows
    CHECK(covered(0) == 0 && covered(-1) == 0 && covered(-(1ll << 40)) == 0 && covered(16) == 16);
    for (int row = 0; row < 256; ++row) CHECK((exchange_of<32, kNoExchange>(row)) == 0);
    // heads that share keys: in parts, or summed by one workgroup (tests/test_gpu_model_edges.py)
    CHECK(attention_parts(70000, 8, 2, 700) == 1 && attention_parts(66000, 6, 2, 660) == 1);
    CHECK(attention_parts(70000, 4, 1, 700) == 2 && attention_parts(300, 4, 1, 3) == 4);
    // sums of p without the target's: a number a row and tile, while one piece holds the vocabulary
    const long long rows[] = {0, 1, 61, 300, 4096, 8191, 70000};
    const int vocabs[] = {1, 64, 128, 129, 300, 5003, 50257, 250000};
    for (long long n : rows)
        for (int v : vocabs)
            for (int width = 8; width <= 1600; width += 199 * 8)
                for (int size = 2; size <= 4; size += 2) {
                    const Cut c = cut_of(n, width, v, size);
                    const Layout l = layout_of(c, n, width, size);
                    CHECK(c.pieces == (v + c.piece - 1) / c.piece);
                    const long long tiles = (v + kSides[c.logits][0] - 1) / kSides[c.logits][0];
                    CHECK(l.dl + c.rows_padded * c.piece * size <= l.others && l.others <= l.dx_sums);
                    CHECK(c.pieces > 1 || l.others + tiles * n * 4 <= l.dx_sums);
                }
    std::puts("ok");
    return 0;
}
