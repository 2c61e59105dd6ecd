// Where things lie in the tiles of the model operators' products (eager_tiles.h), on the CPU with sanitizers.
// Run by tests/test_model_host.py.
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
    std::puts("ok");
    return 0;
}
