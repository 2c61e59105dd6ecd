// Where things lie in the tiles of eager_matrix.h: plain arithmetic, checked on the CPU.
#pragma once

namespace eager {

// What is applied to the index of a 16-byte chunk in `row` of a tile whose rows hold `Chunks` of them.  Reads take
// the same chunk of 32 rows; the exchange spreads 16 consecutive rows over the 256 bytes of banks, and the four rows
// of a transposing read over different pairs of chunks.
template <int Chunks>
constexpr int exchange(int row)
{
    if (Chunks >= 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    return ((row & 2) << 1) | ((row >> 1) & 2) | ((row >> 3) & 1);
}

// The same by choice: the above, the row's last two bits from bit `Shift` of the index on, or none (fp32 columns, whose
// reads of 32 consecutive values meet no conflict).
constexpr int kOfRows = -1, kNoExchange = -2;
template <int Chunks, int Shift>
constexpr int exchange_of(int row)
{
    static_assert(Shift < 0 || (3 << (Shift < 0 ? 0 : Shift)) < Chunks, "chunks stay in their row");
    return Shift == kOfRows ? exchange<Chunks>(row) : Shift == kNoExchange ? 0 : (row & 3) << (Shift < 0 ? 0 : Shift);
}

constexpr unsigned kOutside = 0x80000000u;     // an offset no descriptor covers

// The length of a descriptor that covers `bytes` from a tile's first row on; a tile's own are at most kOutside: 256 rows, 2^23
// bytes apart.
constexpr unsigned covered(long long bytes) { return bytes <= 0 ? 0 : bytes < kOutside ? static_cast<unsigned>(bytes) : kOutside; }

}  // namespace eager
