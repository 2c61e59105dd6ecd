// Matrix instructions and the tiles in shared memory that feed them (gfx950).
//
// One 32x32x16 step is the unit: a lane holds 8 elements of each operand, of row (column)
// lane % 32, at k = 8 * (lane / 32) + 0..7; of the result it holds column lane % 32 and rows
// 8 * (i / 4) + 4 * (lane / 32) + i % 4, i = 0..15.  bf16 takes one instruction for it, fp32 six, on
// operands cut into bf16 pieces in registers.  The order of k inside a step is free as long as both
// operands agree, and both types share every layout below.
//
// Tiles come from global memory straight into shared memory, 16 bytes a lane, through buffer
// descriptors whose length makes reads beyond an operand's end return zeros.  The shared-memory
// side of such a load is contiguous over the wavefront, so the exchange of 16-byte chunks that
// keeps reads free of bank conflicts is applied to the global address.
#pragma once

#include "eager_tiles.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eager {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

typedef __attribute__((address_space(3))) char lds_char;

template <typename T> struct Operand;
template <> struct Operand<__bf16> {
    typedef bf16x8 frag;
    typedef bf16x4 quad;
};
template <> struct Operand<float> {
    typedef f32x8 frag;
    typedef f32x4 quad;
};

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// fp32 operands as three bf16 pieces, each what rounding left of the one before: their sum is the
// operand exactly.  (Magnitudes from 2^128 (1 - 2^-9) on count as infinite, and below 2^-104 the smaller pieces leave the
// range of the instructions that form them: of a result's norm 2e-7 are lost at 2^-112, 4e-5 at 2^-120.)
struct Pieces {
    bf16x8 high, middle, low;
};

// x less its piece: a product of two pairs with an addend, so the pieces need not be unpacked (exact: the
// difference has no more digits than x, and the pair's other element counts nothing); with unpacked pieces 44
// instructions instead of 28 for both cuts, and 15 % more time in attention
__device__ __forceinline__ f32x8 less(f32x8 x, bf16x8 piece)
{
    // (-1, 0) and (0, -1), from registers: as a constant in the instruction the first one is taken for the second
    unsigned low = 0x0000bf80u, high = 0xbf800000u;
    asm("" : "+s"(low), "+s"(high));
    const bf16x2 first = __builtin_bit_cast(bf16x2, low), second = __builtin_bit_cast(bf16x2, high);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const bf16x2 pair = {piece[j], piece[j + 1]};
        x[j] = __builtin_amdgcn_fdot2_f32_bf16(pair, first, x[j], false);
        x[j + 1] = __builtin_amdgcn_fdot2_f32_bf16(pair, second, x[j + 1], false);
    }
    return x;
}

__device__ __forceinline__ Pieces cut(f32x8 x)
{
    Pieces p;
    p.high = __builtin_convertvector(x, bf16x8);
    x = less(x, p.high);
    p.middle = __builtin_convertvector(x, bf16x8);
    x = less(x, p.middle);
    p.low = __builtin_convertvector(x, bf16x8);
    return p;
}

// The product of such operands without the three smallest of the nine products of pieces, together at
// most 2^-23 of the operands' product (two roundings of an fp32 product).  Six instructions of
// 32 clocks, where the fp32 ones take eight of 64; cutting costs 28 vector instructions an operand, which run beside them.
// Measured against the fp32 instructions: attention over 8192 tokens, 16 heads of 64, 1 sequence: forward 1153 us -> 823,
// backward 4091 -> 2853; 16 sequences 95 -> 71 and 365 -> 269; 8 heads of 128, 16 sequences 109 -> 87 and 371 -> 308.
__device__ __forceinline__ f32x16 mma(const Pieces &a, const Pieces &b, f32x16 c)
{
    c = mma(a.low, b.high, c);
    c = mma(a.high, b.low, c);
    c = mma(a.middle, b.middle, c);
    c = mma(a.middle, b.high, c);
    c = mma(a.high, b.middle, c);
    return mma(a.high, b.high, c);
}

__device__ __forceinline__ bf16x8 operand(bf16x8 x) { return x; }
__device__ __forceinline__ Pieces operand(f32x8 x) { return cut(x); }

// Four results rounded to the type of an operand or an output (round to nearest even).
__device__ __forceinline__ bf16x4 to_quad(f32x4 x, __bf16 *) { return __builtin_convertvector(x, bf16x4); }
__device__ __forceinline__ f32x4 to_quad(f32x4 x, float *) { return x; }

// Rows 8t .. 8t+7 of a lane's results (t = 0, 1) as an operand whose k order is that of the
// results: k = 16 t + 8 (j / 4) + 4 (lane / 32) + j % 4.
template <typename T>
__device__ __forceinline__ typename Operand<T>::frag as_operand(const f32x16 &c, int t)
{
    typename Operand<T>::frag f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = static_cast<T>(c[8 * t + j]);
    return f;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *base, unsigned bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00020000);
}

__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t r, char *lds, unsigned offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds), 16, offset, 0, 0, 0);
}

// What this wavefront has asked for in shared memory is there (its loads from global memory are
// waited for); a barrier after it says the same of the other wavefronts'.
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }   // vmcnt(0)

// ---- tiles whose rows are operand rows and hold consecutive k: `Chunks` 16-byte chunks a row.

// Rows of a matrix from `base` on into a tile; rows from rows_left on and chunks from chunks_left on
// are zeros (rows_left may be negative).  stride: bytes.
template <int Rows, int Chunks, int Waves>
__device__ __forceinline__ void stage_rows(char *tile, const char *base, long long stride, int rows_left,
                                           int chunks_left, int wave, int lane)
{
    constexpr int RowsALoad = Waves * 64 / Chunks;
    static_assert(Rows % RowsALoad == 0 && (RowsALoad % 16 == 0 || Chunks > 8), "loads of whole rows, the same exchange in each");
    const int rows = min(max(rows_left, 0), Rows);
    const unsigned step = static_cast<unsigned>(stride);
    const __amdgpu_buffer_rsrc_t r = buffer(base, rows ? (rows - 1) * step + chunks_left * 16 : 0u);
    const int id = wave * 64 + lane, row = id / Chunks;
#pragma unroll
    for (int s = 0; s < Rows / RowsALoad; ++s) {
        const int chunk = (id % Chunks) ^ exchange<Chunks>(row + s * RowsALoad);
        const unsigned at = chunk < chunks_left ? row * step + chunk * 16 : kOutside;
        load_lds16(r, tile + (s * Waves + wave) * 1024, at + s * RowsALoad * step);
    }
}

// Operand of 32 rows from `row0` on, k step `step` (16 elements), from such a tile.
template <int Chunks>
__device__ __forceinline__ bf16x8 read_rows(const char *tile, int row0, int step, int lane, __bf16 *)
{
    const int row = row0 + (lane & 31), chunk = 2 * step + (lane >> 5);
    return *reinterpret_cast<const bf16x8 *>(tile + row * Chunks * 16 + (chunk ^ exchange<Chunks>(row)) * 16);
}
template <int Chunks>
__device__ __forceinline__ f32x8 read_rows(const char *tile, int row0, int step, int lane, float *)
{
    const int row = row0 + (lane & 31), chunk = 4 * step + 2 * (lane >> 5), x = exchange<Chunks>(row);
    const f32x4 a = *reinterpret_cast<const f32x4 *>(tile + row * Chunks * 16 + (chunk ^ x) * 16);
    const f32x4 b = *reinterpret_cast<const f32x4 *>(tile + row * Chunks * 16 + ((chunk + 1) ^ x) * 16);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The transposed operand from such a tile: rows are columns col0 .. col0 + 31 of the tile, k runs
// over tile rows: j = 0..3 of the lane's half from k0 + k_half * (lane / 32) on, j = 4..7 from
// k_quad later.  bf16 has a read for it: 16 lanes get 16 columns of 4 rows.
template <int Chunks, int Shift = kOfRows>
__device__ __forceinline__ bf16x8 read_columns(const char *tile, int col0, int k0, int k_half, int k_quad, int lane,
                                               __bf16 *)
{
    const int i = lane & 15;
    const int chunk = (col0 >> 3) + 2 * ((lane >> 4) & 1) + ((i >> 1) & 1);
    const int row = k0 + k_half * (lane >> 5) + (i >> 2), later = row + k_quad;
    const char *a = tile + row * Chunks * 16 + (chunk ^ exchange_of<Chunks, Shift>(row)) * 16 + (i & 1) * 8;
    const char *b = tile + later * Chunks * 16 + (chunk ^ exchange_of<Chunks, Shift>(later)) * 16 + (i & 1) * 8;
    const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(a));
    const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(b));
    typedef short i16x8 __attribute__((ext_vector_type(8)));
    const i16x8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, z);
}
template <int Chunks, int Shift = kOfRows>
__device__ __forceinline__ f32x8 read_columns(const char *tile, int col0, int k0, int k_half, int k_quad, int lane,
                                              float *)
{
    const int col = col0 + (lane & 31), first = k0 + k_half * (lane >> 5);
    f32x8 f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = first + (j & 3) + (j >> 2) * k_quad;
        f[j] = *reinterpret_cast<const float *>(tile + row * Chunks * 16 +
                                                ((col >> 2) ^ exchange_of<Chunks, Shift>(row)) * 16 + (col & 3) * 4);
    }
    return f;
}

// Tells the compiler's scheduler to issue Reads reads of shared memory evenly among the first three quarters of the next
// Products matrix instructions, so that the last ones arrive before the step after needs them, and Loads loads from
// global memory among all.  Measured in turns, whole calls in bf16, reads among all of them, three quarters, half, a quarter:
// 4096 x 1024 x 50257 forward 463, 450, 446, 447 us, backward 1236, 1226, 1251, 1262; 8191 x 1600 x 50257 1137, 1134, 1132, 1134
// and 3661, 3671, 3740, 3814.
template <int Products, int Reads, int Loads, int I = 0>
__device__ __forceinline__ void spread()
{
    if constexpr (I < Products) {
        constexpr int first = (3 * Products + 3) / 4;
        constexpr int reads = I < first ? (I + 1) * Reads / first - I * Reads / first : 0;
        constexpr int loads = (I + 1) * Loads / Products - I * Loads / Products;
        if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
        if constexpr (loads > 0) __builtin_amdgcn_sched_group_barrier(0x20, loads, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        spread<Products, Reads, Loads, I + 1>();
    }
}

// base-2 exponential and logarithm of the hardware: one unit in the last place for normal results
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

}  // namespace eager
