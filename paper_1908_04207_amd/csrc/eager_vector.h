// 16 bytes of a row at a time as fp32 values, and sums over the lanes that share a row.
#pragma once

#include "eager_matrix.h"

namespace eager {

template <typename T> struct Vector;
template <> struct Vector<__bf16> { typedef bf16x8 type; };
template <> struct Vector<float> { typedef f32x4 type; };
template <typename T> constexpr int kVector = 16 / sizeof(T);

template <typename T>
__device__ __forceinline__ typename Vector<T>::type load16(const T *p) { return *reinterpret_cast<const typename Vector<T>::type *>(p); }

template <typename T>
__device__ __forceinline__ void store16(T *p, const float *x)
{
    typename Vector<T>::type v;
#pragma unroll
    for (int i = 0; i < kVector<T>; ++i) v[i] = static_cast<T>(x[i]);
    *reinterpret_cast<typename Vector<T>::type *>(p) = v;
}

template <int Control>
__device__ __forceinline__ float moved(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), Control, 0xf, 0xf, false));
}

// The sum over `Lanes` neighbouring lanes (16 or 64), the same bits in each of them: pairs, quads, halves and rows of
// 16 inside the vector unit, rows and halves of the wavefront by exchanging them between two registers.  (Through shared
// memory's permutation, as __shfl_xor goes, a step takes some 60 clocks and not 8.)
template <int Lanes>
__device__ __forceinline__ float lanes_sum(float x)
{
    static_assert(Lanes == 16 || Lanes == 64, "a row or a wavefront");
    x += moved<0xb1>(x);        // 1 0 3 2
    x += moved<0x4e>(x);        // 2 3 0 1
    x += moved<0x141>(x);       // 7 - i
    x += moved<0x140>(x);       // 15 - i
    if (Lanes == 16) return x;
    // (results by way of integers: a cast of the second one itself gives the first)
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned even = rows[0], odd = rows[1];
    x = __builtin_bit_cast(float, even) + __builtin_bit_cast(float, odd);
    const unsigned v = __builtin_bit_cast(unsigned, x);
    const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const unsigned low = halves[0], high = halves[1];
    return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
}

}  // namespace eager
