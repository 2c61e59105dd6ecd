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

// x of the two rows of 16 of a half, and of the two halves of a wavefront, by exchanging rows and halves between two registers.  (Results
// by way of integers: a cast of the second one itself gives the first.)
struct Both {
    float first, second;
};
__device__ __forceinline__ Both exchange_rows(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned even = r[0], odd = r[1];
    return {__builtin_bit_cast(float, even), __builtin_bit_cast(float, odd)};
}
__device__ __forceinline__ Both exchange_halves(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned low = r[0], high = r[1];
    return {__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}

// The sum over `Lanes` neighbouring lanes (16 or 64), the same bits in each of them: pairs, quads, halves and rows of
// 16 inside the vector unit, then rows and halves of the wavefront.  (Through shared memory's permutation, as
// __shfl_xor goes, a step takes some 60 clocks and not 8.)
template <int Lanes>
__device__ __forceinline__ float lanes_sum(float x)
{
    static_assert(Lanes == 16 || Lanes == 64, "a row or a wavefront");
    x += moved<0xb1>(x);        // 1 0 3 2
    x += moved<0x4e>(x);        // 2 3 0 1
    x += moved<0x141>(x);       // 7 - i
    x += moved<0x140>(x);       // 15 - i
    if (Lanes == 16) return x;
    const Both r = exchange_rows(x), h = exchange_halves(r.first + r.second);
    return h.first + h.second;
}

// The same in 64 bits: both words of a number are moved.
template <int Control>
__device__ __forceinline__ double moved(double x)
{
    return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(x), Control, 0xf, 0xf, false),
                            __builtin_amdgcn_mov_dpp(__double2loint(x), Control, 0xf, 0xf, false));
}
__device__ __forceinline__ double rows_sum(double x)
{
    const auto h = __builtin_amdgcn_permlane16_swap(__double2hiint(x), __double2hiint(x), false, false);
    const auto l = __builtin_amdgcn_permlane16_swap(__double2loint(x), __double2loint(x), false, false);
    const unsigned h0 = h[0], h1 = h[1], l0 = l[0], l1 = l[1];
    return __hiloint2double(h0, l0) + __hiloint2double(h1, l1);
}
__device__ __forceinline__ double halves_sum(double x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__double2hiint(x), __double2hiint(x), false, false);
    const auto l = __builtin_amdgcn_permlane32_swap(__double2loint(x), __double2loint(x), false, false);
    const unsigned h0 = h[0], h1 = h[1], l0 = l[0], l1 = l[1];
    return __hiloint2double(h0, l0) + __hiloint2double(h1, l1);
}
template <int Lanes>
__device__ __forceinline__ double lanes_sum(double x)
{
    static_assert(Lanes == 16 || Lanes == 64, "a row or a wavefront");
    x += moved<0xb1>(x);
    x += moved<0x4e>(x);
    x += moved<0x141>(x);
    x += moved<0x140>(x);
    return Lanes == 16 ? x : halves_sum(rows_sum(x));
}

// The largest of a wavefront.
__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, moved<0xb1>(x));
    x = fmaxf(x, moved<0x4e>(x));
    x = fmaxf(x, moved<0x141>(x));
    x = fmaxf(x, moved<0x140>(x));
    const Both r = exchange_rows(x), h = exchange_halves(fmaxf(r.first, r.second));
    return fmaxf(h.first, h.second);
}

}  // namespace eager
