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

// the sum over `Lanes` neighbouring lanes (a power of two), in each of them
template <int Lanes>
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int m = 1; m < Lanes; m *= 2) x += __shfl_xor(x, m, 64);
    return x;
}

}  // namespace eager
