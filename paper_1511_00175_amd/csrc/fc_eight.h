// Eight neighbours of a row at a time, in fp32, whatever the row's type and alignment.
#pragma once

#include <hip/hip_runtime.h>

namespace fc {

// 8 neighbours of a row, which may start at any element: global memory takes any
// alignment.
template <typename T> struct Eight {
    typedef T vec __attribute__((ext_vector_type(8)));
    typedef vec any __attribute__((aligned(alignof(T))));
};
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Up to 8 elements from p on, `left` of them in the row; zeros past it.
template <typename T> __device__ __forceinline__ f32x8 load8(const T* p, int left) {
    if (left >= 8) return __builtin_convertvector(*reinterpret_cast<const typename Eight<T>::any*>(p), f32x8);
    f32x8 v{};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < left) v[e] = (float)p[e];
    return v;
}

// 8 elements in the row's type, all of them in the row.
template <typename T> __device__ __forceinline__ typename Eight<T>::vec raw8(const T* p) { return *reinterpret_cast<const typename Eight<T>::any*>(p); }

template <typename T> __device__ __forceinline__ void put8(T* p, f32x8 v) {
    *reinterpret_cast<typename Eight<T>::any*>(p) = __builtin_convertvector(v, typename Eight<T>::vec);
}

template <typename T> __device__ __forceinline__ void store8(T* p, int left, f32x8 v) {
    if (left >= 8) {
        *reinterpret_cast<typename Eight<T>::any*>(p) = __builtin_convertvector(v, typename Eight<T>::vec);
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < left) p[e] = (T)v[e];
}

}  // namespace fc
