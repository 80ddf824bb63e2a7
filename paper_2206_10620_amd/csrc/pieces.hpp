// Loads and stores of a few consecutive values of a row whose length and start are multiples of nothing, gfx950.
#pragma once

#include <hip/hip_runtime.h>

namespace ppc {

// N consecutive values that start on a multiple of their own size only: rows of any length
template <typename T, int N> struct K8Any { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };
template <typename T> struct K8Any<T, 1> { typedef T type; };

template <typename T, int N> using k8_any = typename K8Any<T, N>::type;
template <typename V, typename T> __device__ __forceinline__ T k8_at(const V& v, int i) {
    if constexpr (sizeof(V) == sizeof(T)) return v;
    else return v[i];
}
template <typename V, typename T> __device__ __forceinline__ void k8_put(V& v, int i, T x) {
    if constexpr (sizeof(V) == sizeof(T)) v = x;
    else v[i] = x;
}

// N values at p, of which `left` are there (the others: 0)
template <typename T, int N> __device__ __forceinline__ k8_any<T, N> k8_load(const T* p, int left) {
    k8_any<T, N> v;
    if (left >= N) {
        v = *reinterpret_cast<const k8_any<T, N>*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) k8_put(v, i, i < left ? p[i] : (T)0.0f);
    }
    return v;
}
template <typename T, int N> __device__ __forceinline__ void k8_store(T* p, int left, const k8_any<T, N>& v) {
    if (left >= N) {
        *reinterpret_cast<k8_any<T, N>*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = k8_at<k8_any<T, N>, T>(v, i);
    }
}

}  // namespace ppc
