// Loads and stores of a few consecutive values of a row whose length and start are multiples of nothing, gfx950.
#pragma once

#include <hip/hip_runtime.h>

namespace ppc {

// N consecutive values that start on a multiple of their own size only: rows of any length
template <typename T, int N> struct K8Any { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };
template <typename T> struct K8Any<T, 1> { typedef T type; };

// N values at p, of which `left` are there (the others: 0)
template <typename T, int N> __device__ __forceinline__ void k8_load(const T* p, int left, T (&v)[N]) {
    if (left >= N) {
        const typename K8Any<T, N>::type w = *reinterpret_cast<const typename K8Any<T, N>::type*>(p);
        if constexpr (N == 1) v[0] = w;
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = w[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < left ? p[i] : (T)0.0f;
    }
}
template <typename T, int N> __device__ __forceinline__ void k8_store(T* p, int left, const T (&v)[N]) {
    if (left >= N) {
        typename K8Any<T, N>::type w;
        if constexpr (N == 1) w = v[0];
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = v[i];
        }
        *reinterpret_cast<typename K8Any<T, N>::type*>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = v[i];
    }
}

}  // namespace ppc
