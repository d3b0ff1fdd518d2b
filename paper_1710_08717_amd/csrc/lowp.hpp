// Element types of the sequence-layer operators (layer norm, clipping, the gated delta rule): 16-bit storage, arithmetic in 32 bits (64 for double).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace la {

using bf16_t = __bf16;
using f16_t = _Float16;

template <typename T>
struct AccOf {
    using type = float;
};
template <>
struct AccOf<double> {
    using type = double;
};
template <typename T>
using acc_of = typename AccOf<T>::type;

// N elements that one lane loads or stores at once.  Memory is read and written at any element's address: the hardware takes
// vector loads and stores off their own alignment.
template <typename T, int N>
struct PackOf {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T>
struct PackOf<T, 1> {
    typedef T type;
};
template <typename T, int N>
using pack_t = typename PackOf<T, N>::type;

template <typename T, int N>
__device__ __forceinline__ void load_pack(const T *p, acc_of<T> (&v)[N])
{
    if constexpr (N == 1) {
        v[0] = (acc_of<T>)*p;
    } else {
        const pack_t<T, N> x = *reinterpret_cast<const pack_t<T, N> *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = (acc_of<T>)x[i];
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const acc_of<T> (&v)[N])
{
    if constexpr (N == 1) {
        *p = (T)v[0];
    } else {
        pack_t<T, N> x;
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = (T)v[i];
        *reinterpret_cast<pack_t<T, N> *>(p) = x;
    }
}

// the first `n` of N elements, the rest zero; `n` may be negative
template <typename T, int N>
__device__ __forceinline__ void load_part(const T *p, int n, acc_of<T> (&v)[N])
{
    if (n >= N) {
        load_pack<T, N>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = i < n ? (acc_of<T>)p[i] : acc_of<T>(0);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_part(T *p, int n, const acc_of<T> (&v)[N])
{
    if (n >= N) {
        store_pack<T, N>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n)
                p[i] = (T)v[i];
    }
}

template <typename A>
__device__ __forceinline__ A wave_sum(A x)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1)
        x += __shfl_xor(x, m, 64);
    return x;
}

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace la
