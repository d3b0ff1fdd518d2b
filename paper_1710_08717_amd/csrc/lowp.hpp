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
    typedef T whole __attribute__((ext_vector_type(N)));
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    typedef const type __attribute__((address_space(1))) *source;
    typedef type __attribute__((address_space(1))) *target;
};

// Memory of the device, for the compiler: where it loses sight of a pointer's origin it would use accesses that may be LDS as well, and wait for both.
template <typename T>
using global_ptr = T __attribute__((address_space(1))) *;
template <typename T>
__device__ __forceinline__ global_ptr<T> in_memory(T *p)
{
    return (global_ptr<T>)p;
}

template <typename T, int N>
__device__ __forceinline__ void load_pack(const T *p, acc_of<T> (&v)[N])
{
    if constexpr (N == 1) {
        v[0] = (acc_of<T>)*in_memory(p);
    } else {
        const typename PackOf<T, N>::whole x = *(typename PackOf<T, N>::source)p;
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = (acc_of<T>)x[i];
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const acc_of<T> (&v)[N])
{
    if constexpr (N == 1) {
        *in_memory(p) = (T)v[0];
    } else {
        typename PackOf<T, N>::whole x;
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = (T)v[i];
        *(typename PackOf<T, N>::target)p = x;
    }
}

// A pointer that the compiler does not see through: in a loop it would keep the address of every element of a partial pack in registers of its own.
template <typename T>
__device__ __forceinline__ T *opaque(T *p)
{
    asm("" : "+v"(p));
    return p;
}

// the first `n` of N elements, the rest zero; `n` may be negative
template <typename T, int N>
__device__ __forceinline__ void load_part(const T *p, int n, acc_of<T> (&v)[N])
{
    if (n >= N) {
        load_pack<T, N>(p, v);
    } else {
        p = opaque(p);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = i < n ? (acc_of<T>)in_memory(p)[i] : acc_of<T>(0);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_part(T *p, int n, const acc_of<T> (&v)[N])
{
    if (n >= N) {
        store_pack<T, N>(p, v);
    } else {
        p = opaque(p);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n)
                in_memory(p)[i] = (T)v[i];
    }
}

// as they are in memory, zeros past `n`
template <typename T, int N>
__device__ __forceinline__ typename PackOf<T, N>::whole load_raw(const T *p, int n)
{
    typename PackOf<T, N>::whole x;
    if (n >= N) {
        x = *(typename PackOf<T, N>::source)p;
    } else {
        p = opaque(p);
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = i < n ? in_memory(p)[i] : (T)0;
    }
    return x;
}

template <typename A>
__device__ __forceinline__ A wave_sum(A x)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1)
        x += __shfl_xor(x, m, 64);
    return x;
}


}  // namespace la
