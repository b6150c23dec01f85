// Device-side values of the three types that tensors of the language-model
// operators hold, and their vectors.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace micro {

using f16 = _Float16;
using bf16 = __bf16;

// N consecutive values as one access.  The type's alignment is the element's:
// a global access of up to 16 bytes need not be aligned on gfx950, so rows and
// tensors may start anywhere; aligned ones cost nothing extra.
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[N];
};

template <class T, int N>
__device__ __forceinline__ void load_floats(const T* p, float (&out)[N]) {
    const Pack<T, N> q = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = static_cast<float>(q.v[i]);
}

// x rounded to T, to nearest even.  For binary16 the compiler would otherwise
// join the product or sum that x comes from and this conversion into one
// instruction, which rounds once where the definition rounds twice.
template <class T>
__device__ __forceinline__ T rounded(float x) {
    if constexpr (__is_same(T, f16)) asm("" : "+v"(x));
    return static_cast<T>(x);
}

template <class T, int N>
__device__ __forceinline__ void store_floats(T* p, const float (&in)[N]) {
    Pack<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = rounded<T>(in[i]);
    *reinterpret_cast<Pack<T, N>*>(p) = q;
}

// The same past the caches: for outputs that do not fit them, which would only
// push out what is read next.
template <class T, int N>
__device__ __forceinline__ void stream_floats(T* p, const float (&in)[N]) {
    static_assert(sizeof(T) * N == 16, "one 16-byte store");
    using Words = uint32_t __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(2))) Anywhere {
        Words v;
    };
    Pack<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = rounded<T>(in[i]);
    __builtin_nontemporal_store(__builtin_bit_cast(Words, q), &reinterpret_cast<Anywhere*>(p)->v);
}

}  // namespace micro
