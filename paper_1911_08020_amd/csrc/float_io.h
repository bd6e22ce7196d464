// Loads and stores of fp32, fp16 and bf16 elements as fp32 values.  Vectors may start at any
// element (global accesses need no alignment on gfx950); a store rounds to nearest even.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "darb.h"

namespace darb {

using half_t = _Float16;
using bf16_t = __bf16;

// Elements of 16 bytes.
template <typename T> constexpr int kVec = 16 / int(sizeof(T));

template <typename T, int V> struct VecOf {
    typedef T Type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <typename T> struct VecOf<T, 1> { typedef T Type; };

template <typename T, int V> struct Loaded {
    typename VecOf<T, V>::Type raw;
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (V == 1) return float(raw);
        else return float(raw[i]);
    }
};

template <typename T, int V> __device__ __forceinline__ Loaded<T, V> load_vec(const T *p) {
    return {*reinterpret_cast<const typename VecOf<T, V>::Type *>(p)};
}

// Keeps the compiler from holding what it has computed from x so far (fp32 values of 16-bit
// elements, say) until x is used again: x itself takes the fewest registers.
template <typename T, int V> __device__ __forceinline__ void forget_uses(Loaded<T, V> &x) {
    if constexpr (sizeof(x.raw) == 16) {
        typedef uint32_t U __attribute__((ext_vector_type(4)));
        U u;
        __builtin_memcpy(&u, &x.raw, 16);
        asm volatile("" : "+v"(u));
        __builtin_memcpy(&x.raw, &u, 16);
    } else if constexpr (sizeof(x.raw) == 4) {
        asm volatile("" : "+v"(x.raw));
    }
}

// STREAM: to memory that nothing reads while it could stay in a cache.
template <typename T, int V, bool STREAM = false> __device__ __forceinline__ void store_vec(T *p, const float (&f)[V]) {
    typename VecOf<T, V>::Type t;
    if constexpr (V == 1) {
        t = T(f[0]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) t[i] = T(f[i]);
    }
    typename VecOf<T, V>::Type *to = reinterpret_cast<typename VecOf<T, V>::Type *>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(t, to);
    else *to = t;
}

// F with the C++ type of a darb_dtype (which the caller has checked).
template <typename F> auto with_type(int dtype, F &&f) {
    if (dtype == DARB_F32) return f(float{});
    if (dtype == DARB_F16) return f(half_t{});
    return f(bf16_t{});
}

}  // namespace darb
