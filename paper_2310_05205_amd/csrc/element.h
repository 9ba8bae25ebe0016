// Elements of the learner's tensors on the device: fp16, bf16 and fp32 values
// in short vectors, loaded and stored whatever their alignment, computed in
// 32 bits and rounded to nearest even once, when they are stored.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gear.h"

namespace gear {

template <typename E, int N>
struct Vec {
    typedef E raw __attribute__((ext_vector_type(N)));
    typedef float wide __attribute__((ext_vector_type(N)));
    static_assert(sizeof(raw) == sizeof(E) * N, "no padding");

    typedef uint32_t words __attribute__((ext_vector_type(sizeof(raw) / 4)));
    typedef words loose __attribute__((aligned(sizeof(E))));

    // N elements at p, which need no alignment beyond the element's own; with
    // STREAM past the caches, 5 to 15% faster where tensors exceed them and a wave
    // reads whole lines.
    template <bool STREAM = false>
    static __device__ __forceinline__ raw load(const E* p) {
        if (STREAM) return __builtin_bit_cast(raw, __builtin_nontemporal_load(reinterpret_cast<const loose*>(p)));
        return __builtin_bit_cast(raw, *reinterpret_cast<const loose*>(p));
    }
    static __device__ __forceinline__ void unpack(raw v, float (&f)[N]) {
        const wide w = __builtin_convertvector(v, wide);
#pragma unroll
        for (int j = 0; j < N; j++) f[j] = w[j];
    }
    static __device__ __forceinline__ raw round(const float (&f)[N]) {
        wide w;
#pragma unroll
        for (int j = 0; j < N; j++) w[j] = f[j];
        return __builtin_convertvector(w, raw);
    }
    // With STREAM written past the caches.
    template <bool STREAM = false>
    static __device__ __forceinline__ void store(E* p, const float (&f)[N]) {
        const words v = __builtin_bit_cast(words, round(f));
        if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<loose*>(p));
        else *reinterpret_cast<loose*>(p) = v;
    }
};
template <typename E>
struct Vec<E, 1> {
    typedef E raw;
    template <bool STREAM = false>
    static __device__ __forceinline__ raw load(const E* p) { return *p; }
    static __device__ __forceinline__ void unpack(raw v, float (&f)[1]) { f[0] = (float)v; }
    template <bool STREAM = false>
    static __device__ __forceinline__ void store(E* p, const float (&f)[1]) { *p = (E)f[0]; }
};

// Natural exp by the hardware's base-2 instruction: its relative error grows as
// |x| 2^-24 (the product's rounding).
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Whether the library's float operators take tensors of this type, and its size.
inline int float_bytes(int32_t dtype) {
    return dtype == GEAR_DTYPE_F32 ? 4 : dtype == GEAR_DTYPE_F16 || dtype == GEAR_DTYPE_BF16 ? 2 : 0;
}

}  // namespace gear
