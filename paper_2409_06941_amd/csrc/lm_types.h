// Number types of the kernels for text generation (not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "freeride.h"

// Two 16-bit types and float, by the codes of the C ABI: what a kernel loads, and how it goes to 32 bits and back (nearest even).
// Two numbers of 16 bits, kOnes being their exponents' bits: whether both are finite; with 0 for one that is not, where asked for.
template <uint32_t kOnes> struct Finite {
    static __device__ __forceinline__ bool both_finite(uint32_t w) { return (w & kOnes) != kOnes && (w & kOnes << 16) != kOnes << 16; }
    static __device__ __forceinline__ uint32_t finite_or_0(uint32_t w, bool lo, bool hi)
    {
        if (lo && (w & kOnes) == kOnes) w &= 0xffff0000u;
        if (hi && (w & kOnes << 16) == kOnes << 16) w &= 0xffffu;
        return w;
    }
};

struct Bf16 : Finite<0x7f80> {
    typedef uint16_t Bits;
    typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 x8;
    static __device__ __forceinline__ float up(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        const f2 x = {lo, hi};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, b2));
    }
};

struct F16 : Finite<0x7c00> {
    typedef uint16_t Bits;
    typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 x8;
    static __device__ __forceinline__ float up(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const f2 x = {lo, hi};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, h2));
    }
};

struct F32 {
    typedef float Bits;
    static __device__ __forceinline__ float up(float x) { return x; }
};

// Threads of a launch, at most: a dimension of a grid takes less than 2^32 (of more, some workgroups are left out, without an error).
constexpr int64_t kMostThreads = (int64_t)1 << 31;

// What fr_kv_pages promises, as far as the host can see.
inline bool kv_pages_shape_ok(const fr_kv_pages& c)
{
    return (c.dtype == FR_DTYPE_BF16 || c.dtype == FR_DTYPE_F16) && (c.head_dim == 64 || c.head_dim == 128) &&
           c.n_kv_heads >= 1 && c.n_kv_heads <= 1024 && c.page_size >= 1 && c.page_size <= 4096 && !(c.page_size & (c.page_size - 1));
}

inline bool kv_pages_ok(const fr_kv_pages& c)
{
    if (!kv_pages_shape_ok(c) || !c.k || !c.v || (((uintptr_t)c.k | (uintptr_t)c.v) & 15)) return false;
    if (c.n_pages < 1 || c.n_pages > 0x7fffffff) return false;
    for (int64_t s : {c.page_stride, c.head_stride, c.slot_stride})
        if (s < 0 || s > 0x7fffffff || s % 8) return false;
    return true;
}
