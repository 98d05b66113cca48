// A cache of keys and values held in 8 bits: what its kernels and their callers share (not part of the C ABI).
#pragma once

#include "lm_types.h"

// Scale bytes that count.  The smallest code is 2^-9 and the largest 1.75 2^8, so that with these powers of two every number of the
// cache is one of the type: of bfloat16 a normal one (2^-9 2^-117 = 2^-126, 1.75 2^8 2^119 < 2^128), of fp16 a multiple of 2^-24 up to
// 57344.  For the same reason fp16 numbers that are subnormal lose nothing but their third bit after the first.
template <typename T> struct ScaleRange;
template <> struct ScaleRange<Bf16> { static constexpr int kLo = 10, kHi = 246; };
template <> struct ScaleRange<F16> { static constexpr int kLo = 112, kHi = 134; };

constexpr float kE4m3Max = 448.0f;
template <typename T> __device__ __forceinline__ int scale_byte(int s) { return min(max(s, ScaleRange<T>::kLo), ScaleRange<T>::kHi); }
__device__ __forceinline__ float power_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }      // 2^(byte - 127), byte 1 .. 254

// What fr_kv8_pages promises, as far as the host can see.
inline bool kv8_pages_shape_ok(const fr_kv8_pages& c)
{
    return (c.dtype == FR_DTYPE_BF16 || c.dtype == FR_DTYPE_F16) && (c.head_dim == 64 || c.head_dim == 128) && c.n_kv_heads >= 1 &&
           c.n_kv_heads <= 1024 && c.page_size >= 1 && c.page_size <= 4096 && !(c.page_size & (c.page_size - 1)) && c.block >= 1 &&
           c.block <= 128 && c.block <= c.page_size && !(c.block & (c.block - 1));
}

inline bool kv8_pages_ok(const fr_kv8_pages& c)
{
    if (!kv8_pages_shape_ok(c) || !c.k || !c.v || !c.k_scale || !c.v_scale || (((uintptr_t)c.k | (uintptr_t)c.v) & 15)) return false;
    if (c.n_pages < 1 || c.n_pages > 0x7fffffff) return false;
    for (int64_t s : {c.page_stride, c.head_stride, c.slot_stride})
        if (s < 0 || s > 0x7fffffff || s % 16) return false;
    for (int64_t s : {c.scale_page_stride, c.scale_head_stride, c.scale_block_stride})
        if (s < 0 || s > 0x7fffffff) return false;
    return true;
}
