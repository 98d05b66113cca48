// What kernels of attention share: matrix blocks, tiles of keys and values in LDS, the running softmax of a wavefront's rows.
#pragma once

#include <type_traits>

#include "lm_types.h"

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short i16x4;
typedef __attribute__((address_space(3))) char* LdsBytes;
__device__ __forceinline__ LdsBytes lds_at(uint32_t address) { return reinterpret_cast<LdsBytes>(address); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kXcds = 8, kUnits = 256, kThreads = 256, kWaves = 4;
constexpr float kSlack = 8.0f;             // a running maximum may lag behind by a factor of 2^8 in the weights

// The instruction scheduler keeps what stands on either side of this apart.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ int32_t within(int32_t x, int32_t lo, int32_t hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// The largest (the sum) over the lanes l, l + kCols, .. that hold parts of one row.
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
template <int kCols, typename F> __device__ __forceinline__ float over_row(float x, F f)
{
    if constexpr (kCols == 16) {
        const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
        x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int kCols> __device__ __forceinline__ float top_of_row(float x) { return over_row<kCols>(x, [](float y, float z) { return fmaxf(y, z); }); }
template <int kCols> __device__ __forceinline__ float sum_of_row(float x) { return over_row<kCols>(x, [](float y, float z) { return y + z; }); }

__device__ __forceinline__ f32x16 mfma(Bf16::x8 a, Bf16::x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(F16::x8 a, F16::x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(Bf16::x8 a, Bf16::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(F16::x8 a, F16::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// LDS of a workgroup: tiles of keys and values (rows of head_dim elements, 16-byte chunk c of row r at place c ^ f(r)), page ids.
// f keeps the lanes that are served together on different banks: K is read 16 bytes a lane, lanes along rows; V 8 bytes a lane,
// transposed on the way, by 32 columns four rows and 64 bytes at a time, by 16 columns eight rows and 32 bytes.
template <int D, int kCols> struct Lds {
    static constexpr uint32_t kRow = D * 2, kChunks = D / 8, kRowsALoad = 1024 / kRow;
    static constexpr uint32_t kBytes = 512 * D;                   // 64 KB at D = 128: two workgroups share a compute unit
    static __device__ __forceinline__ uint32_t fk(uint32_t r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ uint32_t fv(uint32_t r)
    {
        if (kCols == 16) return D == 128 ? (r & 7) * 2 : (r >> 1 & 3) * 2;
        return D == 128 ? (r & 3) * 4 : (r & 2) * 2;
    }
    // the chunk that a lane loads in load y of rows y * kRowsALoad + lane / kChunks: the one whose place is its own
    static __device__ __forceinline__ uint32_t k_piece(uint32_t lane, int y) { return (lane % kChunks) ^ fk(y * kRowsALoad + lane / kChunks); }
    static __device__ __forceinline__ uint32_t v_piece(uint32_t lane, int y) { return (lane % kChunks) ^ fv(y * kRowsALoad + lane / kChunks); }
};

// The state of kCols query rows in a wavefront: lane l holds row l % kCols, for a part of the keys and of the result's elements (it
// stands transposed in the MFMA blocks' registers: rows of a block are keys or elements, columns are query rows).
template <typename T, int D, int kCols, int kUp = std::is_same_v<T, F16> ? 7 : 0> struct Softmax {
    typedef std::conditional_t<kCols == 32, f32x16, f32x4> Block;
    static constexpr int kInBlock = kCols * kCols / 64, kParts = 64 / kCols;          // elements of a block in a lane; lanes of a row
    Block o[D / kCols];
    float m, l, l1;                        // running maximum of the scores (before the scale); sums of the lane's weights, even and odd keys
    typename T::x8 q[D * kCols / 512];     // kCols x 512 / kCols elements a fragment

    // element of the block that register i of a lane is
    static __device__ __forceinline__ int in_block(int i, int lane) { return i / 4 * 4 * kParts + lane / kCols * 4 + i % 4; }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int d = 0; d < D / kCols; ++d)
#pragma unroll
            for (int i = 0; i < kInBlock; ++i) o[d][i] = 0.0f;
    }
    __device__ __forceinline__ void start()
    {
        m = -INFINITY;
        l = l1 = 0.0f;
        clear();
    }
    // Scores of two blocks of keys: those from `end` on are not seen.
    static __device__ __forceinline__ void hide(Block (&s)[2], int first, int end, int lane)
    {
        if (first + 2 * kCols > end) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < kInBlock; ++i)
                    if (first + b * kCols + in_block(i, lane) >= end) s[b][i] = -INFINITY;
        }
    }
    // A larger maximum, if the one in use lags behind by more than kSlack (m = -infinity: the first keys a row sees).
    __device__ __forceinline__ void grow(float top, float c)
    {
        if (__any((top - m) * c > kSlack)) {
            const float now = fmaxf(top, m), old = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - now) * c);
            m = now;
            l *= old;
            l1 *= old;
#pragma unroll
            for (int d = 0; d < D / kCols; ++d)
#pragma unroll
                for (int i = 0; i < kInBlock; ++i) o[d][i] *= old;
        }
    }
    // What weights are relative to, a power of 2: weights of fp16 end at 2^-25, so they are up to 2^7 (with kSlack 2^15 of the type's
    // nearly 2^16) instead of 1, and those from 2^-32 of the largest on count.
    static constexpr float kLift = kUp;
    __device__ __forceinline__ float reference(float c) const { return m * c - kLift; }
    __device__ __forceinline__ float base(float c) const { return m == -INFINITY ? 0.0f : reference(c); }
    // Two weights for the product with the values, rounded to the type (the matrix cores take 16 bits: half an ulp of a weight is
    // what the result's own rounding costs); their sum is of the weights as they are.
    __device__ __forceinline__ uint32_t weigh(float s0, float s1, float c, float base)
    {
        const float w0 = __builtin_amdgcn_exp2f(fmaf(s0, c, -base)), w1 = __builtin_amdgcn_exp2f(fmaf(s1, c, -base));
        l += w0;
        l1 += w1;
        return T::pack(w0, w1);
    }
    // The same of the scores' distances from the maximum, for scores so large that s c - m c, with m c rounded, would be off by several powers of 2.
    __device__ __forceinline__ float zero_point() const { return m == -INFINITY ? 0.0f : m; }
    __device__ __forceinline__ uint32_t weigh_from(float s0, float s1, float c, float zero)
    {
        const float w0 = __builtin_amdgcn_exp2f(fmaf(s0 - zero, c, kLift)), w1 = __builtin_amdgcn_exp2f(fmaf(s1 - zero, c, kLift));
        l += w0;
        l1 += w1;
        return T::pack(w0, w1);
    }
    // The eight keys of a lane's fragment of weights are twice four neighbours, as they come out of the scores; a transposed read
    // of V takes four neighbouring keys, so that it has the same order.
    static __device__ __forceinline__ typename T::x8 fragment(const uint32_t* w) { return __builtin_bit_cast(typename T::x8, make_uint4(w[0], w[1], w[2], w[3])); }
};

// Where a lane's fragments lie in a tile.  With c = kCols and g = lane / c: of K, row lane % c, elements 512 / c f + 8 g .. + 7 of fragment
// f; of V, transposed, element c d + lane % c of the keys 4 g .. + 3 and 256 / c + 4 g .. + 3.
template <typename T, int D, int kCols> struct Fragments {
    typedef Lds<D, kCols> L;
    typedef const __attribute__((address_space(3))) typename T::x8* Eight;
    typedef __attribute__((address_space(3))) i16x4* Quad;
    uint32_t k, v;                         // of the first fragment; the others' chunks differ in bits that f leaves alone (lds on 1024 bytes)
    __device__ __forceinline__ Fragments(uint32_t lds, int lane)
    {
        const uint32_t r = lane % kCols, i = lane & 15, rv = 4 * (lane / kCols) + (i >> 2);
        k = lds + r * L::kRow + ((uint32_t)(lane / kCols) ^ L::fk(r)) * 16;
        v = lds + rv * L::kRow + ((uint32_t)((lane % kCols >> 4) * 2 + ((i & 3) >> 1)) ^ L::fv(rv)) * 16 + (i & 1) * 8;
    }
    __device__ __forceinline__ typename T::x8 of_k(int tile, int f) const { return *reinterpret_cast<Eight>(lds_at(k ^ (uint32_t)(f * 1024 / kCols)) + tile); }
    __device__ __forceinline__ typename T::x8 of_v(int tile, int d) const
    {                                      // (rows r + 8 and r + 16 have r's order of chunks)
        const LdsBytes at = lds_at(v ^ (uint32_t)(d * 2 * kCols)) + tile;
        struct { i16x4 lo, hi; } y = {__builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<Quad>(at)),
                                      __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<Quad>(at + 256 / kCols * (int)L::kRow))};
        return __builtin_bit_cast(typename T::x8, y);
    }
};

}  // namespace
