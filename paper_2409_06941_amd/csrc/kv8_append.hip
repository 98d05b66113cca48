// Keys and values of new tokens into a cache of pages held in 8 bits, keys and queries rotated by their positions on the way.
//
// A block's codes are x 2^(127 - s), rounded to 4 significant bits; its scale s is the least with which no number goes beyond 448, so
// that the largest magnitude of the block's tokens has to be known before the first code: a wavefront has all tokens of a block and head.

#include <algorithm>

#include "common.h"
#include "kv8.h"

namespace {

struct Append8Args {
    fr_kv8_pages c;
    const uint16_t *k, *v, *q;
    uint16_t* q_out;
    int64_t k_stride, v_stride, q_stride, q_out_stride, n_slots;
    const int64_t* slot;
    const int32_t* position;
    const float* rotary;
    int32_t n_positions, rotary_dim, style, n_q_heads, page_shift;
    int32_t n_tokens;                      // of the call, and the first of this launch
    int32_t first;
};

constexpr int kThreads = 256, kWaves = kThreads / 64;

// The 32-bit number next to d on the side of zero, with its last bit set where d is not that number: what is rounded to fewer bits
// from it is rounded as from d.
__device__ __forceinline__ float to_odd(double d)
{
    const float f = (float)d;
    if ((double)f == d) return f;
    uint32_t b = __float_as_uint(f);
    if (fabs((double)f) > fabs(d)) b -= 1;             // (an infinity becomes the largest number)
    return __uint_as_float(b | 1);
}

// Sixteen elements of a token and head, as two pieces of 8 that hold whole pairs of the rotation: e[0] and e[1].
struct Pieces {
    int e[2];
    bool turned, halves;
    __device__ __forceinline__ Pieces(const Append8Args& a, int u, bool turns)
    {
        turned = turns && u * 16 < a.rotary_dim;
        halves = a.style == FR_ROTARY_HALVES && u * 16 < a.rotary_dim;
        e[0] = halves ? u * 8 : u * 16;
        e[1] = halves ? u * 8 + a.rotary_dim / 2 : u * 16 + 8;
    }
};

__device__ __forceinline__ const float* table_row(const Append8Args& a, int64_t t)
{
    if (!a.rotary_dim) return nullptr;
    const int32_t p = a.position[t];
    return a.rotary + (int64_t)(p < 0 ? 0 : p < a.n_positions ? p : a.n_positions - 1) * a.rotary_dim;
}

// The elements as numbers of 32 bits from which codes are rounded as from the exact ones.
template <typename T> __device__ __forceinline__ void numbers(const uint16_t* from, const Pieces& p, const float* row, int u, int half, float (&x)[16])
{
    const uint4 b[2] = {*reinterpret_cast<const uint4*>(from + p.e[0]), *reinterpret_cast<const uint4*>(from + p.e[1])};
    const uint32_t w[8] = {b[0].x, b[0].y, b[0].z, b[0].w, b[1].x, b[1].y, b[1].z, b[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[2 * i] = T::up((uint16_t)w[i]), x[2 * i + 1] = T::up((uint16_t)(w[i] >> 16));
    if (!p.turned) return;
    const float *c = row + u * 8, *s = c + half;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float &f = p.halves ? x[i] : x[2 * i], &g = p.halves ? x[i + 8] : x[2 * i + 1];
        const double y = f, z = g, cd = c[i], sd = s[i];
        f = to_odd(y * cd - z * sd);
        g = to_odd(z * cd + y * sd);
    }
}

__device__ __forceinline__ float finite_magnitude(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }

// The least s with 448 2^(s - 127) >= top: 448 is 1.75 2^8, so the exponent less 8, and one more for what is beyond 1.75.
template <typename T> __device__ __forceinline__ int byte_for(float top) { return scale_byte<T>((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8); }

__device__ __forceinline__ float clipped(float y) { return fminf(fmaxf(y, -kE4m3Max), kE4m3Max); }
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(clipped(a), clipped(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clipped(c), clipped(d), lo, true);
}
// Codes of x 2^(127 - s); `by` is that power.
__device__ __forceinline__ uint2 eight_codes(const float* x, float by)
{
    uint2 y = {four_codes(x[0] * by, x[1] * by, x[2] * by, x[3] * by), four_codes(x[4] * by, x[5] * by, x[6] * by, x[7] * by)};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(fabsf(x[i]) < INFINITY)) (i < 4 ? y.x : y.y) |= 0x7fu << (i % 4 * 8);
    return y;
}

// Codes of four numbers of the block again, the scale having grown: `by` = 2^(old - new).
__device__ __forceinline__ uint32_t again(uint32_t w, float by)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    const int x = __builtin_amdgcn_cvt_pk_fp8_f32(lo.x * by, lo.y * by, 0, false);
    uint32_t y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi.x * by, hi.y * by, x, true);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((w >> i * 8 & 0x7f) == 0x7f) y |= 0x7fu << i * 8;
    return y;
}

// One workgroup per token: its queries, and, if a run of tokens of a block begins with it, that run's keys and values, a wavefront a
// head of K or V at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_kv8_append(Append8Args a)
{
    const int64_t t = a.first + (int64_t)blockIdx.x;
    const int D = a.c.head_dim, units = D / 16, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = a.rotary_dim / 2;
    if (a.n_q_heads) {
        const float* row = table_row(a, t);
        for (int x = threadIdx.x; x < a.n_q_heads * units; x += kThreads) {
            const int h = x / units, u = x % units;
            const uint16_t* from = a.q + t * a.q_stride + h * D;
            uint16_t* to = a.q_out + t * a.q_out_stride + h * D;
            const Pieces p(a, u, true);
            uint4 b[2] = {*reinterpret_cast<const uint4*>(from + p.e[0]), *reinterpret_cast<const uint4*>(from + p.e[1])};
            if (p.turned) {
                const float *c = row + u * 8, *s = c + half;
                uint32_t w[8] = {b[0].x, b[0].y, b[0].z, b[0].w, b[1].x, b[1].y, b[1].z, b[1].w};
                if (p.halves) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x0 = T::up((uint16_t)w[i]), x1 = T::up((uint16_t)(w[i] >> 16)), y0 = T::up((uint16_t)w[i + 4]), y1 = T::up((uint16_t)(w[i + 4] >> 16));
                        const float c0 = c[2 * i], c1 = c[2 * i + 1], s0 = s[2 * i], s1 = s[2 * i + 1];
                        w[i] = T::pack(x0 * c0 - y0 * s0, x1 * c1 - y1 * s1);
                        w[i + 4] = T::pack(y0 * c0 + x0 * s0, y1 * c1 + x1 * s1);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x0 = T::up((uint16_t)w[i]), y0 = T::up((uint16_t)(w[i] >> 16));
                        w[i] = T::pack(x0 * c[i] - y0 * s[i], y0 * c[i] + x0 * s[i]);
                    }
                }
                b[0] = make_uint4(w[0], w[1], w[2], w[3]);
                b[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
            *reinterpret_cast<uint4*>(to + p.e[0]) = b[0];
            *reinterpret_cast<uint4*>(to + p.e[1]) = b[1];
        }
    }
    const int64_t slot = a.slot[t];
    if (slot < 0 || slot >= a.n_slots) return;
    const int block = a.c.block, in_block = (int)(slot & (block - 1)), most = block - in_block;
    if (t > 0 && in_block && a.slot[t - 1] == slot - 1) return;        // (the run began before)
    int run = 0;
    for (int i0 = 0; i0 < most; i0 += 64) {
        const int i = i0 + lane;
        const uint64_t same = __ballot(i < most && t + i < a.n_tokens && a.slot[t + i] == slot + i);
        const int n = ~same ? __builtin_ctzll(~same) : 64;
        run += n;
        if (n < 64) break;
    }
    const int64_t page = slot >> a.page_shift;
    const int first = (int)(slot & (a.c.page_size - 1)), at_once = 64 / units, u = lane % units;
    for (int task = wave; task < 2 * a.c.n_kv_heads; task += kWaves) {
        const int h = task >> 1;
        const bool value = task & 1;
        const Pieces p(a, u, !value);
        const uint16_t* from = (value ? a.v : a.k) + h * D;
        const int64_t stride = value ? a.v_stride : a.k_stride;
        uint8_t* to = static_cast<uint8_t*>(value ? a.c.v : a.c.k) + page * a.c.page_stride + h * a.c.head_stride;
        uint8_t* scale = (value ? a.c.v_scale : a.c.k_scale) + page * a.c.scale_page_stride + h * a.c.scale_head_stride + first / block * a.c.scale_block_stride;
        float x[16], top = 0.0f;
        for (int r = lane / units; r < run; r += at_once) {
            numbers<T>(from + (t + r) * stride, p, p.turned ? table_row(a, t + r) : nullptr, u, half, x);
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, finite_magnitude(x[i]));
        }
#pragma unroll
        for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
        int s = byte_for<T>(top);
        if (in_block) {
            const int old = scale_byte<T>(*scale);
            if (old >= s) {
                s = old;
            } else {
                const float by = power_of(max(127 + old - s, 1));      // (2^-126 and less: all but NaN become 0)
                for (int r = lane / (units); r < block; r += at_once) {
                    if (r >= in_block && r < in_block + run) continue;
                    uint4* w = reinterpret_cast<uint4*>(to + (int64_t)(first - in_block + r) * a.c.slot_stride + u * 16);
                    uint4 y = *w;
                    *w = make_uint4(again(y.x, by), again(y.y, by), again(y.z, by), again(y.w, by));
                }
            }
        }
        const float by = power_of(254 - s);
        for (int r = lane / units; r < run; r += at_once) {
            numbers<T>(from + (t + r) * stride, p, p.turned ? table_row(a, t + r) : nullptr, u, half, x);
            uint8_t* at = to + (int64_t)(first + r) * a.c.slot_stride;
            *reinterpret_cast<uint2*>(at + p.e[0]) = eight_codes(x, by);
            *reinterpret_cast<uint2*>(at + p.e[1]) = eight_codes(x + 8, by);
        }
        if (lane == 0) *scale = (uint8_t)s;
    }
}

bool row_ok(const void* p, int64_t stride, int64_t width, int32_t n)
{
    return p && !((uintptr_t)p & 15) && stride % 8 == 0 && stride >= 0 && (n <= 1 || stride >= width) && stride <= ((int64_t)1 << 45);
}

}  // namespace

extern "C" int fr_kv8_append(const fr_kv8_append_desc* d, void* stream)
{
    if (!d || !kv8_pages_ok(d->cache) || d->n_tokens < 0) return FR_ERR_ARG;
    const fr_kv8_pages& c = d->cache;
    if (d->n_q_heads < 0 || d->n_q_heads > 1024) return FR_ERR_ARG;
    if (d->rotary_dim < 0 || d->rotary_dim > c.head_dim || d->rotary_dim % 16) return FR_ERR_ARG;
    if (d->style != FR_ROTARY_HALVES && d->style != FR_ROTARY_PAIRS) return FR_ERR_ARG;
    if (d->n_tokens == 0) return FR_OK;
    const int64_t kv = (int64_t)c.n_kv_heads * c.head_dim, qw = (int64_t)d->n_q_heads * c.head_dim;
    if (!d->slot || !row_ok(d->k, d->k_stride, kv, d->n_tokens) || !row_ok(d->v, d->v_stride, kv, d->n_tokens)) return FR_ERR_ARG;
    if (d->n_q_heads && (!row_ok(d->q, d->q_stride, qw, d->n_tokens) || !row_ok(d->q_out, d->q_out_stride, qw, d->n_tokens))) return FR_ERR_ARG;
    if (d->n_q_heads && d->q == d->q_out && d->q_stride != d->q_out_stride && d->n_tokens > 1) return FR_ERR_ARG;
    if (d->rotary_dim && (!d->position || !d->rotary || ((uintptr_t)d->rotary & 15) || d->n_positions < 1)) return FR_ERR_ARG;
    Append8Args a = {c, (const uint16_t*)d->k, (const uint16_t*)d->v, (const uint16_t*)d->q, (uint16_t*)d->q_out, d->k_stride, d->v_stride,
                     d->q_stride, d->q_out_stride, c.n_pages * (int64_t)c.page_size, d->slot, d->position, d->rotary, d->n_positions,
                     d->rotary_dim, d->style, d->n_q_heads, __builtin_ctz(c.page_size), d->n_tokens, 0};
    for (int64_t left = d->n_tokens; left > 0;) {
        const int64_t n = std::min<int64_t>(left, kMostThreads / kThreads);
        if (c.dtype == FR_DTYPE_BF16) hipLaunchKernelGGL(k_kv8_append<Bf16>, dim3((unsigned)n), dim3(kThreads), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(k_kv8_append<F16>, dim3((unsigned)n), dim3(kThreads), 0, (hipStream_t)stream, a);
        left -= n;
        a.first += (int32_t)n;
    }
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}
