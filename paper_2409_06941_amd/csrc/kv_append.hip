// Keys and values of new tokens into a cache of pages, keys and queries rotated by their positions on the way.
//
// A rotated pair (x, y) becomes (x c - y s, y c + x s) with its position's cosine c and sine s, in 32 bits, rounded once.  Every
// element is read and written once and the rest is a few operations, so that memory bounds it: 16384 tokens of 64 + 2 x 8 heads of
// 128, 679 MB in 127 us, 5.33 TB/s (a plain copy reaches 4.6 to 5.2).  A step's few tokens are bound by the launch: 64 of them 4.2 us.

#include <algorithm>

#include "common.h"
#include "lm_types.h"

namespace {

struct AppendArgs {
    fr_kv_pages c;
    const uint16_t *k, *v, *q;
    uint16_t* q_out;
    int64_t k_stride, v_stride, q_stride, q_out_stride, n_slots;
    const int64_t* slot;
    const int32_t* position;
    const float* rotary;
    int32_t n_positions, rotary_dim, style, n_q_heads, page_shift;
};

// One workgroup per token, whose slot, position and row of the table it reads once; a thread takes 16 elements of a head at a time,
// as two pieces of 8 that hold whole pairs of the rotation: pieces c and c + rotary_dim / 16 (halves), neighbouring pieces otherwise.
template <typename T>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a)
{
    const int64_t t = blockIdx.x;
    const int units = a.c.head_dim / 16, heads = a.n_q_heads + 2 * a.c.n_kv_heads;
    const int64_t slot = a.slot[t];
    const bool stored = slot >= 0 && slot < a.n_slots;
    const int64_t at = stored ? (slot >> a.page_shift) * a.c.page_stride + (slot & (a.c.page_size - 1)) * a.c.slot_stride : 0;
    const float* row = nullptr;
    if (a.rotary_dim) {
        const int32_t p = a.position[t];
        row = a.rotary + (int64_t)(p < 0 ? 0 : p < a.n_positions ? p : a.n_positions - 1) * a.rotary_dim;
    }
    for (int x = threadIdx.x; x < heads * units; x += blockDim.x) {
        const int h = x / units, u = x % units;
        const uint16_t* from;
        uint16_t* to;
        if (h < a.n_q_heads) {
            from = a.q + t * a.q_stride + h * a.c.head_dim;
            to = a.q_out + t * a.q_out_stride + h * a.c.head_dim;
        } else {
            if (!stored) continue;
            const bool value = h >= a.n_q_heads + a.c.n_kv_heads;
            const int g = h - a.n_q_heads - (value ? a.c.n_kv_heads : 0);
            from = value ? a.v + t * a.v_stride + g * a.c.head_dim : a.k + t * a.k_stride + g * a.c.head_dim;
            to = static_cast<uint16_t*>(value ? a.c.v : a.c.k) + at + g * a.c.head_stride;
        }
        const bool turned = u * 16 < a.rotary_dim && h < a.n_q_heads + a.c.n_kv_heads, halves = a.style == FR_ROTARY_HALVES && u * 16 < a.rotary_dim;
        const int e0 = halves ? u * 8 : u * 16, e1 = halves ? u * 8 + a.rotary_dim / 2 : u * 16 + 8;
        uint4 b[2] = {*reinterpret_cast<const uint4*>(from + e0), *reinterpret_cast<const uint4*>(from + e1)};
        if (turned) {
            const float *c = row + u * 8, *s = c + a.rotary_dim / 2;
            uint32_t w[8] = {b[0].x, b[0].y, b[0].z, b[0].w, b[1].x, b[1].y, b[1].z, b[1].w};
            if (halves) {
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
        *reinterpret_cast<uint4*>(to + e0) = b[0];
        *reinterpret_cast<uint4*>(to + e1) = b[1];
    }
}

bool row_ok(const void* p, int64_t stride, int64_t width, int32_t n)
{
    return p && !((uintptr_t)p & 15) && stride % 8 == 0 && (n <= 1 || stride >= width) && stride <= ((int64_t)1 << 45);
}

}  // namespace

extern "C" int fr_kv_append(const fr_kv_append_desc* d, void* stream)
{
    if (!d || !kv_pages_ok(d->cache) || d->n_tokens < 0) return FR_ERR_ARG;
    const fr_kv_pages& c = d->cache;
    if (d->n_q_heads < 0 || d->n_q_heads > 1024) return FR_ERR_ARG;
    if (d->rotary_dim < 0 || d->rotary_dim > c.head_dim || d->rotary_dim % 16) return FR_ERR_ARG;
    if (d->style != FR_ROTARY_HALVES && d->style != FR_ROTARY_PAIRS) return FR_ERR_ARG;
    if (d->n_tokens == 0) return FR_OK;
    const int64_t kv = (int64_t)c.n_kv_heads * c.head_dim, qw = (int64_t)d->n_q_heads * c.head_dim;
    if (!d->slot || !row_ok(d->k, d->k_stride, kv, d->n_tokens) || !row_ok(d->v, d->v_stride, kv, d->n_tokens)) return FR_ERR_ARG;
    if (d->n_q_heads && (!row_ok(d->q, d->q_stride, qw, d->n_tokens) || !row_ok(d->q_out, d->q_out_stride, qw, d->n_tokens))) return FR_ERR_ARG;
    if (d->n_q_heads && d->q == d->q_out && d->q_stride != d->q_out_stride && d->n_tokens > 1) return FR_ERR_ARG;
    if (d->rotary_dim && (!d->position || !d->rotary || ((uintptr_t)d->rotary & 15) || d->n_positions < 1)) return FR_ERR_ARG;
    AppendArgs a = {c, (const uint16_t*)d->k, (const uint16_t*)d->v, (const uint16_t*)d->q, (uint16_t*)d->q_out, d->k_stride, d->v_stride,
                    d->q_stride, d->q_out_stride, c.n_pages * (int64_t)c.page_size, d->slot, d->position, d->rotary, d->n_positions,
                    d->rotary_dim, d->style, d->n_q_heads, __builtin_ctz(c.page_size)};
    constexpr int kThreads = 256;
    for (int64_t left = d->n_tokens; left > 0;) {
        const int64_t n = std::min<int64_t>(left, kMostThreads / kThreads);
        if (c.dtype == FR_DTYPE_BF16) hipLaunchKernelGGL(k_kv_append<Bf16>, dim3((unsigned)n), dim3(kThreads), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(k_kv_append<F16>, dim3((unsigned)n), dim3(kThreads), 0, (hipStream_t)stream, a);
        if ((left -= n) == 0) break;
        a.k += n * a.k_stride, a.v += n * a.v_stride, a.slot += n;
        if (a.n_q_heads) a.q += n * a.q_stride, a.q_out += n * a.q_out_stride;
        if (a.rotary_dim) a.position += n;
    }
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}
