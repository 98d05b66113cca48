// Keys and values of new tokens into a cache of pages held in 8 bits, keys and queries rotated by their positions on the way.
//
// A block's codes are x 2^(127 - s), rounded to 4 significant bits; its scale s is the least with which no number goes beyond 448, so
// that the largest magnitude of the block's tokens has to be known before the first code: a wavefront has all tokens of a block and head.
// A rotated key is a c - b s.  Its two products are exact in 64 bits, their sum is rounded there and then to an odd number of 32 bits, so
// that scale and code are those of the exact number but for one in 2^50; in 32 bits one code in a million would be its neighbour.
// Every element is read and written once, so that memory bounds it: 16384 tokens of 64 + 2 x 8 heads of 128, 646 MB in 121 us, 5.3 TB/s (a
// plain copy reaches 4.9).  A step's few tokens are bound by latency, four loads that depend on one another and the launch: 64 of them 6 us.

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
    int32_t n_tokens, share;               // tokens, and how many of them a workgroup has whose keys and values it stores
    int64_t stores, first;                 // such workgroups; the first workgroup of this launch
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

struct Raw { uint4 b[2]; };
__device__ __forceinline__ Raw raw_at(const uint16_t* from, const Pieces& p)
{
    return {{*reinterpret_cast<const uint4*>(from + p.e[0]), *reinterpret_cast<const uint4*>(from + p.e[1])}};
}

// Cosines and sines of a lane's eight pairs.
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ Turn turn_at(const Append8Args& a, const Pieces& p, int64_t t, int u)
{
    Turn y = {};
    if (p.turned) {
        const float4 *c = reinterpret_cast<const float4*>(table_row(a, t) + u * 8), *s = reinterpret_cast<const float4*>(table_row(a, t) + u * 8 + a.rotary_dim / 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 f = c[i], g = s[i];
            y.c[4 * i] = f.x, y.c[4 * i + 1] = f.y, y.c[4 * i + 2] = f.z, y.c[4 * i + 3] = f.w;
            y.s[4 * i] = g.x, y.s[4 * i + 1] = g.y, y.s[4 * i + 2] = g.z, y.s[4 * i + 3] = g.w;
        }
    }
    return y;
}

// Four elements of each piece, 4 q .. 4 q + 3 of its eight, as numbers of 32 bits from which codes are rounded as from the exact ones.
template <typename T> __device__ __forceinline__ void numbers(const Raw& of, const Pieces& p, const Turn& by, int q, float (&x)[8])
{
    const uint32_t w[8] = {of.b[0].x, of.b[0].y, of.b[0].z, of.b[0].w, of.b[1].x, of.b[1].y, of.b[1].z, of.b[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = T::up((uint16_t)(w[i / 4 * 4 + 2 * q + i % 4 / 2] >> i % 2 * 16));
    if (!p.turned) return;
    auto turn = [&](float& f, float& g, int i) {
        float c = by.c[i], s = by.s[i];
        asm volatile("" : "+v"(c), "+v"(s));               // (made into 64 bits here: kept so through all heads they take 64 registers)
        const double y = f, z = g, cd = c, sd = s;
        f = to_odd(y * cd - z * sd);
        g = to_odd(z * cd + y * sd);
    };
    if (p.halves) {
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(x[i], x[i + 4], 4 * q + i);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(x[2 * i], x[2 * i + 1], i / 2 * 4 + 2 * q + i % 2);
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
__device__ __forceinline__ uint32_t codes_of(const float* x, float by)
{
    uint32_t y = four_codes(x[0] * by, x[1] * by, x[2] * by, x[3] * by);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabsf(x[i]) < INFINITY)) y |= 0x7fu << i * 8;
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

// How many tokens of a block follow one another from token t on.
__device__ __forceinline__ int run_at(const Append8Args& a, int64_t t, int64_t slot, int lane)
{
    const int most = a.c.block - (int)(slot & (a.c.block - 1));
    if (most == 1) return 1;
    int run = 0;
    for (int i0 = 0; i0 < most; i0 += 64) {
        const int i = i0 + lane;
        const uint64_t same = __ballot(i < most && t + i < a.n_tokens && a.slot[t + i] == slot + i);
        const int n = ~same ? __builtin_ctzll(~same) : 64;
        run += n;
        if (n < 64) break;
    }
    return run;
}

// Keys and values of such a run: of heads `task0`, task0 + step, .. (of K, then of V).  A wavefront's lanes are dealt out over the elements of
// a row, as many rows as the run has, and heads.  kRowsHeld rows of a lane (two: 16 tokens of a block with head_dim 128, 32 with 64) stay in
// registers, with their angles for all heads, and the next head's elements come while those of this one are made into codes; of longer runs (0)
// rows are read twice, once for the scale and once for the codes.
template <typename T, int kRowsHeld> __device__ __forceinline__ void store_run(const Append8Args& a, int64_t t, int64_t slot, int run, int task0, int step, int lane)
{
    const int D = a.c.head_dim, units = D / 16, block = a.c.block, in_block = (int)(slot & (block - 1));
    int rows = 64 / units;
    while (rows > 1 && rows / 2 >= run) rows /= 2;
    const int heads = 64 / (units * rows), u = lane % units, my_row = lane / units % rows, tasks = 2 * a.c.n_kv_heads;
    const int64_t page = slot >> a.page_shift;
    const int first = (int)(slot & (a.c.page_size - 1));
    constexpr bool kLong = kRowsHeld == 0;
    constexpr int kHeld = kRowsHeld, kRoom = kLong ? 1 : kRowsHeld;
    const Pieces turned(a, u, true), plain(a, u, false);
    Turn turn[kRoom];
#pragma unroll
    for (int y = 0; y < kHeld; ++y) turn[y] = turn_at(a, turned, t + min(my_row + y * rows, run - 1), u);
    struct Task {
        const uint16_t* from;
        int64_t stride;
        uint8_t *to, *scale;
        bool there, value;
    };
    auto task_of = [&](int i) {                            // heads of K, then of V
        Task x;
        x.there = i < tasks;
        x.value = i >= a.c.n_kv_heads;
        const int h = x.there ? x.value ? i - a.c.n_kv_heads : i : 0;
        x.from = (x.value ? a.v : a.k) + h * D;
        x.stride = x.value ? a.v_stride : a.k_stride;
        x.to = static_cast<uint8_t*>(x.value ? a.c.v : a.c.k) + page * a.c.page_stride + h * a.c.head_stride;
        x.scale = (x.value ? a.c.v_scale : a.c.k_scale) + page * a.c.scale_page_stride + h * a.c.scale_head_stride + first / block * a.c.scale_block_stride;
        return x;
    };
    auto ask = [&](const Task& x, Raw (&held)[kRoom], int& old) {
#pragma unroll
        for (int y = 0; y < kHeld; ++y) held[y] = raw_at(x.from + (t + min(my_row + y * rows, run - 1)) * x.stride, x.value ? plain : turned);
        old = in_block ? *x.scale : 0;
    };
    Raw next[kRoom];
    int next_old;
    int i = task0 * heads + lane / (units * rows);
    ask(task_of(i), next, next_old);
    for (; __any(i < tasks); i += step * heads) {
        const Task x = task_of(i);
        const Pieces p = x.value ? plain : turned;
        Raw held[kRoom];
#pragma unroll
        for (int y = 0; y < kHeld; ++y) held[y] = next[y];
        const int old = next_old;
        if (__any(i + step * heads < tasks)) ask(task_of(i + step * heads), next, next_old);
        auto each = [&](auto f) {
#pragma unroll
            for (int y = 0; y < kHeld; ++y)
                if (my_row + y * rows < run) f(my_row + y * rows, held[y], turn[y]);
            if constexpr (kLong)
#pragma unroll 1
                for (int r = my_row; r < run; r += rows) f(r, raw_at(x.from + (t + r) * x.stride, p), turn_at(a, p, t + r, u));
        };
        float top = 0.0f;
        each([&](int, const Raw& w, const Turn& by) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float y[8];
                numbers<T>(w, p, by, q, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_magnitude(y[e]));
                __builtin_amdgcn_sched_barrier(0);         // (the next ones' registers are these)
            }
        });
        for (int e = 1; e < units * rows; e *= 2) top = fmaxf(top, __shfl_xor(top, e));
        int s = byte_for<T>(top);
        if (in_block) {
            const int before = scale_byte<T>(old);
            if (before >= s) {
                s = before;
            } else if (x.there) {
                const float by = power_of(max(127 + before - s, 1));       // (2^-126 and less: all but NaN become 0)
                for (int r = my_row; r < block; r += rows) {
                    if (r >= in_block && r < in_block + run) continue;
                    uint4* w = reinterpret_cast<uint4*>(x.to + (int64_t)(first - in_block + r) * a.c.slot_stride + u * 16);
                    const uint4 y = *w;
                    *w = make_uint4(again(y.x, by), again(y.y, by), again(y.z, by), again(y.w, by));
                }
            }
        }
        if (!x.there) continue;
        const float power = power_of(254 - s);
        // (the numbers are made again, not kept: with them, a wavefront's registers leave room for half as many)
#pragma unroll
        for (int y = 0; y < kHeld; ++y)
#pragma unroll
            for (int b = 0; b < 2; ++b) asm volatile("" : "+v"(held[y].b[b].x), "+v"(held[y].b[b].y), "+v"(held[y].b[b].z), "+v"(held[y].b[b].w));
        each([&](int r, const Raw& w, const Turn& by) {
            uint32_t codes[2][2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float y[8];
                numbers<T>(w, p, by, q, y);
                codes[0][q] = codes_of(y, power);
                codes[1][q] = codes_of(y + 4, power);
                __builtin_amdgcn_sched_barrier(0);
            }
            uint8_t* at = x.to + (int64_t)(first + r) * a.c.slot_stride;
            *reinterpret_cast<uint2*>(at + p.e[0]) = make_uint2(codes[0][0], codes[0][1]);
            *reinterpret_cast<uint2*>(at + p.e[1]) = make_uint2(codes[1][0], codes[1][1]);
        });
        if (lane % (units * rows) == 0) *x.scale = (uint8_t)s;
    }
}

template <typename T> __device__ __forceinline__ void turn_queries(const Append8Args& a, int64_t t)
{
    const int D = a.c.head_dim, units = D / 16, half = a.rotary_dim / 2;
    const float* row = table_row(a, t);
    constexpr int kHeld = 2;                               // pieces whose loads are under way at once
    for (int x0 = threadIdx.x; x0 < a.n_q_heads * units; x0 += kHeld * kThreads) {
        Raw held[kHeld];
#pragma unroll
        for (int y = 0; y < kHeld; ++y) {
            const int x = min(x0 + y * kThreads, a.n_q_heads * units - 1);
            held[y] = raw_at(a.q + t * a.q_stride + x / units * D, Pieces(a, x % units, true));
        }
#pragma unroll
        for (int y = 0; y < kHeld; ++y) {
            const int x = x0 + y * kThreads, h = x / units, u = x % units;
            if (x >= a.n_q_heads * units) break;
            const Pieces p(a, u, true);
            const Raw& b = held[y];
            uint32_t w[8] = {b.b[0].x, b.b[0].y, b.b[0].z, b.b[0].w, b.b[1].x, b.b[1].y, b.b[1].z, b.b[1].w};
            if (p.turned) {
                const float *c = row + u * 8, *s = c + half;
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
            }
            uint16_t* to = a.q_out + t * a.q_out_stride + h * D;
            *reinterpret_cast<uint4*>(to + p.e[0]) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(to + p.e[1]) = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}

// The first workgroups take the keys and values, those of `share` tokens (up to 16) each; then comes one per token with its queries.
template <typename T, int kRowsHeld>
__global__ __launch_bounds__(kThreads) void k_kv8_append(Append8Args a)
{
    const int64_t id = a.first + (int64_t)blockIdx.x;
    if (id >= a.stores) {
        turn_queries<T>(a, id - a.stores);
        return;
    }
    // runs that begin with one of the tokens
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t0 = id * a.share, t = t0 + lane;
    const int64_t slot = lane < a.share && t < a.n_tokens ? a.slot[t] : -1, before = lane < a.share && t < a.n_tokens && t > 0 ? a.slot[t - 1] : -1;
    const bool begins = slot >= 0 && slot < a.n_slots && (!(slot & (a.c.block - 1)) || before != slot - 1);
    const uint64_t all = __ballot(begins);
    const bool apart = __popcll(all) >= kWaves;            // a run each for the wavefronts, or its heads
    int n = 0;
    for (uint64_t left = all; left; left &= left - 1, ++n) {
        if (apart && n % kWaves != wave) continue;
        const int i = __ffsll((unsigned long long)left) - 1;
        const int64_t at = (int64_t)((uint64_t)(uint32_t)__shfl((int)(uint32_t)(slot & 0xffffffff), i) | (uint64_t)(uint32_t)__shfl((int)(slot >> 32), i) << 32);
        const int run = run_at(a, t0 + i, at, lane), task0 = apart ? 0 : wave, step = apart ? 1 : kWaves;
        if (kRowsHeld == 1 || run <= kRowsHeld * 64 / (a.c.head_dim / 16)) store_run<T, kRowsHeld>(a, t0 + i, at, run, task0, step, lane);
        else store_run<T, 0>(a, t0 + i, at, run, task0, step, lane);
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
                     d->rotary_dim, d->style, d->n_q_heads, __builtin_ctz(c.page_size), d->n_tokens};
    // A block's tokens are stored by the workgroup that has its first one, so that with blocks of 16 and a token a workgroup 15 of 16 only look; tokens in
    // blocks of their own are one after another where a workgroup has more than four.  32 + 2 x 8 heads of 128, blocks of 16, by 1, 4, 8 and 16 tokens a workgroup:
    //   prompts: 1024 tokens 32, 16, 15, 16 us, 2048 55, 22, 17, 17, 4096 109, 39, 27, 21, 8192 224, 81, 56, 44; of 300 each, 3000 31, 24, 25, 29, 6000 54, 37, 35, 37
    //   a token a sequence: 512 7.4, 8.1, 12.6, 22, 1024 11.6, 9.4, 14.3, 24, 2048 20, 13, 15, 25;  two: 1022 12.5, 14.2, 19.5, 28, 2044 22, 17, 21, 29, 4100 44, 30, 26, 33
    // and 20 + 2 x 5 heads of 64 with blocks of 1: 2048 12.0, 8.4, 9.3, 15.2, 4096 21, 13.8, 13.2, 16.1, 8192 39, 25, 24, 24.  (Other numbers are no faster than these.)
    a.share = d->n_tokens < 1024 ? 1 : d->n_tokens < 4096 ? 4 : d->n_tokens < 8192 ? 8 : 16;
    a.stores = (d->n_tokens + (int64_t)a.share - 1) / a.share;
    const int64_t all = a.stores + (d->n_q_heads ? d->n_tokens : 0);
    for (a.first = 0; a.first < all; a.first += kMostThreads / kThreads) {
        const dim3 grid((unsigned)std::min<int64_t>(all - a.first, kMostThreads / kThreads));
        // Where a lane has one row of a block at most, a kernel with room for no more and no way for longer runs: 124 registers instead of 165, four
        // workgroups a unit instead of three (4099 tokens with a scale each, 5 key heads of 64, 16.8 -> 13.8 us).
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, a); };
        const bool one = c.block <= 64 / (c.head_dim / 16);
        if (c.dtype == FR_DTYPE_BF16) one ? go(k_kv8_append<Bf16, 1>) : go(k_kv8_append<Bf16, 2>);
        else one ? go(k_kv8_append<F16, 1>) : go(k_kv8_append<F16, 2>);
    }
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}
