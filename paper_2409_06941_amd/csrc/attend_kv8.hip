// Attention of a batch of sequences to keys and values held in 8 bits, to all of them or to a window and the first few.
//
// A query row q (a token, a head) that sees keys k_j with values v_j gets  out = sum_j w_j v_j / sum_j w_j,  w_j = exp(s_j - m),
// s_j = scale q . k_j,  and lse = m + log sum_j w_j, m being the largest score so far: where it rises, the sums so far are multiplied by
// exp(m_before - m), so that one pass over the keys is enough.

#include <algorithm>
#include <cmath>

#include "common.h"
#include "kv8.h"

namespace {

struct Attend8Args {
    fr_kv8_pages c;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_stride, out_stride, pages_stride;
    const int32_t *q_begin, *pages, *lens;
    int32_t n_tokens, n_seqs, n_q_heads, max_q, max_len, window, sinks, page_shift, group;
    float scale;
    int64_t first;
};

constexpr int kThreads = 256;

__device__ __forceinline__ int32_t within(int32_t x, int32_t lo, int32_t hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ float code_value(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }

// One workgroup per token and head, 256 keys at a time: a thread a key, then a thread an element.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_attend8(Attend8Args a)
{
    __shared__ float q[D], weight[kThreads], of[kThreads], reduce[kThreads];
    __shared__ uint64_t place[kThreads];
    __shared__ float power[kThreads];
    const int64_t id = a.first + blockIdx.x;
    const int token = (int)(id / a.n_q_heads), head = (int)(id % a.n_q_heads), kv = head / a.group, tid = threadIdx.x;
    int b = token, t0 = token, t1 = token + 1;
    if (a.q_begin) {
        b = 0;
        int end = a.n_seqs;
        while (end - b > 1) {
            const int middle = b + (end - b) / 2;
            if (within(a.q_begin[middle], 0, a.n_tokens) <= token) b = middle;
            else end = middle;
        }
        t0 = within(a.q_begin[b], 0, a.n_tokens), t1 = within(a.q_begin[b + 1], t0, a.n_tokens);
        if (token < t0 || token >= t1 || token - t0 >= a.max_q) return;
    }
    const int len = a.max_len ? within(a.lens[b], 0, a.max_len) : 0, n = max(0, len - (t1 - t0) + 1 + token - t0);
    const int start = a.window ? max(0, n - a.window) : 0, few = min(a.sinks, start);
    if (tid < D) q[tid] = T::up(a.q[token * a.q_stride + (int64_t)head * D + tid]) * a.scale;
    float m = -INFINITY, l = 0.0f, o = 0.0f;
    const int d = tid % D, share = tid / D, shares = kThreads / D;
    for (int j0 = 0; j0 < few + n - start; j0 += kThreads) {
        const int v = j0 + tid, j = v < few ? v : start + v - few;
        float s = -INFINITY;
        __syncthreads();
        if (v < few + n - start) {
            const int32_t page = within(a.pages[b * a.pages_stride + (j >> a.page_shift)], 0, (int32_t)a.c.n_pages - 1);
            const int slot = j & (a.c.page_size - 1), block = slot / a.c.block;
            const uint64_t at = (uint64_t)page * a.c.page_stride + (uint64_t)kv * a.c.head_stride + (uint64_t)slot * a.c.slot_stride;
            const uint64_t sat = (uint64_t)page * a.c.scale_page_stride + (uint64_t)kv * a.c.scale_head_stride + (uint64_t)block * a.c.scale_block_stride;
            const uint8_t* k = (const uint8_t*)a.c.k + at;
            s = 0.0f;
            for (int e = 0; e < D; ++e) s = fmaf(q[e], code_value(k[e]), s);
            s *= power_of(scale_byte<T>(a.c.k_scale[sat]));
            place[tid] = at;
            power[tid] = power_of(scale_byte<T>(a.c.v_scale[sat]));
        }
        reduce[tid] = s;
        __syncthreads();
        float top = m;
        for (int i = 0; i < kThreads; ++i) top = fmaxf(top, reduce[i]);
        const float was = top == -INFINITY ? 1.0f : expf(m - top);
        m = top;
        const float w = s == -INFINITY ? 0.0f : expf(s - m);
        weight[tid] = w;
        __syncthreads();
        l *= was;
        o *= was;
        for (int i = 0; i < kThreads; ++i) l += weight[i];
        const int here = min(kThreads, few + n - start - j0);
        for (int i = share; i < here; i += shares) o = fmaf(weight[i], code_value(((const uint8_t*)a.c.v)[place[i] + d]) * power[i], o);
    }
    __syncthreads();
    of[tid] = o;
    __syncthreads();
    if (tid < D) {
        for (int i = 1; i < shares; ++i) o += of[tid + i * D];
        of[tid] = l == 0.0f ? 0.0f : o / l;
    }
    __syncthreads();
    if (tid < D && tid % 2 == 0)
        *reinterpret_cast<uint32_t*>(a.out + token * a.out_stride + (int64_t)head * D + tid) = T::pack(of[tid], of[tid + 1]);
    if (a.lse && tid == 0) a.lse[(int64_t)token * a.n_q_heads + head] = l == 0.0f ? -INFINITY : m + logf(l);
}

bool sizes_ok(const fr_attend_kv8_desc& d)
{
    if (!kv8_pages_shape_ok(d.cache) || d.n_tokens < 0 || d.n_seqs < 0 || d.max_q < 1) return false;
    if (d.n_q_heads < 1 || d.n_q_heads > 1024 || d.n_q_heads % d.cache.n_kv_heads) return false;
    if ((int64_t)d.n_tokens * d.n_q_heads > 0x7fffffff - 4096) return false;
    return d.max_len >= 0 && d.max_len <= 0x7fffffff - 8191 && d.window >= 0 && d.sinks >= 0;
}

template <typename T, int D> int launch(Attend8Args a, hipStream_t stream)
{
    const int64_t all = (int64_t)a.n_tokens * a.n_q_heads;
    for (a.first = 0; a.first < all; a.first += kMostThreads / kThreads)
        hipLaunchKernelGGL((k_attend8<T, D>), dim3((unsigned)std::min<int64_t>(all - a.first, kMostThreads / kThreads)), dim3(kThreads), 0, stream, a);
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}

}  // namespace

extern "C" {

int fr_attend_kv8_workspace_bytes(const fr_attend_kv8_desc* d, uint64_t* bytes_out)
{
    if (!d || !bytes_out || !sizes_ok(*d)) return FR_ERR_ARG;
    *bytes_out = 0;
    return FR_OK;
}

int fr_attend_kv8(const fr_attend_kv8_desc* d, void* stream)
{
    if (!d || !sizes_ok(*d) || !kv8_pages_ok(d->cache)) return FR_ERR_ARG;
    if (!(d->scale > 0.0f) || std::isinf(d->scale)) return FR_ERR_ARG;
    if (d->n_tokens == 0 || d->n_seqs == 0) return FR_OK;
    const fr_kv8_pages& c = d->cache;
    const int64_t width = (int64_t)d->n_q_heads * c.head_dim, most = (int64_t)1 << 45;
    if (!d->q || !d->out || d->q == d->out || (((uintptr_t)d->q | (uintptr_t)d->out) & 15)) return FR_ERR_ARG;
    for (int64_t s : {d->q_stride, d->out_stride})
        if (s % 8 || s > most || s < 0 || (d->n_tokens > 1 && s < width)) return FR_ERR_ARG;
    if (!d->q_begin && d->n_tokens != d->n_seqs) return FR_ERR_ARG;
    if (d->max_len && (!d->pages || !d->lens || d->pages_stride < ((int64_t)d->max_len + c.page_size - 1) / c.page_size || d->pages_stride > most)) return FR_ERR_ARG;
    const Attend8Args a = {c, (const uint16_t*)d->q, (uint16_t*)d->out, d->lse, d->q_stride, d->out_stride, d->pages_stride, d->q_begin, d->pages, d->lens,
                           d->n_tokens, d->n_seqs, d->n_q_heads, d->q_begin ? d->max_q : 1, d->max_len, d->window, d->sinks,
                           __builtin_ctz(c.page_size), d->n_q_heads / c.n_kv_heads, d->scale, 0};
    hipStream_t s = (hipStream_t)stream;
    if (c.dtype == FR_DTYPE_BF16) return c.head_dim == 64 ? launch<Bf16, 64>(a, s) : launch<Bf16, 128>(a, s);
    return c.head_dim == 64 ? launch<F16, 64>(a, s) : launch<F16, 128>(a, s);
}

}  // extern "C"
