// Attention of a batch of sequences behind a shared prefix, keys and values in a cache of pages.

#include <cmath>

#include "common.h"
#include "lm_types.h"

namespace {

struct AttendArgs {
    fr_kv_pages c;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_stride, out_stride, pages_stride;
    const int32_t *q_begin, *prefix_pages, *pages, *own_len;
    int32_t n_tokens, n_seqs, n_q_heads, max_q, prefix_len, max_own_len, page_shift, group;
    float scale;
};

__device__ __forceinline__ int32_t within(int32_t x, int32_t lo, int32_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// One wavefront per token and query head: keys in rounds of 64, a lane each.
template <typename T, int D>
__global__ __launch_bounds__(64) void k_attend(AttendArgs a)
{
    const int lane = threadIdx.x, head = blockIdx.y, kv = head / a.group, b = blockIdx.z, i = blockIdx.x;
    const int t0 = a.q_begin ? within(a.q_begin[b], 0, a.n_tokens) : b, t1 = a.q_begin ? within(a.q_begin[b + 1], t0, a.n_tokens) : b + 1;
    if (i >= t1 - t0) return;
    const int own = a.max_own_len ? within(a.own_len[b], 0, a.max_own_len) : 0;
    int seen = own - (t1 - t0) + 1 + i;
    seen = a.prefix_len + (seen < 0 ? 0 : seen);
    const int token = t0 + i;
    const uint16_t* q = a.q + token * a.q_stride + (int64_t)head * D;
    auto at = [&](int j) {
        const int32_t x = j < a.prefix_len ? j : j - a.prefix_len;
        const int32_t id = j < a.prefix_len ? a.prefix_pages[x >> a.page_shift] : a.pages[b * a.pages_stride + (x >> a.page_shift)];
        return within(id, 0, (int32_t)a.c.n_pages - 1) * a.c.page_stride + kv * a.c.head_stride + (x & (a.c.page_size - 1)) * a.c.slot_stride;
    };
    float m = -INFINITY, total = 0.0f, acc[D / 64];
    for (int x = 0; x < D / 64; ++x) acc[x] = 0.0f;
    for (int j0 = 0; j0 < seen; j0 += 64) {
        const int n = seen - j0 < 64 ? seen - j0 : 64;
        const int64_t mine = at(lane < n ? j0 + lane : j0);
        float s = -INFINITY;
        if (lane < n) {
            const uint16_t* k = static_cast<const uint16_t*>(a.c.k) + mine;
            s = 0.0f;
            for (int x = 0; x < D; ++x) s += T::up(q[x]) * T::up(k[x]);
            s *= a.scale;
        }
        float top = s;
        for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
        top = fmaxf(top, m);
        const float base = top == -INFINITY ? 0.0f : top, p = expf(s - base), old = expf(m - base);
        float sum = p;
        for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        total = total * old + sum;
        m = top;
        for (int x = 0; x < D / 64; ++x) acc[x] *= old;
        for (int j = 0; j < n; ++j) {
            const float w = __shfl(p, j);
            const int64_t where = __shfl(mine, j);
            for (int x = 0; x < D / 64; ++x) acc[x] += w * T::up(static_cast<const uint16_t*>(a.c.v)[where + x * 64 + lane]);
        }
    }
    for (int x = 0; x < D / 64; ++x)
        a.out[token * a.out_stride + (int64_t)head * D + x * 64 + lane] = (uint16_t)T::pack(seen ? acc[x] / total : 0.0f, 0.0f);
    if (a.lse && lane == 0) a.lse[(int64_t)token * a.n_q_heads + head] = seen ? m + logf(total) : -INFINITY;
}

bool sizes_ok(const fr_attend_desc& d)
{
    if (!kv_pages_shape_ok(d.cache) || d.n_tokens < 0 || d.n_seqs < 0 || d.max_q < 1) return false;
    if (d.n_q_heads < 1 || d.n_q_heads > 1024 || d.n_q_heads % d.cache.n_kv_heads) return false;
    return d.prefix_len >= 0 && d.max_own_len >= 0 && (int64_t)d.prefix_len + d.max_own_len < 0x7fffffff - 4096;
}

}  // namespace

extern "C" {

int fr_attend_shared_workspace_bytes(const fr_attend_desc* d, uint64_t* bytes_out)
{
    if (!d || !bytes_out || !sizes_ok(*d)) return FR_ERR_ARG;
    *bytes_out = 0;
    return FR_OK;
}

int fr_attend_shared(const fr_attend_desc* d, void* stream)
{
    if (!d || !sizes_ok(*d) || !kv_pages_ok(d->cache)) return FR_ERR_ARG;
    if (!(d->scale > 0.0f) || std::isinf(d->scale)) return FR_ERR_ARG;
    if (d->n_tokens == 0 || d->n_seqs == 0) return FR_OK;
    const fr_kv_pages& c = d->cache;
    const int64_t width = (int64_t)d->n_q_heads * c.head_dim, most = (int64_t)1 << 45;
    if (!d->q || !d->out || d->q == d->out || (((uintptr_t)d->q | (uintptr_t)d->out) & 15)) return FR_ERR_ARG;
    for (int64_t s : {d->q_stride, d->out_stride})
        if (s % 8 || s > most || s < 0 || (d->n_tokens > 1 && s < width)) return FR_ERR_ARG;
    if (!d->q_begin && (d->n_tokens != d->n_seqs)) return FR_ERR_ARG;
    if (d->prefix_len && !d->prefix_pages) return FR_ERR_ARG;
    if (d->max_own_len && (!d->pages || !d->own_len || d->pages_stride < ((int64_t)d->max_own_len + c.page_size - 1) / c.page_size || d->pages_stride > most))
        return FR_ERR_ARG;
    AttendArgs a = {c, (const uint16_t*)d->q, (uint16_t*)d->out, d->lse, d->q_stride, d->out_stride, d->pages_stride, d->q_begin, d->prefix_pages,
                    d->pages, d->own_len, d->n_tokens, d->n_seqs, d->n_q_heads, d->max_q, d->prefix_len, d->max_own_len, __builtin_ctz(c.page_size),
                    d->n_q_heads / c.n_kv_heads, d->scale};
    const dim3 grid((unsigned)d->max_q, (unsigned)d->n_q_heads, (unsigned)d->n_seqs);
    if (c.dtype == FR_DTYPE_BF16) {
        if (c.head_dim == 64) hipLaunchKernelGGL((k_attend<Bf16, 64>), grid, dim3(64), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((k_attend<Bf16, 128>), grid, dim3(64), 0, (hipStream_t)stream, a);
    } else {
        if (c.head_dim == 64) hipLaunchKernelGGL((k_attend<F16, 64>), grid, dim3(64), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((k_attend<F16, 128>), grid, dim3(64), 0, (hipStream_t)stream, a);
    }
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}

}  // extern "C"
