// Pages copied inside the caches of a model's layers.
//
// Every byte of a page is read and written once: memory bounds it (701 pages of 64 KB in 16 caches, 1.47 GB read and written, 274 us, 5.4 TB/s; a
// plain copy 4.9), and a launch where pages are few (24 pages of 16 caches 7.9 us).  A thread has one piece of 16 bytes under way: with four the
// large copy takes 361 us.

#include <algorithm>

#include "common.h"
#include "kv8.h"

namespace {

constexpr int kThreads = 256, kCachesALaunch = 64;

// Where an array of a cache has the bytes of a page: rows of `row` bytes, n0 x n1 of them.
struct Shape {
    int64_t page_stride, s0, s1;
    int32_t n0, n1, row, grain;            // grain: bytes moved at a time, 16 or 1
};

struct CopyArgs {
    Shape codes, scales;                   // (scales.row 0: there are none)
    int64_t n_pages;
    const int32_t *source, *target;
    int32_t* copied;
    int32_t n_pairs, n_caches, share;      // share: caches of a workgroup
    char* k[kCachesALaunch];
    char* v[kCachesALaunch];
    char* ks[kCachesALaunch];
    char* vs[kCachesALaunch];
};

template <typename X> __device__ __forceinline__ void copy_rows(char* base, const Shape& s, int64_t from, int64_t to)
{
    const char* x = base + from * s.page_stride;
    char* y = base + to * s.page_stride;
    const int a_row = s.row / (int)sizeof(X), all = s.n0 * s.n1 * a_row;
    const bool whole = s.n0 * s.n1 == 1;                   // (rows that lie side by side are one: no division)
    auto place = [&](int i) {
        if (whole) return (int64_t)i * (int)sizeof(X);
        const int r = i / a_row;
        return (int64_t)(r / s.n1) * s.s0 + (int64_t)(r % s.n1) * s.s1 + (int64_t)(i % a_row) * (int)sizeof(X);
    };
    for (int i = threadIdx.x; i < all; i += kThreads) *reinterpret_cast<X*>(y + place(i)) = *reinterpret_cast<const X*>(x + place(i));
}

__device__ __forceinline__ void copy_array(char* base, const Shape& s, int64_t from, int64_t to)
{
    if (s.grain == 16) copy_rows<uint4>(base, s, from, to);
    else copy_rows<uint8_t>(base, s, from, to);
}

// Two workgroups per pair and share of the caches, for K and for V.  Whether the pair is carried out is found by a look at all others.
__global__ __launch_bounds__(kThreads) void k_copy_pages(CopyArgs a)
{
    const int i = blockIdx.x % a.n_pairs, of = blockIdx.x / a.n_pairs;
    const bool value = of & 1;
    const int32_t from = a.source[i], to = a.target[i];
    bool out = from < 0 || to < 0 || from >= a.n_pages || to >= a.n_pages || from == to;
    if (!out) {
        bool hit = false;
        for (int j = threadIdx.x; j < a.n_pairs; j += kThreads) {
            const int32_t y = a.target[j];
            if (j == i || (y != to && y != from)) continue;
            const int32_t x = a.source[j];
            if (x < 0 || x >= a.n_pages || x == y) continue;          // (y is one of this pair's pages: inside)
            hit |= y == from || j > i;
        }
        out = __syncthreads_or(hit);
    }
    if (a.copied && of == 0 && threadIdx.x == 0) a.copied[i] = !out;
    if (out) return;
    for (int c = (of >> 1) * a.share, end = min(c + a.share, a.n_caches); c < end; ++c) {
        copy_array(value ? a.v[c] : a.k[c], a.codes, from, to);
        if (a.scales.row) copy_array(value ? a.vs[c] : a.ks[c], a.scales, from, to);
    }
}

// Rows that lie side by side become one; the largest piece that all addresses are multiples of.
Shape shape_of(int64_t page_stride, int64_t s0, int n0, int64_t s1, int n1, int row, uintptr_t bases)
{
    if (n0 == 1 || (n1 > 1 && s0 < s1)) std::swap(s0, s1), std::swap(n0, n1);
    if (n1 == 1 || s1 == row) {
        row *= n1;
        s1 = s0, n1 = n0, s0 = 0, n0 = 1;
        if (n1 == 1 || s1 == row) row *= n1, s1 = 0, n1 = 1;
    }
    const bool wide = !((bases | (uintptr_t)page_stride | (uintptr_t)(n0 > 1 ? s0 : 0) | (uintptr_t)(n1 > 1 ? s1 : 0) | (uintptr_t)row) & 15);
    return {page_stride, s0, s1, n0, n1, row, wide ? 16 : 1};
}

bool same(const Shape& a, const Shape& b)
{
    return a.page_stride == b.page_stride && a.s0 == b.s0 && a.s1 == b.s1 && a.n0 == b.n0 && a.n1 == b.n1 && a.row == b.row && a.grain == b.grain;
}

}  // namespace

extern "C" int fr_kv_copy_pages(const fr_kv_copy_desc* d, void* stream)
{
    if (!d || d->n_caches < 0 || d->n_caches8 < 0 || d->n_caches > 4096 || d->n_caches8 > 4096 || d->n_pairs < 0 || d->n_pairs > 1 << 16) return FR_ERR_ARG;
    if ((d->n_caches && !d->caches) || (d->n_caches8 && !d->caches8)) return FR_ERR_ARG;
    int64_t n_pages = 0;
    for (int i = 0; i < d->n_caches; ++i) {
        if (!kv_pages_ok(d->caches[i]) || (n_pages && d->caches[i].n_pages != n_pages)) return FR_ERR_ARG;
        n_pages = d->caches[i].n_pages;
    }
    for (int i = 0; i < d->n_caches8; ++i) {
        if (!kv8_pages_ok(d->caches8[i]) || (n_pages && d->caches8[i].n_pages != n_pages)) return FR_ERR_ARG;
        n_pages = d->caches8[i].n_pages;
    }
    if (d->n_pairs == 0 || !n_pages) return FR_OK;
    if (!d->source || !d->target) return FR_ERR_ARG;
    CopyArgs a = {};
    a.n_pages = n_pages;
    a.source = d->source, a.target = d->target, a.copied = d->copied, a.n_pairs = d->n_pairs;
    // One cache a workgroup, more where there are so many pairs that looking at them takes as long as copying a page.  16 caches, one for every 256, 512, 1024 pairs
    // and one always: pages of 2 KB, 1024 pairs 33, 46, 71, 71 us, 2048 54, 68, 104, 176, 16384 1001, 1001, 1001, 5630; of 16 KB 202, 199, 197, 197, 419, 407, 400,
    // 428, 3472, 3472, 3469, 8796.
    a.share = std::max(1, d->n_pairs / 512);
    auto go = [&] {
        const int shares = (a.n_caches + a.share - 1) / a.share;          // (2^23 / 2 pairs a launch are at least 64 of the most that a call has)
        for (int done = 0; done < shares; done += kMostThreads / kThreads / 2 / a.n_pairs) {
            CopyArgs x = a;
            const int first = done * a.share, n = (int)std::min<int64_t>(a.n_caches - first, kMostThreads / kThreads / 2 / a.n_pairs * a.share);
            x.n_caches = n;
            for (int c = 0; c < n; ++c) x.k[c] = a.k[first + c], x.v[c] = a.v[first + c], x.ks[c] = a.ks[first + c], x.vs[c] = a.vs[first + c];
            hipLaunchKernelGGL(k_copy_pages, dim3((unsigned)((n + a.share - 1) / a.share) * a.n_pairs * 2), dim3(kThreads), 0, (hipStream_t)stream, x);
        }
        a.n_caches = 0;
        a.copied = nullptr;
    };
    auto add = [&](const Shape& codes, const Shape& scales, void* k, void* v, void* ks, void* vs) {
        if (a.n_caches == kCachesALaunch || (a.n_caches && !(same(a.codes, codes) && same(a.scales, scales)))) go();
        a.codes = codes, a.scales = scales;
        a.k[a.n_caches] = (char*)k, a.v[a.n_caches] = (char*)v, a.ks[a.n_caches] = (char*)ks, a.vs[a.n_caches] = (char*)vs;
        ++a.n_caches;
    };
    for (int i = 0; i < d->n_caches; ++i) {
        const fr_kv_pages& c = d->caches[i];
        add(shape_of(c.page_stride * 2, c.head_stride * 2, c.n_kv_heads, c.slot_stride * 2, c.page_size, c.head_dim * 2, (uintptr_t)c.k | (uintptr_t)c.v), Shape{},
            c.k, c.v, nullptr, nullptr);
    }
    for (int i = 0; i < d->n_caches8; ++i) {
        const fr_kv8_pages& c = d->caches8[i];
        add(shape_of(c.page_stride, c.head_stride, c.n_kv_heads, c.slot_stride, c.page_size, c.head_dim, (uintptr_t)c.k | (uintptr_t)c.v),
            shape_of(c.scale_page_stride, c.scale_head_stride, c.n_kv_heads, c.scale_block_stride, c.page_size / c.block, 1, (uintptr_t)c.k_scale | (uintptr_t)c.v_scale),
            c.k, c.v, c.k_scale, c.v_scale);
    }
    if (a.n_caches) go();
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}
