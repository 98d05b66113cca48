// One token for every row of logits, from a given random number: temperature, top-k, top-p and min-p.
//
// The entries kept are a prefix of the row in falling order, so nothing is sorted: the prefix' end is searched for, digit by
// digit, by histograms of the entries' counts and masses.  Masses are 64-bit integers, whose sums do not depend on the order of
// the additions.  The first digit is a step of 1/64 on the scale of (m - l) / temperature, over which a language model's logits
// spread evenly (equal digits of a float's bits would put thousands of entries on one counter); the rest are digits of the
// logit's bits, in an order that rises with the logit.

#include <cmath>

#include "common.h"
#include "lm_types.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2 * kThreads, kMostVocab = 1 << 19;
constexpr float kMassOne = 8796093022208.0f;           // 2^43: the sum over 2^19 entries stays below 2^63
constexpr uint32_t kMinusInf = 0x007fffffu;            // key of -infinity

struct SampleArgs {
    const void* logits;
    int64_t row_stride;
    int32_t n_vocab;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t* top_k;
    int32_t* token;
};

__device__ __forceinline__ float cleaned(float x) { return x == x ? x + 0.0f : -INFINITY; }      // (-0 becomes 0)
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

struct Scale {
    float top, per_t;
    __device__ __forceinline__ float weight(float x) const
    {
        if (x == top) return 1.0f;
        if (x == -INFINITY) return 0.0f;
        return expf((x - top) * per_t);
    }
    __device__ __forceinline__ uint64_t mass(float w) const { return w > 0.0f ? (uint64_t)(w * kMassOne) : 0; }
    __device__ __forceinline__ uint32_t bin(float x) const
    {
        if (x == top) return 0;
        return (uint32_t)fminf((top - x) * per_t * 64.0f, (float)(kBins - 1));      // (a NaN from 0 * infinity gives the last bin)
    }
};

struct Found { uint32_t digit, count_before, count; uint64_t mass_before, mass; };

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    __shared__ uint64_t mass[kBins > kMostVocab / 64 ? kBins : kMostVocab / 64];
    __shared__ uint32_t count[kBins];
    __shared__ uint64_t wave_mass[kWaves], wave_key[kWaves];
    __shared__ uint32_t wave_count[kWaves];
    __shared__ Found found;
    __shared__ uint32_t shared_index;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.n_vocab;
    const int64_t r = blockIdx.x;
    const typename T::Bits* row = static_cast<const typename T::Bits*>(a.logits) + r * a.row_stride;
    auto at = [&](int i) { return cleaned(T::up(row[i])); };

    // the largest logit, the lowest index of equals
    uint64_t best = 0;
    for (int i = tid; i < V; i += kThreads) {
        const uint64_t x = (uint64_t)key_of(at(i)) << 32 | (uint32_t)~i;
        best = x > best ? x : best;
    }
    for (int x = 1; x < 64; x *= 2) { const uint64_t y = __shfl_xor(best, x); best = y > best ? y : best; }
    if (lane == 0) wave_key[wave] = best;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) best = wave_key[w] > best ? wave_key[w] : best;
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if ((uint32_t)(best >> 32) <= kMinusInf || !(temperature > 0.0f)) {
        if (tid == 0) a.token[r] = (uint32_t)(best >> 32) <= kMinusInf ? -1 : (int32_t)~(uint32_t)best;
        return;
    }
    const Scale scale = {value_of((uint32_t)(best >> 32)), 1.0f / temperature};
    const int k = a.top_k && a.top_k[r] > 0 && a.top_k[r] < V ? a.top_k[r] : V;
    const float p = a.top_p ? a.top_p[r] : 1.0f;
    float min_p = a.min_p ? a.min_p[r] : 0.0f;
    min_p = min_p > 1.0f ? 1.0f : min_p;

    // first digit at which the running count (by_mass: mass) of the histogram reaches `need`; ends behind a barrier
    auto search = [&](bool by_mass, uint64_t need) {
        __syncthreads();
        const uint32_t c0 = count[2 * tid], c1 = count[2 * tid + 1];
        const uint64_t m0 = mass[2 * tid], m1 = mass[2 * tid + 1];
        uint32_t c = c0 + c1;
        uint64_t m = m0 + m1;
        for (int x = 1; x < 64; x *= 2) {
            const uint32_t cc = __shfl_up(c, x);
            const uint64_t mm = __shfl_up(m, x);
            if (lane >= x) { c += cc; m += mm; }
        }
        if (lane == 63) { wave_count[wave] = c; wave_mass[wave] = m; }
        __syncthreads();
        for (int w = 0; w < wave; ++w) { c += wave_count[w]; m += wave_mass[w]; }
        c -= c0 + c1;
        m -= m0 + m1;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t cx = x ? c1 : c0;
            const uint64_t mx = x ? m1 : m0, before = by_mass ? m : c, here = by_mass ? mx : cx;
            if (before < need && before + here >= need) found = {(uint32_t)(2 * tid + x), c, cx, m, mx};
            c += cx;
            m += mx;
        }
        __syncthreads();
        return found;
    };
    auto clear = [&] {
        __syncthreads();
        for (int x = tid; x < kBins; x += kThreads) { count[x] = 0; mass[x] = 0; }
        __syncthreads();
    };
    auto put = [&](uint32_t digit, float x) {
        atomicAdd(&count[digit], 1u);
        atomicAdd((unsigned long long*)&mass[digit], (unsigned long long)scale.mass(scale.weight(x)));
    };
    // the end of a prefix: all of the bins before `bin`, and of it all (whole) or the keys above `key` and `ties` entries of it
    struct End { uint32_t bin, key, ties, equal; bool whole; uint64_t mass; };
    End end = {kBins - 1, 0, 0, 0, true, 0};
    auto descend = [&](bool by_mass, const Found& in, uint64_t need) {
        End e = {in.digit, 0, 0, 0, false, in.mass_before};
        uint32_t above = 0;
        const int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
        for (int level = 0; level < 3; ++level) {
            const int shift = shifts[level], width = widths[level];
            const uint32_t ones = (1u << width) - 1;
            clear();
            for (int i = tid; i < V; i += kThreads) {
                const float x = at(i);
                const uint32_t key = key_of(x);
                if (scale.bin(x) == in.digit && (level == 0 || key >> (shift + width) == above)) put(ones - (key >> shift & ones), x);
            }
            const Found f = search(by_mass, need);
            above = above << width | (ones - f.digit);
            need -= by_mass ? f.mass_before : f.count_before;
            e.mass += f.mass_before;
            e.equal = f.count;
        }
        e.key = above;
        const uint64_t each = scale.mass(scale.weight(value_of(above)));
        e.ties = (uint32_t)(by_mass ? (need + each - 1) / each : need);
        e.mass += e.ties * each;
        return e;
    };

    if (k < V || p < 1.0f) {
        clear();
        for (int i = tid; i < V; i += kThreads) { const float x = at(i); put(scale.bin(x), x); }
        const Found in_k = search(false, (uint64_t)k);
        Found in_p = in_k;
        uint64_t total = in_k.mass_before + in_k.mass, need = 0;
        end.bin = in_k.digit;
        bool cut_k = (uint64_t)k - in_k.count_before < in_k.count;
        if (p < 1.0f && !cut_k) {
            const double want = ceil((double)p * (double)total);
            need = want >= 1.0 ? (uint64_t)want : 1;
            in_p = search(true, need);
        }
        if (cut_k) {
            end = descend(false, in_k, (uint64_t)k - in_k.count_before);
            total = end.mass;
            if (p < 1.0f) {
                const double want = ceil((double)p * (double)total);
                need = want >= 1.0 ? (uint64_t)want : 1;
                clear();
                for (int i = tid; i < V; i += kThreads) { const float x = at(i); put(scale.bin(x), x); }
                in_p = search(true, need);
            }
        }
        if (p < 1.0f) {
            end = {in_p.digit, 0, 0, 0, true, 0};
            if (need - in_p.mass_before < in_p.mass || cut_k) end = descend(true, in_p, need - in_p.mass_before);
        }
    }
    // equal logits of which not all are kept: the index of the first one that is not
    uint32_t ties_end = (uint32_t)V;
    const int segments = (V + 63) / 64;
    auto lowest = [&](uint64_t need, auto amount) -> uint32_t {          // the index at which the running amount reaches `need`
        __syncthreads();
        for (int s = wave; s < segments; s += kWaves) {
            const int i = s * 64 + lane;
            uint64_t m = i < V ? amount(i) : 0;
            for (int x = 1; x < 64; x *= 2) m += __shfl_xor(m, x);
            if (lane == 0) mass[s] = m;
        }
        __syncthreads();
        if (wave == 0) {
            uint64_t before = 0;
            for (int s0 = 0; s0 < segments; s0 += 64) {
                uint64_t m = s0 + lane < segments ? mass[s0 + lane] : 0;
                for (int x = 1; x < 64; x *= 2) { const uint64_t y = __shfl_up(m, x); if (lane >= x) m += y; }
                const uint64_t hit = __ballot(before + m >= need);
                if (hit) {
                    const int f = __ffsll((unsigned long long)hit) - 1;
                    if (f) before += __shfl(m, f - 1);
                    const int i = (s0 + f) * 64 + lane;
                    uint64_t y = i < V ? amount(i) : 0;
                    for (int x = 1; x < 64; x *= 2) { const uint64_t z = __shfl_up(y, x); if (lane >= x) y += z; }
                    const uint64_t here = __ballot(before + y >= need);
                    if (lane == 0) shared_index = (uint32_t)((s0 + f) * 64 + __ffsll((unsigned long long)here) - 1);
                    break;
                }
                before += __shfl(m, 63);
            }
        }
        __syncthreads();
        return shared_index;
    };
    if (!end.whole && end.ties < end.equal)
        ties_end = lowest(end.ties, [&](int i) { return (uint64_t)(key_of(at(i)) == end.key); }) + 1;
    auto kept = [&](int i) -> uint64_t {
        const float x = at(i);
        const uint32_t b = scale.bin(x), key = key_of(x);
        if (b > end.bin || (!end.whole && b == end.bin && (key < end.key || (key == end.key && (uint32_t)i >= ties_end)))) return 0;
        const float w = scale.weight(x);
        return w < min_p ? 0 : scale.mass(w);
    };
    uint64_t total = 0;
    for (int i = tid; i < V; i += kThreads) total += kept(i);
    for (int x = 1; x < 64; x *= 2) total += __shfl_xor(total, x);
    __syncthreads();
    if (lane == 0) wave_mass[wave] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kWaves; ++w) total += wave_mass[w];
    const float u = a.uniform[r];
    uint64_t passed = 0;
    if (u > 0.0f) {
        const double want = floor((double)u * (double)total);
        passed = want < (double)total ? (uint64_t)want : total - 1;
        if (passed >= total) passed = total - 1;
    }
    const uint32_t token = lowest(passed + 1, kept);
    if (tid == 0) a.token[r] = (int32_t)token;
}

bool sizes_ok(const fr_sample_desc& d)
{
    return d.dtype >= FR_DTYPE_BF16 && d.dtype <= FR_DTYPE_F32 && d.n_rows >= 0 && d.n_vocab >= 1 && d.n_vocab <= kMostVocab;
}

}  // namespace

extern "C" {

int fr_sample_workspace_bytes(const fr_sample_desc* d, uint64_t* bytes_out)
{
    if (!d || !bytes_out || !sizes_ok(*d)) return FR_ERR_ARG;
    *bytes_out = 0;
    return FR_OK;
}

int fr_sample(const fr_sample_desc* d, void* stream)
{
    if (!d || !sizes_ok(*d)) return FR_ERR_ARG;
    if (d->n_rows == 0) return FR_OK;
    const uintptr_t size = d->dtype == FR_DTYPE_F32 ? 4 : 2;
    if (!d->logits || !d->uniform || !d->token || (uintptr_t)d->logits % size) return FR_ERR_ARG;
    if (d->row_stride < 0 || d->row_stride > ((int64_t)1 << 45) || (d->n_rows > 1 && d->row_stride < d->n_vocab)) return FR_ERR_ARG;
    const SampleArgs a = {d->logits, d->row_stride, d->n_vocab, d->temperature, d->top_p, d->min_p, d->uniform, d->top_k, d->token};
    const dim3 grid((unsigned)d->n_rows);
    if (d->dtype == FR_DTYPE_BF16) hipLaunchKernelGGL(k_sample<Bf16>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    else if (d->dtype == FR_DTYPE_F16) hipLaunchKernelGGL(k_sample<F16>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(k_sample<F32>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}

}  // extern "C"
