// One token for every row of logits, from a given random number: temperature, top-k, top-p and min-p.
//
// The entries kept are a prefix of the row in falling order, so nothing is sorted: the prefix' end is searched for by histograms of
// the entries' counts and masses.  Masses are 64-bit integers, whose sums do not depend on the order of the additions.  A
// histogram's digit is a step of 1/64 on the scale of (m - l) / temperature, over which a language model's logits spread evenly
// (digits of a float's bits would put thousands of entries on one counter).
//
// A workgroup takes a row, and reads it twice:
//   first for the largest logit, of the row and of every thread's share;
//   then, for rows that are cut by count or mass, to put the entries that can be kept into LDS.  The rank-th largest of the threads'
//   own largest logits has at least `rank` entries above it, and seldom many more: with rank = top_k all of the first top_k are
//   among them; for a cut by mass rank is 640, and the pass adds up the mass of the whole row, which says whether what is in LDS
//   holds enough of it.  What is left happens in LDS.
//   Rows that are not cut, or by weight alone, need the masses of runs of 64 lanes' entries instead, and one run again.
// Rows that none of this fits (many thousands of entries that can be kept, or as many equal ones, infinities) go through the row
// for every digit of the search.

#include <cmath>

#include "common.h"
#include "lm_types.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2 * kThreads, kMostVocab = 1 << 19;
constexpr float kMassOne = 8796093022208.0f;           // 2^43: the sum over 2^19 entries stays below 2^63

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

constexpr int kCandidates = 4096, kList = 1024, kRank = 640;
constexpr uint32_t kNoMass = 1909;                     // from this digit on (29.83 and more below the top) masses are 0: 43 ln 2 = 29.81

// A row of any alignment in pieces of 16 bytes: `head` entries up to the first such piece, `pieces` of kEach, `tail` entries.
template <typename T> struct Row {
    static constexpr int kEach = 16 / (int)sizeof(typename T::Bits);
    const typename T::Bits* p;
    int head, pieces, tail, n;
    __device__ __forceinline__ Row(const typename T::Bits* row, int V) : p(row), n(V)
    {
        head = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(typename T::Bits));
        pieces = (V - head) / kEach;
        tail = V - head - pieces * kEach;
    }
    __device__ __forceinline__ float at(int i) const { return T::up(p[i]); }
    struct Piece { float x[kEach]; };
    __device__ __forceinline__ Piece piece(int v) const
    {
        const uint4 b = *reinterpret_cast<const uint4*>(p + head + v * kEach);
        const uint32_t w[4] = {b.x, b.y, b.z, b.w};
        Piece y;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if constexpr (kEach == 4) y.x[e] = __uint_as_float(w[e]);
            else y.x[e] = T::up((typename T::Bits)(w[e / 2] >> (16 * (e % 2))));
        }
        return y;
    }
    // every entry once: f(index, value)
    template <typename F> __device__ __forceinline__ void each(int tid, F f) const
    {
        int v = tid;
        for (; v + 3 * kThreads < pieces; v += 4 * kThreads) {
            Piece y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = piece(v + q * kThreads);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < kEach; ++e) f(head + (v + q * kThreads) * kEach + e, y[q].x[e]);
        }
        for (; v < pieces; v += kThreads) {
            const Piece y = piece(v);
#pragma unroll
            for (int e = 0; e < kEach; ++e) f(head + v * kEach + e, y.x[e]);
        }
        if (tid < head) f(tid, at(tid));
        if (tid < tail) f(n - tail + tid, at(n - tail + tid));
    }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    // (the slow path's masses of 64 entries each take the room of histogram, candidates and list)
    __shared__ __align__(16) uint64_t room[kMostVocab / 64];
    __shared__ uint32_t count[kBins];
    __shared__ uint64_t wave_mass[kWaves];
    __shared__ uint32_t wave_count[kWaves];
    __shared__ float wave_top[kWaves];
    __shared__ Found found;
    __shared__ uint64_t shared_key, shared_mass;
    __shared__ uint32_t shared_index, filled;
    uint64_t* mass = room;                                                         // [kBins]
    float* cand_value = reinterpret_cast<float*>(room + kBins);                    // [kCandidates]
    uint32_t* cand_index = reinterpret_cast<uint32_t*>(cand_value + kCandidates);  // [kCandidates]
    uint64_t* list_key = reinterpret_cast<uint64_t*>(cand_index + kCandidates);    // [kList]
    uint64_t* list_mass = list_key + kList;
    static_assert(8 * kBins + 8 * kCandidates + 16 * kList <= (int)sizeof(room), "");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.n_vocab;
    const int64_t r = blockIdx.x;
    const Row<T> row(static_cast<const typename T::Bits*>(a.logits) + r * a.row_stride, V);
    auto at = [&](int i) { return cleaned(row.at(i)); };

    float top = -INFINITY;
    row.each(tid, [&](int, float x) { top = fmaxf(top, x); });                     // (fmaxf passes NaN over)
    const float my_top = top;
    for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
    if (lane == 0) wave_top[wave] = top;
    if (tid == 0) shared_index = 0xffffffffu;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, wave_top[w]);
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (top == -INFINITY) {
        if (tid == 0) a.token[r] = -1;
        return;
    }
    if (!(temperature > 0.0f)) {
        uint32_t lowest = 0xffffffffu;
        if (my_top == top) row.each(tid, [&](int i, float x) { if (x == top) lowest = min(lowest, (uint32_t)i); });
        if (my_top == top) atomicMin(&shared_index, lowest);
        __syncthreads();
        if (tid == 0) a.token[r] = (int32_t)shared_index;
        return;
    }
    const Scale scale = {top, 1.0f / temperature};
    const int k = a.top_k && a.top_k[r] > 0 && a.top_k[r] < V ? a.top_k[r] : V;
    const float p = a.top_p ? a.top_p[r] : 1.0f;
    float min_p = a.min_p ? a.min_p[r] : 0.0f;
    min_p = min_p > 1.0f ? 1.0f : min_p;
    const float u = a.uniform[r];
    auto mass_passed = [&](uint64_t total) -> uint64_t {                            // floor(u total), below total
        if (!(u > 0.0f)) return 0;
        const double want = floor((double)u * (double)total);
        const uint64_t x = want < (double)total ? (uint64_t)want : total;
        return x < total ? x : total - 1;
    };
    auto mass_needed = [&](uint64_t total) -> uint64_t {                            // ceil(p total), 1 at least
        const double want = ceil((double)p * (double)total);
        return want >= 1.0 ? (uint64_t)want : 1;
    };
    // the sum over the workgroup; ends behind a barrier
    auto add_up = [&](uint64_t x) {
        for (int y = 1; y < 64; y *= 2) x += __shfl_xor(x, y);
        __syncthreads();
        if (lane == 0) wave_mass[wave] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += wave_mass[w];
        return x;
    };
    const bool plain = top < INFINITY && scale.per_t > 0.0f && scale.per_t < INFINITY;
    // mass of an entry as a float that is a whole number (the floor is exact: from 2^24 on all are whole); 0 for NaN
    auto whole_mass = [&](float x) { return fmaxf(floorf(expf((x - top) * scale.per_t) * kMassOne), 0.0f); };

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
    if (plain && k == V && !(p < 1.0f)) {
        // not cut: masses of runs of 64 pieces; head and tail are runs of their own
        constexpr int kEach = Row<T>::kEach;
        const int runs = (row.pieces + 63) / 64, all = runs + 2;
        auto amount = [&](float x) -> double {
            const float w = expf((x - top) * scale.per_t);
            return w < min_p ? 0.0f : fmaxf(floorf(w * kMassOne), 0.0f);
        };
        auto lane_sum = [&](int s, double (&m)[kEach]) {                            // entries of run s: what a lane has of it
            double sum = 0.0;
            const int v = (s - 1) * 64 + lane;
#pragma unroll
            for (int e = 0; e < kEach; ++e) m[e] = 0.0;
            if (s == 0 || s == all - 1) {
                const int n = s ? row.tail : row.head, i = s ? V - row.tail + lane : lane;
                if (lane < n) m[0] = amount(row.at(i));
            } else if (v < row.pieces) {
                const typename Row<T>::Piece y = row.piece(v);
#pragma unroll
                for (int e = 0; e < kEach; ++e) m[e] = amount(y.x[e]);
            }
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum += m[e];
            return sum;
        };
        double m[kEach];
        uint64_t sum = 0;
        for (int s = wave; s < all; s += kWaves) {
            double x = lane_sum(s, m);                                              // (whole numbers below 2^53: exact)
            for (int y = 1; y < 64; y *= 2) x += __shfl_xor(x, y);
            if (lane == 0) room[s] = (uint64_t)x;
            sum += lane == 0 ? (uint64_t)x : 0;
        }
        const uint64_t need = mass_passed(add_up(sum)) + 1;
        if (wave == 0) {
            uint64_t before = 0;
            for (int s0 = 0; s0 < all; s0 += 64) {
                uint64_t x = s0 + lane < all ? room[s0 + lane] : 0;
                for (int y = 1; y < 64; y *= 2) { const uint64_t z = __shfl_up(x, y); if (lane >= y) x += z; }
                const uint64_t hit = __ballot(before + x >= need);
                if (hit) {
                    const int f = __ffsll((unsigned long long)hit) - 1, s = s0 + f;
                    if (f) before += __shfl(x, f - 1);
                    uint64_t mine = (uint64_t)lane_sum(s, m), z = mine;
                    for (int y = 1; y < 64; y *= 2) { const uint64_t q = __shfl_up(z, y); if (lane >= y) z += q; }
                    const uint64_t here = __ballot(before + z >= need);
                    if (lane == __ffsll((unsigned long long)here) - 1) {
                        before += z - mine;
                        int e = 0;
                        if (s != 0 && s != all - 1)
                            for (; e < kEach - 1; ++e) {
                                before += (uint64_t)m[e];
                                if (before >= need) break;
                            }
                        a.token[r] = s == 0 ? lane : s == all - 1 ? V - row.tail + lane : row.head + ((s - 1) * 64 + lane) * kEach + e;
                    }
                    break;
                }
                before += __shfl(x, 63);
            }
        }
        return;
    }
    // The element of `digit` at which the running count or mass of the list's keys, the largest first, reaches `need`: its key, and
    // the mass up to it; false if the digit has more entries than the list has room for.
    auto resolve = [&](int n, uint32_t digit, bool by_mass, uint64_t need, auto digit_of, auto key_at, auto mass_at) {
        __syncthreads();
        if (tid == 0) filled = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
            if (digit_of(i) == digit) {
                const uint64_t m = mass_at(i);
                const uint32_t to = atomicAdd(&filled, 1u);
                if (to < kList) { list_key[to] = key_at(i); list_mass[to] = m; }
            }
        __syncthreads();
        const int here = (int)filled;
        if (here > kList) return false;
        if (tid < here) {
            const uint64_t key = list_key[tid], mine = list_mass[tid];
            uint64_t before = 0, above = 0;
            for (int j = 0; j < here; ++j)
                if (list_key[j] > key) { before += list_mass[j]; ++above; }
            const uint64_t x = by_mass ? before : above, y = by_mass ? mine : 1;
            if (x < need && x + y >= need) { shared_key = key; shared_mass = before + mine; }
        }
        __syncthreads();
        return true;
    };
    bool fast = plain && (k == V || k <= kThreads || V <= kCandidates);
    if (fast) {
        // digits up to `last` can be kept
        uint32_t last = kNoMass - 1;
        if (V > kCandidates) {
            for (int x = tid; x < kBins; x += kThreads) { count[x] = 0; mass[x] = 0; }
            __syncthreads();
            if (my_top > -INFINITY) atomicAdd(&count[scale.bin(my_top)], 1u);
            if (tid == 0) found = {kBins, 0, 0, 0, 0};
            last = min(last, search(false, (uint64_t)(k < V ? k : kRank)).digit);
        }
        if (tid == 0) filled = 0;
        __syncthreads();
        const float edge = (float)(last + 1);
        uint64_t total = 0;
        auto take = [&](int i, float x) {
            if ((top - x) * scale.per_t * 64.0f < edge) {                            // (false for NaN)
                const uint32_t to = atomicAdd(&filled, 1u);
                if (to < kCandidates) { cand_value[to] = x + 0.0f; cand_index[to] = (uint32_t)i; }
            }
        };
        if (k < V) {
            row.each(tid, take);
        } else {
            double sum = 0.0;                          // (whole numbers, at most 512 of 2^43: exact)
            row.each(tid, [&](int i, float x) { sum += (double)whole_mass(x); take(i, x); });
            total = add_up((uint64_t)sum);
        }
        __syncthreads();
        const int n = (int)filled;
        fast = n <= kCandidates;
        if (fast) {
            auto digit_of = [&](int i) { return scale.bin(cand_value[i]); };
            auto key_at = [&](int i) { return (uint64_t)key_of(cand_value[i]) << 32 | (uint32_t)~cand_index[i]; };
            auto mass_at = [&](int i) { return (uint64_t)whole_mass(cand_value[i]); };
            clear();
            for (int i = tid; i < n; i += kThreads) put(digit_of(i), cand_value[i]);
            // kept: digits before `digit`, and of it the keys from `key` on
            uint32_t digit = kBins;
            uint64_t key = 0;
            if (k < n) {
                const Found f = search(false, (uint64_t)k);
                const uint64_t need = (uint64_t)k - f.count_before;
                digit = f.digit;
                total = f.mass_before + f.mass;
                if (need < f.count) {
                    fast = resolve(n, digit, false, need, digit_of, key_at, mass_at);
                    if (fast) { key = shared_key; total = f.mass_before + shared_mass; }
                }
            } else if (k < V) {                        // (fewer entries with a mass than top_k)
                uint64_t sum = 0;
                for (int i = tid; i < n; i += kThreads) sum += mass_at(i);
                total = add_up(sum);
            }
            if (fast && p < 1.0f) {
                const uint64_t need = mass_needed(total);
                __syncthreads();
                if (tid == 0) found = {kBins, 0, 0, 0, 0};
                const Found f = search(true, need);
                fast = f.digit < kBins;                // (else the candidates hold too little)
                if (fast) {
                    digit = f.digit;
                    key = 0;
                    fast = resolve(n, digit, true, need - f.mass_before, digit_of, key_at, mass_at);
                    if (fast) key = shared_key;
                }
            }
            if (fast) {
                auto kept = [&](int i) -> uint64_t {
                    const uint32_t d = digit_of(i);
                    if (d > digit || (d == digit && key_at(i) < key)) return 0;
                    if (expf((cand_value[i] - top) * scale.per_t) < min_p) return 0;
                    return mass_at(i);
                };
                // the same search along the index: 2048 runs of the vocabulary
                int shift = 0;
                while (((V - 1) >> shift) >= kBins) ++shift;
                clear();
                uint64_t sum = 0;
                for (int i = tid; i < n; i += kThreads) {
                    const uint64_t m = kept(i);
                    if (m) atomicAdd((unsigned long long*)&mass[cand_index[i] >> shift], (unsigned long long)m);
                    sum += m;
                }
                const uint64_t need = mass_passed(add_up(sum)) + 1;
                const Found f = search(true, need);
                fast = resolve(n, f.digit, true, need - f.mass_before, [&](int i) { return cand_index[i] >> shift; },
                               [&](int i) { return (uint64_t)(uint32_t)~cand_index[i]; }, kept);
                if (fast) {
                    if (tid == 0) a.token[r] = (int32_t)~(uint32_t)shared_key;
                    return;
                }
            }
        }
    }
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
            need = mass_needed(total);
            in_p = search(true, need);
        }
        if (cut_k) {
            end = descend(false, in_k, (uint64_t)k - in_k.count_before);
            total = end.mass;
            if (p < 1.0f) {
                need = mass_needed(total);
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
    const uint64_t passed = mass_passed(total);
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
