// One token for every row of logits, from a given random number: temperature, top-k, top-p and min-p.
//
// An entry of logit l has the weight w = exp((l - m) / temperature), m being the row's largest.  Kept are the first top_k in falling
// order, of those the fewest that hold top_p of their weight, of those the ones with w >= min_p; the token is the first in the
// vocabulary's order at which the running weight of the kept passes uniform times all of it.  Masses, the weights in 64-bit integers
// of 2^-43 (every weight is rounded down once, to the 24 bits that it has in 32 anyway), add up to the same sum in any order.
//
// The entries kept are a prefix of the row in falling order, so nothing is sorted: the prefix' end is searched for by histograms of
// the entries' counts and masses.  A histogram's digit is a step of 1/64 on the scale of (m - l) / temperature, over which a language
// model's logits spread evenly (digits of a float's bits would put thousands of entries on one counter).
//
// A workgroup of 1024 threads takes a row (112 KB of LDS: one on a unit), and goes through it twice:
//   first for the largest logit, of the row and of every thread's share, the largest outside of the share's piece of 16 bytes that holds
//   it, and for rows that are cut by mass alone the share's mass, roughly;
//   then, for rows that are cut by count or mass, to put the entries that can be kept into LDS: for most shares that have any from the
//   one piece alone.  The rank-th largest of the threads' two values has at least `rank` entries above it, and seldom many more: with
//   rank = top_k all of the first top_k are among them; how far down a cut by mass goes is estimated from the same values, and the
//   rough mass of the others says whether what is in LDS holds enough.  What is left happens in LDS.
//   Rows that are not cut, or by weight alone, need the masses of runs of 512 pieces instead, and one run again.
// Rows that none of this fits (many thousands of entries that can be kept, or as many equal ones, infinities) take the long way: a
// histogram of the whole row, and the masses of runs together with the digit in which the kept entries end.
//
// What bounds it, at 256 rows of 131072 in 32 bits, 134 MB: greedy 23 us, 5.8 TB/s, memory; top-k 50 31 and top-p 0.9 36 the steps in
// LDS, each behind barriers that nothing fills; no cut 51, of which 28 the vector units at 131072 exps a unit, as in the long way: 128
// at temperature 1.3 and top-p 0.98, 108 for a flat row.  One row of 32768: 13 us, the steps one after another.

#include <algorithm>
#include <cmath>
#include <type_traits>

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
// The order of entries, the largest first: of its logit (bits in an order that rises with it; 32), then of the index, the lowest first (19).
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index)
{
    const uint32_t u = __float_as_uint(x);
    return (uint64_t)(u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u)) << 19 | (kMostVocab - 1 - index);
}

struct Scale {
    float top, per_t;
    // the largest logit, the factor and hence every (x - top) per_t of a number x are numbers
    __device__ __forceinline__ bool usual() const { return top < INFINITY && per_t > 0.0f && per_t < INFINITY; }
    __device__ __forceinline__ float weight(float x) const
    {
        if (x == top) return 1.0f;
        if (x == -INFINITY) return 0.0f;
        return expf((x - top) * per_t);
    }
    // the same of a row as usual, whose exponents are numbers or -infinity (NaN for NaN)
    __device__ __forceinline__ float usual_weight(float x) const { return expf((x - top) * per_t); }
    // the mass as a float that is a whole number (from 2^24 on all floats are); 0 for NaN
    static __device__ __forceinline__ float whole(float weight) { return fmaxf(floorf(weight * kMassOne), 0.0f); }
    __device__ __forceinline__ float whole_mass(float x) const { return whole(weight(x)); }
    __device__ __forceinline__ uint64_t mass(float x) const { return (uint64_t)whole_mass(x); }
    __device__ __forceinline__ uint64_t usual_mass(float x) const { return (uint64_t)whole(usual_weight(x)); }
    __device__ __forceinline__ uint32_t bin(float x) const
    {
        if (x == top) return 0;
        return (uint32_t)fminf((top - x) * per_t * 64.0f, (float)(kBins - 1));      // (a NaN from 0 * infinity gives the last bin)
    }
};

struct Found { uint32_t digit, count_before, count; uint64_t mass_before, mass; };

// kRank: what is tried at most.  1740 of the threads' 2048 values are above a line that about 2840 entries are above, so that 4096 have
// room; top-k of 400, 1000, 1740: 39, 57, 65 us this way and 95 to 101 the long way.
constexpr int kCandidates = 4096, kList = 1024, kRank = 1740, kMostRuns = kBins;
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
    __device__ __forceinline__ int lone(int j) const { return j < head ? j : n - tail - head + j; }      // entries outside of the pieces: head + tail
    struct Piece { float x[kEach]; };
    __device__ __forceinline__ uint4 bits(int v) const { return *reinterpret_cast<const uint4*>(p + head + v * kEach); }
    static __device__ __forceinline__ Piece unpacked(const uint4& b)
    {
        const uint32_t w[4] = {b.x, b.y, b.z, b.w};
        Piece y;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if constexpr (kEach == 4) y.x[e] = __uint_as_float(w[e]);
            else y.x[e] = T::up((typename T::Bits)(w[e / 2] >> (16 * (e % 2))));
        }
        return y;
    }
    __device__ __forceinline__ Piece piece(int v) const { return unpacked(bits(v)); }
    // every piece once, by(number, piece), and the entries before and behind them, one(index, value)
    template <int kAtOnce, typename P, typename F> __device__ __forceinline__ void visit(int tid, P by, F one) const
    {
        for (int v = tid; v < pieces; v += kAtOnce * kThreads) {
            uint4 b[kAtOnce];
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) b[q] = bits(min(v + q * kThreads, pieces - 1));
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q)
                if (v + q * kThreads < pieces) by(v + q * kThreads, unpacked(b[q]));
        }
        if (tid < head + tail) one(lone(tid), at(lone(tid)));
    }
    // every entry once: f(index, value)
    template <int kAtOnce = 1, typename F> __device__ __forceinline__ void each(int tid, F f) const
    {
        visit<kAtOnce>(tid, [&](int v, const Piece& y) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) f(head + v * kEach + e, y.x[e]);
        }, f);
    }
    static __device__ __forceinline__ float top_of(const Piece& y)       // (NaN passed over)
    {
        float m = y.x[0];
#pragma unroll
        for (int e = 1; e < kEach; ++e) m = fmaxf(m, y.x[e]);
        return m;
    }
};

// What lane 63 gets is the result over all of the wavefront, what lane i gets the one over the lanes up to it: rows of 16 lanes
// first, then a row's last value goes to the rows behind it.  All 64 lanes have to be there.
template <int kControl, int kRows, typename X> __device__ __forceinline__ X moved(X x, X none)
{
    static_assert(sizeof(X) == 4 || sizeof(X) == 8);
    if constexpr (sizeof(X) == 4) {
        return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), kControl, kRows, 0xf, false));
    } else {
        const uint64_t n = __builtin_bit_cast(uint64_t, none), b = __builtin_bit_cast(uint64_t, x);
        const uint32_t low = __builtin_amdgcn_update_dpp((int)n, (int)b, kControl, kRows, 0xf, false);
        const uint32_t high = __builtin_amdgcn_update_dpp((int)(n >> 32), (int)(b >> 32), kControl, kRows, 0xf, false);
        return __builtin_bit_cast(X, (uint64_t)high << 32 | low);
    }
}
template <typename X, typename F> __device__ __forceinline__ X up_to(X x, X none, F f)
{
    x = f(x, moved<0x111, 0xf>(x, none));              // row_shr by 1, 2, 4, 8
    x = f(x, moved<0x112, 0xf>(x, none));
    x = f(x, moved<0x114, 0xf>(x, none));
    x = f(x, moved<0x118, 0xf>(x, none));
    x = f(x, moved<0x142, 0xa>(x, none));              // row_bcast 15, then 31
    return f(x, moved<0x143, 0xc>(x, none));
}
template <typename X> __device__ __forceinline__ X sum_up_to(X x) { return up_to(x, X(0), [](X a, X b) { return a + b; }); }
// (a value of lane `from`, the same for all of the wavefront)
__device__ __forceinline__ uint64_t of_lane(uint64_t x, int from)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), from) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, from);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    constexpr int kEach = Row<T>::kEach;
    __shared__ uint32_t count[kBins], top_count[kBins];        // histograms: of the entries, of the threads' largest logits
    __shared__ uint64_t mass[kBins];
    __shared__ uint64_t run_mass[kMostRuns];                   // masses of runs of the vocabulary
    __shared__ uint64_t many[kCandidates];                     // the entries that can be kept, or the keys of a digit's
    float* const cand_value = reinterpret_cast<float*>(many);
    uint32_t* const cand_index = reinterpret_cast<uint32_t*>(many) + kCandidates;
    __shared__ uint64_t list_key[kList], list_mass[kList];
    __shared__ uint32_t hot[kCandidates];                      // pieces that hold entries which can be kept
    __shared__ uint64_t wave_mass[kWaves], wave_low[kWaves];
    __shared__ uint32_t wave_count[kWaves];
    __shared__ float wave_top[kWaves];
    __shared__ double wave_others[kWaves];
    __shared__ Found found;
    __shared__ uint64_t shared_key, shared_mass;
    __shared__ uint32_t shared_index, filled[10];
    const int V = a.n_vocab;
    int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // (from here on what hangs on them is worked out anew, not kept in registers from one part of the kernel to the next)
    auto afresh = [&] { asm volatile("" : "+v"(tid)); lane = tid & 63; wave = tid >> 6; };
    const int64_t r = blockIdx.x;
    const Row<T> row(static_cast<const typename T::Bits*>(a.logits) + r * a.row_stride, V);

    const float temperature = a.temperature ? a.temperature[r] : 1.0f, per_t = 1.0f / temperature, to_exp2 = per_t * 1.44269504f;
    const int k = a.top_k && a.top_k[r] > 0 && a.top_k[r] < V ? a.top_k[r] : V;
    const float p = a.top_p ? a.top_p[r] : 1.0f, u = a.uniform[r];
    float min_p = a.min_p ? a.min_p[r] : 0.0f;
    min_p = min_p > 1.0f ? 1.0f : min_p;
    // First pass: the largest logit of the thread's share, the piece that it is in and the largest of the other pieces (an entry before
    // or behind the pieces counts as one); for rows cut by mass alone also the share's mass, roughly, apart for that piece, relative to
    // `from` (which lags behind the largest by up to a factor of 2^8).  The error of a weight in it is below 2^-16 of the weight: of
    // the exponent's products, differences and constant |x| 5 / 2^24 with |x| <= 43 (where a weight still has a mass), of each exp 2^-23,
    // of sums of eight in 32 bits 2^-22, of up to six factors where `from` moves 2^-22 each.
    const bool by_mass = k == V && p < 1.0f && per_t > 0.0f && per_t < INFINITY;
    float top = -INFINITY, second = -INFINITY, from = -INFINITY, top_mass = 0.0f;
    int top_piece = -1;
    double others = 0.0;
    auto roughly = [&](float x) { return __builtin_amdgcn_exp2f(fmaxf((x - from) * to_exp2, -126.0f)); };         // (NaN: next to nothing)
    auto note = [&](int v, float t) {
        const bool more = t > top;                     // (NaN: passed over)
        second = fmaxf(second, more ? top : t);
        if (more) { top = t; top_piece = v; }
        return more;
    };
    if (by_mass) {
        const float slack = 8.0f / to_exp2;
        auto add = [&](int v, float t, auto sum_of) {
            if (t > from + slack) {
                const float f = __builtin_amdgcn_exp2f((from - t) * to_exp2);
                others *= (double)f;
                top_mass *= f;
                from = t;
            }
            const float sum = sum_of();
            const bool more = note(v, t);
            others += (double)(more ? top_mass : sum);
            if (more) top_mass = sum;
        };
        row.template visit<4>(tid, [&](int v, const typename Row<T>::Piece& y) {
            add(v, Row<T>::top_of(y), [&] {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < kEach; ++e) sum += roughly(y.x[e]);
                return sum;
            });
        }, [&](int, float x) { add(row.pieces + tid, x, [&] { return roughly(x); }); });
    } else {
        row.template visit<4>(tid, [&](int v, const typename Row<T>::Piece& y) { note(v, Row<T>::top_of(y)); }, [&](int, float x) { note(row.pieces + tid, x); });
    }
    // room for n of every lane's: one addition a wavefront, all lanes there
    auto room_for = [&](uint32_t& counter, uint32_t n) {
        const uint32_t up_to_here = sum_up_to(n);
        uint32_t to = 0;
        if (lane == 63 && up_to_here) to = atomicAdd(&counter, up_to_here);
        return (uint32_t)__builtin_amdgcn_readlane((int)to, 63) + up_to_here - n;
    };
    // f(index, value) for the entries of a piece; from row.pieces on a piece is an entry before or behind the others
    auto look_into = [&](int v, auto f) {
        if (v < row.pieces) {
            const typename Row<T>::Piece y = row.piece(v);
#pragma unroll
            for (int e = 0; e < kEach; ++e) f(row.head + v * kEach + e, y.x[e]);
        } else {
            const int i = row.lone(v - row.pieces);
            f(i, row.at(i));
        }
    };
    for (int x = tid; x < kBins; x += kThreads) { count[x] = 0; mass[x] = 0; top_count[x] = 0; run_mass[x] = 0; }
    if (tid < 10) filled[tid] = 0;
    const float my_top = top;
    top = up_to(top, -INFINITY, [](float x, float y) { return fmaxf(x, y); });
    top = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(top), 63));
    if (lane == 0) wave_top[wave] = top;
    if (by_mass) {                                     // relative to the wavefront's largest
        double sum = from > -INFINITY ? (others + (double)top_mass) * (double)__builtin_amdgcn_exp2f((from - top) * to_exp2) : 0.0;
        sum = sum_up_to(sum);
        if (lane == 63) wave_others[wave] = sum;
    }
    if (tid == 0) shared_index = 0xffffffffu;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, wave_top[w]);
    if (top == -INFINITY) {
        if (tid == 0) a.token[r] = -1;
        return;
    }
    if (!(temperature > 0.0f)) {
        if (my_top == top) {
            uint32_t lowest = 0xffffffffu;             // (a share's pieces come in rising order, but for the lone entry)
            look_into(top_piece, [&](int i, float x) { if (x == top) lowest = min(lowest, (uint32_t)i); });
            if (tid < row.head + row.tail && row.at(row.lone(tid)) == top) lowest = min(lowest, (uint32_t)row.lone(tid));
            atomicMin(&shared_index, lowest);
        }
        __syncthreads();
        if (tid == 0) a.token[r] = (int32_t)shared_index;
        return;
    }
    afresh();
    const Scale scale = {top, per_t};
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
        x = sum_up_to(x);
        __syncthreads();
        if (lane == 63) wave_mass[wave] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += wave_mass[w];
        return x;
    };
    auto add_up_row = [&] {                            // (a thread's masses: whole numbers, at most 520 of 2^43: exact in a double)
        double sum = 0.0;
        row.template each<2>(tid, [&](int, float x) { sum += (double)Scale::whole(scale.usual_weight(x)); });
        return add_up((uint64_t)sum);
    };

    // Sums of counts and masses up to every digit of a histogram (either may be left out): a thread has two digits.
    struct Sums { uint32_t c0, c1, before_c, all_c; uint64_t m0, m1, before_m, all_m; };
    auto scan_of = [&](auto counts, auto masses, uint32_t c0, uint32_t c1, uint64_t m0, uint64_t m1) {
        Sums b = {c0, c1, 0, 0, m0, m1, 0, 0};
        const uint32_t c = counts ? sum_up_to(b.c0 + b.c1) : 0;
        const uint64_t m = masses ? sum_up_to(b.m0 + b.m1) : 0;
        if (lane == 63) { wave_count[wave] = c; wave_mass[wave] = m; }
        __syncthreads();
        b.before_c = c - b.c0 - b.c1;
        b.before_m = m - b.m0 - b.m1;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t cw = counts ? wave_count[w] : 0;
            const uint64_t mw = masses ? wave_mass[w] : 0;
            if (w < wave) { b.before_c += cw; b.before_m += mw; }
            b.all_c += cw;
            b.all_m += mw;
        }
        return b;
    };
    const std::true_type yes{};
    const std::false_type no{};
    auto scan = [&](auto counts, auto masses, const uint32_t* c, const uint64_t* m) {
        __syncthreads();
        return scan_of(counts, masses, counts ? c[2 * tid] : 0, counts ? c[2 * tid + 1] : 0, masses ? m[2 * tid] : 0, masses ? m[2 * tid + 1] : 0);
    };
    // The digit at which the running count (by_mass: mass) reaches `need`, which is not more than all of it; ends behind a barrier.
    auto find = [&](const Sums& b, bool by_mass, uint64_t need) {
        __syncthreads();
        uint32_t c = b.before_c;
        uint64_t m = b.before_m;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t cx = x ? b.c1 : b.c0;
            const uint64_t mx = x ? b.m1 : b.m0, before = by_mass ? m : c, here = by_mass ? mx : cx;
            if (before < need && before + here >= need) found = {(uint32_t)(2 * tid + x), c, cx, m, mx};
            c += cx;
            m += mx;
        }
        __syncthreads();
        return found;
    };
    auto put = [&](uint32_t digit, float x) {
        atomicAdd(&count[digit], 1u);
        atomicAdd((unsigned long long*)&mass[digit], (unsigned long long)scale.mass(x));
    };
    // The list's key, the largest first, at which the running count or mass reaches `need`, to shared_key; the mass up to it to
    // shared_mass.  Entries are listed with list(which, key, mass); false if there were more than the list has room for.
    auto list = [&](int which, uint64_t key, uint64_t m) {
        const uint32_t to = atomicAdd(&filled[which], 1u);
        if (to < kList) { list_key[to] = key; list_mass[to] = m; }
    };
    auto resolve = [&](int which, bool by_mass, uint64_t need) {
        __syncthreads();
        const int here = (int)filled[which];
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

    if (scale.usual() && (k < V || p < 1.0f || min_p > 0.0f) && (k == V || k <= kRank || V <= kCandidates)) {
        // digits up to `last` can be kept
        uint32_t last = kNoMass - 1;
        bool fits = true;
        if (k == V && !by_mass) {
            last = min(last, (uint32_t)fminf(-64.0f * logf(min_p) + 1.0f, (float)last));       // (cut by weight alone)
        } else if (V > kCandidates) {
            // (the largest in the lower half of a counter, the second pieces' in the upper)
            if (my_top > -INFINITY) atomicAdd(&top_count[scale.bin(my_top)], 1u);
            if (second > -INFINITY) atomicAdd(&top_count[scale.bin(second)], 0x10000u);
            const Sums tops = scan(yes, no, top_count, nullptr);
            auto noted = [](uint32_t c) { return (c & 0xffff) + (c >> 16); };
            Sums both = tops;
            both.c0 = noted(tops.c0), both.c1 = noted(tops.c1), both.before_c = noted(tops.before_c), both.all_c = noted(tops.all_c);
            uint32_t rank = (uint32_t)k;
            if (by_mass) {
                // As many as hold the mass, going by the threads' values: where c of 1024 threads have their largest above a line, about
                // -1024 log(1 - c / 1024) entries are above it, and as many as there are values above it at least.  5 % more mass (but
                // 30 % less left out, at most) and four digits for what the estimate is off by: too few, and the row takes the long way,
                // too many cost a little.  (With the largest alone, where a thread may have two that count, top-p 0.9 took 48 us instead
                // of 36; with no room 93, with 20 % and 16 digits 67.  Top-p 0.96 and 0.98: with 5 % more always 68 us, 10 % less left out
                // 53 and 81, 30 % 52 and 50, 50 % 53 and 48, and 64 bf16 rows 23, 24, 31.)
                auto entries = [&](uint32_t c) {
                    return fmaxf(-1024.0f * 0.69314718f * __builtin_amdgcn_logf(1.0f - fminf((float)(c & 0xffff), 1023.5f) / 1024.0f), (float)noted(c));
                };
                const float n0 = entries(tops.before_c), n1 = entries(tops.before_c + tops.c0), n2 = entries(tops.before_c + tops.c0 + tops.c1);
                const float w0 = __builtin_amdgcn_exp2f(-(float)(4 * tid + 1) * (1.44269504f / 128.0f)), w1 = w0 * 0.98449644f;      // (of a digit's middle; exp(-1/64))
                static_assert(kWaves == 16);
                const float of_wave = wave_top[lane % kWaves];
                const double in_wave = of_wave > -INFINITY ? wave_others[lane % kWaves] * (double)__builtin_amdgcn_exp2f((of_wave - top) * to_exp2) : 0.0;
                const double all = __builtin_bit_cast(double, of_lane(__builtin_bit_cast(uint64_t, sum_up_to(in_wave)), 15));
                __syncthreads();
                const Sums held = scan_of(no, yes, 0, 0, (uint64_t)(fmaxf(n1 - n0, 0.0f) * w0 * 0x1p30f), (uint64_t)(fmaxf(n2 - n1, 0.0f) * w1 * 0x1p30f));
                const uint64_t want = (uint64_t)fmax(fmin((double)p * 1.05, 1.0 - 0.7 * (1.0 - (double)p)) * all * 0x1p30, 1.0);     // (top_p may be 0 and below)
                if (want <= held.all_m) {
                    last = min(last, find(held, true, want).digit + 4);
                    rank = V;
                } else {
                    // As many as there is room for, and at once the long way if those will hold too little: if what is missing can be
                    // entries below all values (else a thread has several of the largest: seldom, but one row is enough).  Flat rows
                    // 108 us; with the attempt 33 more.
                    const float each = expf(-(float)find(both, false, both.all_c).digit / 64.0f) * 0x1p30f;
                    rank = kRank;
                    fits = (double)held.all_m >= 0.8 * (double)want || (double)(want - held.all_m) > (double)V * each;
                }
            }
            if (rank <= both.all_c) last = min(last, find(both, false, rank).digit);
        }
        if (fits) {
            // Entries whose digit can be kept go to LDS.  A thread reads its share again if its largest is among them; the mass of the others
            // is known roughly, which seldom leaves open where the kept ones end.
            const float edge = (float)(last + 1), low = top - (edge / (64.0f * scale.per_t) * 1.0001f + fabsf(top) * 1e-6f);
            const float scaled = from > -INFINITY ? __builtin_amdgcn_exp2f((from - top) * to_exp2) : 0.0f;
            others *= (double)scaled;
            from = top;
            const bool is_hot = top_piece >= 0 && my_top >= low;
            // The pieces that are looked into: those with the shares' largest, and all of a share whose second is among them too, or
            // where that is too many, those that hold any, for which such shares are read again.
            const bool all_of_it = is_hot && second >= low, lone = tid < row.head + row.tail;
            const int share = (row.pieces - tid + kThreads - 1) / kThreads, n_hot = all_of_it ? max(share, 0) + (lone ? 1 : 0) : is_hot ? 1 : 0;
            const int to = (int)room_for(filled[7], (uint32_t)n_hot);
            if (to + n_hot <= kCandidates) {
                if (all_of_it) {
                    for (int j = 0; j < share; ++j) hot[to + j] = (uint32_t)(tid + j * kThreads);
                    if (lone) hot[to + n_hot - 1] = (uint32_t)(row.pieces + tid);
                } else if (is_hot) {
                    hot[to] = (uint32_t)top_piece;
                }
            }
            __syncthreads();
            const bool too_many = (int)filled[7] > kCandidates;
            if (!is_hot) others += (double)(top_mass * scaled);
            else if (too_many || all_of_it) others = 0.0;
            if (too_many) {
                __syncthreads();
                if (tid == 0) filled[7] = 0;
                __syncthreads();
                auto mark = [&](int v) {
                    const uint32_t to = atomicAdd(&filled[7], 1u);
                    if (to < kCandidates) hot[to] = (uint32_t)v;
                };
                if (is_hot) row.template visit<8>(tid, [&](int v, const typename Row<T>::Piece& y) {
                    if (Row<T>::top_of(y) >= low) {
                        mark(v);
                    } else if (by_mass) {
                        float sum = 0.0f;
#pragma unroll
                        for (int e = 0; e < kEach; ++e) sum += roughly(y.x[e]);
                        others += (double)sum;
                    }
                }, [&](int, float) { mark(row.pieces + tid); });
                __syncthreads();
            }
            const int pieces = min((int)filled[7], kCandidates);
            for (int i0 = 0; i0 < pieces; i0 += kThreads) {
                const bool here = i0 + tid < pieces;
                const int v = here ? (int)hot[i0 + tid] : 0;
                float sum = 0.0f;
                uint32_t bits = 0, bit = 1;
                if (here) look_into(v, [&](int, float x) {
                    if ((top - x) * scale.per_t * 64.0f < edge) bits |= bit;             // (false for NaN)
                    else if (by_mass) sum += roughly(x);
                    bit <<= 1;
                });
                others += (double)sum;
                uint32_t to = room_for(filled[0], (uint32_t)__popc(bits));
                bit = 1;
                if (bits) look_into(v, [&](int j, float x) {
                    if (bits & bit) {
                        if (to < kCandidates) { cand_value[to] = x + 0.0f; cand_index[to] = (uint32_t)j; }
                        ++to;
                    }
                    bit <<= 1;
                });
            }
            if (by_mass) {
                others = sum_up_to(others);
                if (lane == 63) wave_others[wave] = others;
            }
            __syncthreads();
            const int n = (int)filled[0];
            fits = n <= kCandidates && (int)filled[7] <= kCandidates;
            if (fits) {
                auto digit_of = [&](int i) { return scale.bin(cand_value[i]); };
                auto key_at = [&](int i) { return key_of(cand_value[i], cand_index[i]); };
                auto mass_at = [&](int i) { return scale.usual_mass(cand_value[i]); };
                auto among = [&](int which, uint32_t digit, bool by_mass, uint64_t need) {
                    for (int i = tid; i < n; i += kThreads)
                        if (digit_of(i) == digit) list(which, key_at(i), mass_at(i));
                    return resolve(which, by_mass, need);
                };
                for (int i = tid; i < n; i += kThreads) put(digit_of(i), cand_value[i]);
                const Sums sums = scan(yes, yes, count, mass);
                // kept: digits before `digit`, and of it the keys from `key` on
                uint32_t digit = kBins;
                uint64_t key = 0, least = sums.all_m, most = sums.all_m;                // bounds of the mass that top_p is a share of
                if (k < n) {
                    const Found f = find(sums, false, (uint64_t)k);
                    const uint64_t need = (uint64_t)k - f.count_before;
                    digit = f.digit;
                    least = most = f.mass_before + f.mass;
                    if (need < f.count) {
                        fits = among(1, digit, false, need);
                        if (fits) { key = shared_key; least = most = f.mass_before + shared_mass; }
                    }
                } else if (by_mass) {
                    double sum = 0.0;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) sum += wave_others[w];
                    sum *= (double)kMassOne;
                    const double off = sum * 0x1p-16 + (double)V;                       // (V: what the floors take off)
                    least += sum > off ? (uint64_t)(sum - off) : 0;
                    most += (uint64_t)(sum + off);
                }
                for (int pass = 0; fits && p < 1.0f; ++pass) {
                    const uint64_t need = mass_needed(least);
                    fits = need <= sums.all_m;                                          // (else the candidates hold too little)
                    if (!fits) break;
                    const Found f = find(sums, true, need);
                    fits = among(2 + pass, f.digit, true, need - f.mass_before);
                    if (!fits) break;
                    digit = f.digit;
                    key = shared_key;
                    if (mass_needed(most) <= f.mass_before + shared_mass) break;
                    least = most = add_up_row();           // (it matters: every mass of the row)
                }
                if (fits) {
                    auto kept = [&](int i) -> uint64_t {
                        const uint32_t d = digit_of(i);
                        if (d > digit || (d == digit && key_at(i) < key) || scale.usual_weight(cand_value[i]) < min_p) return 0;
                        return mass_at(i);
                    };
                    // the same search along the index: 2048 runs of the vocabulary
                    int shift = 0;
                    while (((V - 1) >> shift) >= kBins) ++shift;
                    for (int i = tid; i < n; i += kThreads) {
                        const uint64_t m = kept(i);
                        if (m) atomicAdd((unsigned long long*)&run_mass[cand_index[i] >> shift], (unsigned long long)m);
                    }
                    const Sums runs = scan(no, yes, nullptr, run_mass);
                    const uint64_t need = mass_passed(runs.all_m) + 1;
                    const Found f = find(runs, true, need);
                    for (int i = tid; i < n; i += kThreads)
                        if (cand_index[i] >> shift == f.digit) list(4, (uint64_t)~cand_index[i], kept(i));
                    resolve(4, true, need - f.mass_before);                             // (a run has at most 256 entries)
                    if (tid == 0) a.token[r] = (int32_t)~(uint32_t)shared_key;
                    return;
                }
            }
        }
    }

    afresh();
    // Through the row for every step: a histogram of all of it, the digits in which the kept entries end looked into.
    float last_kept = -INFINITY;                       // of the kept entries the last one's logit and index
    int last_index = V;
    auto clear = [&] {
        __syncthreads();
        for (int x = tid; x < kBins; x += kThreads) { count[x] = 0; mass[x] = 0; }
        __syncthreads();
    };
    const bool usual = scale.usual();
    auto histogram = [&](bool counts) {
        clear();
        row.template each<2>(tid, [&](int, float x) {
            uint32_t digit;
            uint64_t m;
            if (usual) {                               // (NaN and -infinity in the last digit, without mass)
                digit = (uint32_t)fminf((top - x) * per_t * 64.0f, (float)(kBins - 1));
                m = scale.usual_mass(x);
            } else {
                x = cleaned(x);
                digit = scale.bin(x);
                m = scale.mass(x);
            }
            if (counts) atomicAdd(&count[digit], 1u);
            if (m) atomicAdd((unsigned long long*)&mass[digit], (unsigned long long)m);
        });
    };
    // as resolve, for a digit of the whole row: 51 bits of key in five digits
    auto descend = [&](const Found& in, bool by_mass, uint64_t need) {
        uint64_t above = 0, up_to = 0;
        const int shifts[5] = {40, 29, 19, 9, 0}, widths[5] = {11, 11, 10, 10, 9};
        for (int level = 0; level < 5; ++level) {
            const int shift = shifts[level], width = widths[level];
            const uint32_t ones = (1u << width) - 1;
            afresh();
            clear();
            row.each(tid, [&](int i, float x) {
                x = cleaned(x);
                const uint64_t key = key_of(x, i);
                if (scale.bin(x) == in.digit && (level == 0 || key >> (shift + width) == above)) put(ones - ((uint32_t)(key >> shift) & ones), x);
            });
            const Found f = find(scan(yes, yes, count, mass), by_mass, need);
            above = above << width | (ones - f.digit);
            need -= by_mass ? f.mass_before : f.count_before;
            up_to += f.mass_before + (level == 4 ? f.mass : 0);
        }
        if (tid == 0) { shared_key = above; shared_mass = up_to; }
        __syncthreads();
    };

    // Masses of runs of 512 pieces, eight a lane (head and tail of the row are runs of their own), and the run in which the token is
    // again.  (A thread's sum of whole numbers, 520 of 2^43 at most, is exact in a double.)
    constexpr int kLines = 8, kBatch = 16 / kEach;
    const int runs = (row.pieces + 64 * kLines - 1) / (64 * kLines), all = runs + 2;
    auto sum_runs = [&](auto end_of, auto piece_of) {
        afresh();
        __syncthreads();
        for (int s = wave; s < all; s += kWaves) {
            uint64_t x = 0;                            // (512 pieces can pass 2^53)
            if (s == 0 || s == all - 1) {
                x = (uint64_t)end_of(s);
            } else {
                const int v0 = (s - 1) * 64 * kLines + lane;
                double y = 0.0;
#pragma unroll 1
                for (int q0 = 0; q0 < kLines; q0 += kBatch) {
                    uint4 b[kBatch];
#pragma unroll
                    for (int q = 0; q < kBatch; ++q) b[q] = row.bits(min(v0 + (q0 + q) * 64, row.pieces - 1));
#pragma unroll
                    for (int q = 0; q < kBatch; ++q)
                        if (v0 + (q0 + q) * 64 < row.pieces) y += piece_of(v0 + (q0 + q) * 64, Row<T>::unpacked(b[q]));
                }
                x = (uint64_t)y;
            }
            x = sum_up_to(x);
            if (lane == 63) run_mass[s] = x;
        }
        __syncthreads();
    };
    bool summed = false;                               // (the runs)
    auto value_of = [](uint64_t key) {
        const uint32_t b = (uint32_t)(key >> 19);
        return __uint_as_float(b ^ ((b >> 31) ? 0x80000000u : 0xffffffffu));
    };
    // As resolve, for `here` keys in `many`: digits of 11 bits of what is left of their range, until there is one (keys are unlike).
    auto resolve_many = [&](int here, uint32_t* counts, uint64_t* masses, bool by_mass, uint64_t need) {
        afresh();
        uint64_t low = ~(uint64_t)0, high = 0, before = 0;
        for (int i = tid; i < here; i += kThreads) { low = min(low, many[i]); high = max(high, many[i]); }
        low = up_to(low, ~(uint64_t)0, [](uint64_t x, uint64_t y) { return min(x, y); });
        high = up_to(high, (uint64_t)0, [](uint64_t x, uint64_t y) { return max(x, y); });
        if (lane == 63) { wave_low[wave] = low; wave_mass[wave] = high; }
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) { low = min(low, wave_low[w]); high = max(high, wave_mass[w]); }
        for (;;) {
            const int shift = max(53 - __clzll(high - low | 1), 0);
            __syncthreads();
            for (int x = tid; x < kBins; x += kThreads) { counts[x] = 0; masses[x] = 0; }
            __syncthreads();
            for (int i = tid; i < here; i += kThreads) {
                const uint64_t key = many[i];
                if (key > high || key < low) continue;
                const uint32_t digit = (uint32_t)((high - key) >> shift);
                atomicAdd(&counts[digit], 1u);
                atomicAdd((unsigned long long*)&masses[digit], (unsigned long long)scale.mass(value_of(key)));
            }
            const Found f = find(scan(yes, yes, counts, masses), by_mass, need);
            high -= (uint64_t)f.digit << shift;
            low = max(low, high - (((uint64_t)1 << shift) - 1));
            before += f.mass_before;
            if (f.count == 1) {
                for (int i = tid; i < here; i += kThreads)
                    if (many[i] <= high && many[i] >= low) { shared_key = many[i]; shared_mass = before + f.mass; }
                __syncthreads();
                return;
            }
            need -= by_mass ? f.mass_before : f.count_before;
        }
    };
    // The cut by count, then the one by mass.  The last one's digit is gathered in the pass that adds up the runs.
    uint64_t total = 0;
    bool gone = false;                                 // (the histogram)
    const int first = k < V ? 0 : 1, last_cut = p < 1.0f ? 1 : 0;
#pragma unroll 1
    for (int cut = first; cut <= last_cut; ++cut) {
        const bool by_mass = cut == 1, is_last = cut == last_cut;
        afresh();
        uint32_t &pieces = filled[5 + cut], &keys = filled[8 + cut];
        if (cut == first || gone) histogram(!by_mass);
        const Sums sums = scan(yes, yes, count, mass);
        if (cut == first) total = sums.all_m;
        uint64_t need = by_mass ? mass_needed(total) : (uint64_t)k;
        const Found in = find(sums, by_mass, need);
        need -= by_mass ? in.mass_before : in.count_before;
        const float from_digit = (float)in.digit, behind = in.digit < kBins - 1 ? (float)(in.digit + 1) : NAN;
        const float low = top - (behind / (64.0f * per_t) * 1.0001f + fabsf(top) * 1e-6f);
        auto take = [&](int i, float x) {
            x = cleaned(x);
            if (scale.bin(x) != in.digit) return;
            const uint32_t to = atomicAdd(&keys, 1u);
            if (to < kCandidates) many[to] = key_of(x, i);
        };
        // the mass of a piece's entries that are kept for certain; pieces with entries of the digit are looked into afterwards
        auto look = [&](int v, const typename Row<T>::Piece& y) {
            double sum = 0.0;
            bool any = false;
            if (!usual) {
#pragma unroll 1
                for (int e = 0; e < kEach; ++e) {
                    const float x = cleaned(row.at(row.head + v * kEach + e));
                    any |= scale.bin(x) == in.digit;
                    if (scale.bin(x) < in.digit && !(scale.weight(x) < min_p)) sum += (double)scale.whole_mass(x);
                }
            } else if (!(Row<T>::top_of(y) < low)) {
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const float d = (top - y.x[e]) * per_t * 64.0f, w = scale.usual_weight(y.x[e]), m = Scale::whole(w);
                    any |= !(d < from_digit) && !(d >= behind);
                    sum += (double)(d < from_digit && !(w < min_p) ? m : 0.0f);
                }
            }
            if (any) {
                const uint32_t to = atomicAdd(&pieces, 1u);
                if (to < kCandidates) hot[to] = (uint32_t)v;
            }
            return sum;
        };
        if (!is_last) {
            row.template visit<2>(tid, look, take);
        } else {
            sum_runs([&](int s) {
                const int n = s ? row.tail : row.head, i = s ? V - row.tail + lane : lane;
                if (lane >= n) return 0.0;
                const float x = cleaned(row.at(i));
                take(i, x);
                return scale.bin(x) < in.digit && !(scale.weight(x) < min_p) ? (double)scale.whole_mass(x) : 0.0;
            }, look);
        }
        __syncthreads();
        afresh();
        for (int j = tid; j < min((int)pieces, kCandidates) * kEach; j += kThreads) {
            const int i = row.head + (int)hot[j / kEach] * kEach + j % kEach;
            take(i, row.at(i));
        }
        __syncthreads();
        if ((int)pieces > kCandidates || (int)keys > kCandidates) {
            descend(in, by_mass, need);
            gone = true;
        } else {
            const int here = (int)keys;
            // (the histogram is still needed behind the cut by count, the runs' masses behind the last)
            resolve_many(here, is_last ? count : top_count, is_last ? mass : run_mass, by_mass, need);
            if (is_last) {
                for (int j = tid; j < here; j += kThreads) {
                    const uint64_t key = many[j];
                    const int i = kMostVocab - 1 - (int)(key & (kMostVocab - 1)), v = i - row.head;
                    const float x = value_of(key);
                    if (key >= shared_key && !(scale.weight(x) < min_p))
                        atomicAdd((unsigned long long*)&run_mass[v < 0 ? 0 : v >= row.pieces * kEach ? all - 1 : 1 + v / (kEach * 64 * kLines)],
                                  (unsigned long long)scale.mass(x));
                }
                summed = true;
                __syncthreads();
            }
        }
        last_kept = value_of(shared_key);
        last_index = kMostVocab - 1 - (int)(shared_key & (kMostVocab - 1));
        total = in.mass_before + shared_mass;
    }
    // entries below this have no mass, or less weight than min_p (a little room for the roundings), or are behind the end
    float low = fmaxf(min_p > 0.0f ? logf(min_p) - 0.001f : -30.0f, -30.0f);
    if (last_kept > -INFINITY && last_kept < INFINITY) low = fmaxf(low, (last_kept - top) * scale.per_t);
    const bool uncut = usual && last_kept == -INFINITY && !(min_p > 0.0f);
    auto amount = [&](int i, float x) -> float {
        const float w = usual ? scale.usual_weight(x) : scale.weight(cleaned(x));
        return (x > last_kept || (x == last_kept && i <= last_index)) && !(w < min_p) ? Scale::whole(w) : 0.0f;
    };
    auto ends = [&](int s) -> double {                 // head (run 0) and tail (the last): an entry a lane
        const int n = s ? row.tail : row.head, i = s ? V - row.tail + lane : lane;
        return lane < n ? (double)amount(i, row.at(i)) : 0.0;
    };
    auto in_piece = [&](int v, const typename Row<T>::Piece& y, double (&m)[kEach]) {      // (whole numbers below 2^53, added up exactly)
        double sum = 0.0;
        if (uncut) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum += m[e] = (double)Scale::whole(scale.usual_weight(y.x[e]));
        } else if (!usual || (Row<T>::top_of(y) - top) * scale.per_t >= low) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum += m[e] = (double)amount(row.head + v * kEach + e, y.x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e) m[e] = 0.0;
        }
        return sum;
    };
    double m[kEach];
    afresh();
    if (!summed) sum_runs(ends, [&](int v, const typename Row<T>::Piece& y) { return in_piece(v, y, m); });
    uint64_t sum = 0;
    for (int s = tid; s < all; s += kThreads) sum += run_mass[s];
    const uint64_t need = mass_passed(add_up(sum)) + 1;
    if (wave) return;
    uint64_t before = 0;
    for (int s0 = 0; s0 < all; s0 += 64) {
        const uint64_t x = sum_up_to(s0 + lane < all ? run_mass[s0 + lane] : 0);
        const uint64_t hit = __ballot(before + x >= need);
        if (!hit) {
            before += of_lane(x, 63);
            continue;
        }
        const int f = __ffsll((unsigned long long)hit) - 1, s = s0 + f;
        if (f) before += of_lane(x, f - 1);
        const bool at_end = s == 0 || s == all - 1;
        for (int q = 0; q < kLines; ++q) {             // the run's lines of 64 pieces
            const int v = ((s - 1) * kLines + q) * 64 + lane;
            uint64_t mine = 0;
            if (at_end) mine = (uint64_t)ends(s);
            else if (v < row.pieces) mine = (uint64_t)in_piece(v, row.piece(v), m);
            const uint64_t z = sum_up_to(mine);
            const uint64_t here = __ballot(before + z >= need);
            if (!here) {
                before += of_lane(z, 63);
                continue;
            }
            if (lane == __ffsll((unsigned long long)here) - 1) {
                before += z - mine;
                int e = 0;
#pragma unroll
                for (int y = 0; y < kEach - 1; ++y) {
                    before += (uint64_t)m[y];
                    if (before < need) e = y + 1;
                }
                a.token[r] = s == 0 ? lane : s == all - 1 ? V - row.tail + lane : row.head + v * kEach + e;
            }
            break;
        }
        return;
    }
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
    SampleArgs a = {d->logits, d->row_stride, d->n_vocab, d->temperature, d->top_p, d->min_p, d->uniform, d->top_k, d->token};
    for (int64_t left = d->n_rows; left > 0;) {
        const int64_t n = std::min<int64_t>(left, kMostThreads / kThreads);
        const dim3 grid((unsigned)n);
        if (d->dtype == FR_DTYPE_BF16) hipLaunchKernelGGL(k_sample<Bf16>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        else if (d->dtype == FR_DTYPE_F16) hipLaunchKernelGGL(k_sample<F16>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(k_sample<F32>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        if ((left -= n) == 0) break;
        a.logits = static_cast<const char*>(a.logits) + n * a.row_stride * (int64_t)size;
        a.uniform += n, a.token += n;
        if (a.temperature) a.temperature += n;
        if (a.top_k) a.top_k += n;
        if (a.top_p) a.top_p += n;
        if (a.min_p) a.min_p += n;
    }
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}

}  // extern "C"
