// Attention of a batch of sequences to keys and values held in 8 bits, to all of them or to a window and the first few.
//
// A query row q (a token, a head) that sees keys k_j with values v_j gets  out = sum_j w_j v_j / sum_j w_j,  w_j = exp(s_j - m),
// s_j = scale q . k_j,  and lse = m + log sum_j w_j, for whatever m: the largest score seen so far.  Where m rises, the sums so far
// are multiplied by exp(m_before - m), so that one pass over the keys is enough, and parts of the keys, each with its own m, are
// joined in the same way.  Scores, m, both sums and the parts' results are of 32 bits; weights are rounded to the 16-bit type for the
// product with the values, and the result is, once.  Codes times their block's power of two are numbers of that type, exactly.
//
// The heads that share a key head, and all tokens of a sequence, are rows of one matrix product with its keys.
// What bounds it:
//   Decoding from long caches, the reading: 128 sequences of 4096 keys each with 8 key heads, 1.07 GB, 192 us, 5.6 TB/s (the same loads without a
//     product 5.9; a kernel that only reads one array from end to end 6.5).  Where lengths differ, units that have nothing left: 8 of 20000 to 65536
//     131 us, 4.9 TB/s, 64 of up to 4000 76 us, 3.6.
//   Prompts, the vector units beside the matrix cores (2 exps and 5 other operations of every two weights, and half a conversion of a code):
//     8 sequences of 2048 tokens behind 6144, 32 heads, 1.92 TFLOP in 2.0 ms, 0.96 PFLOP/s.
//   A few short sequences, the launch: 6 us.

#include <algorithm>
#include <cmath>

#include "attend_tiles.h"
#include "common.h"
#include "kv8.h"

namespace {

// What a workgroup's four wavefronts do.  kFewRows: 16 rows, and every wavefront takes every fourth tile of 32 keys for itself, the four
// results being joined at the end.  kWideRows: 128 rows, 32 a wavefront, which share tiles of 64 keys.
enum Kind { kFewRows, kWideRows };
constexpr int columns(Kind k) { return k == kWideRows ? 32 : 16; }                     // rows of a wavefront: columns of its MFMA blocks
constexpr int rows_of(Kind k) { return k == kWideRows ? kWaves * 32 : 16; }            // rows of an item
constexpr int keys_of(Kind k) { return k == kWideRows ? 64 : 32; }                     // keys of a tile

struct Attend8Args {
    fr_kv8_pages c;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_stride, out_stride, pages_stride;
    const int32_t *q_begin, *pages, *lens;
    int32_t n_tokens, n_seqs, n_q_heads, max_q, max_len, window, sinks, page_shift, block_shift, group;
    float q_power, rate;                   // scale * log2 e = q_power * rate: a power of two, 1 at most, that goes into the queries, and the rest
    int32_t row_tiles, splits, split_len;  // row tiles of a sequence and key head; parts of its tiles of keys, and their length
    int32_t groups, units, first_unit;
    int32_t workers;                       // of a key head, among which its tiles of keys are dealt out evenly
    float* part_o;                         // [(group's sequence and key head, part), row tile][rows_of][head_dim], relative to 2^m
    float2* part_ml;                       // the same: m in powers of 2, sum
};

// The keys that rows of tokens i0 .. i1 see, in tiles: those that hold the first `few` keys, then those from `start` (of token i0) to
// `end` (of token i1); tile u begins with key first(u).
template <int kTile> struct Keys {
    int32_t start, few, end, few_tiles, skipped, tiles;
    __device__ __forceinline__ Keys(const Attend8Args& a, int n0, int i0, int i1)
    {
        end = max(0, n0 + i1);
        start = a.window ? max(0, max(0, n0 + i0) - a.window) : 0;
        few = min(a.sinks, start);
        few_tiles = (few + kTile - 1) / kTile;
        skipped = start / kTile - few_tiles;
        if (skipped <= 0) few_tiles = skipped = 0;             // (nothing between the two)
        tiles = (end + kTile - 1) / kTile - skipped;
    }
    __device__ __forceinline__ int first(int u) const { return (u < few_tiles ? u : u + skipped) * kTile; }
    // a key that some row sees in place of one that none does
    __device__ __forceinline__ int seen(int j) const { return j >= end ? end - 1 : j >= few && j < start ? start : j; }
    __device__ __forceinline__ bool all_seen(int first) const { return first + kTile <= end && (first >= start || first + kTile <= few); }
};

// A sequence's part in the call.
struct Sequence {
    int32_t token0, tokens, n0;            // first token; how many are computed; keys that the first one has up to itself (0 and less: none)
    __device__ __forceinline__ Sequence(const Attend8Args& a, int b)
    {
        const int t0 = a.q_begin ? within(a.q_begin[b], 0, a.n_tokens) : b, t1 = a.q_begin ? within(a.q_begin[b + 1], t0, a.n_tokens) : b + 1;
        const int len = a.max_len ? within(a.lens[b], 0, a.max_len) : 0;
        token0 = t0;
        tokens = min(t1 - t0, a.max_q);
        n0 = len - (t1 - t0) + 1;
    }
};

typedef __attribute__((address_space(3))) uint64_t* LdsOffset;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((address_space(3))) f32x2* LdsPair;
typedef __attribute__((address_space(3))) u32x4* LdsWide;
typedef __attribute__((address_space(3))) f32x4* LdsFloats;

// Two codes of a register, times a power of two, as two numbers of the type.
template <typename T, bool kHigh> __device__ __forceinline__ uint32_t two_numbers(uint32_t codes, float power)
{
    if constexpr (std::is_same_v<T, Bf16>) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, kHigh));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, power, kHigh));
}
template <typename T> __device__ __forceinline__ u32x4 eight_numbers(uint32_t lo, uint32_t hi, float power)
{
    return (u32x4){two_numbers<T, false>(lo, power), two_numbers<T, true>(lo, power), two_numbers<T, false>(hi, power), two_numbers<T, true>(hi, power)};
}

// Codes that are NaN: their bytes' top bits.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t nan_or_0(uint32_t w) { return w & ~((nan_codes(w) >> 7) * 255u); }
__device__ __forceinline__ uint4 without_nan(uint4 w) { return make_uint4(nan_or_0(w.x), nan_or_0(w.y), nan_or_0(w.z), nan_or_0(w.w)); }

// Where a row's result goes.
struct Rows {
    const Attend8Args& a;
    int32_t kv, token0, n0;
    __device__ __forceinline__ int32_t token(int r) const { return token0 + r / a.group; }
    __device__ __forceinline__ int32_t head(int r) const { return kv * a.group + r % a.group; }
    __device__ __forceinline__ int32_t keys(int r) const { return max(0, n0 + r / a.group); }
};

template <Kind kKind, int D> struct Lds8 {
    static constexpr uint32_t kTiles = kKind == kWideRows ? 512 * D : kWaves * 64 * D;      // K and V, two tiles each; of few rows, V of a tile a wavefront
    static constexpr uint32_t kTable = kWaves * 2048;                                       // a wavefront: two sets of 64 offsets, two of 64 pairs of powers
};

// The work of one workgroup: rows `row0` .. of `rows` against tiles u0 .. u1 of their keys.
//
// kFewRows: 16 rows, blocks of 16 x 16 x 32.  Codes come to registers, a tile ahead, 8 KB a wavefront at head_dim 128; with what a lane's
// places are made anew where they are used, its registers leave room for four workgroups a unit (166 -> 123, 127 where tiles are dealt out evenly, of 128 that
// four have; 128 sequences' windows of 4096 keys, fp16, 64 heads, 207 -> 185 us).  A lane's 16 bytes of a key are two fragments; values are made into numbers on the way
// into LDS, where they are transposed.
//
// kWideRows: a wavefront's 32 rows are the columns of 32 x 32 x 16 blocks; weights go from the one product to the next without passing
// through LDS.  A wavefront makes a quarter of every tile's codes into numbers, which all four then read: 32 conversions beside 32 MFMAs.
// 8 ragged sequences of up to 2048 tokens: scores, weights and values of a tile one after another 776 us, the next tile's scores beside this one's weights
// 744; with places in LDS worked out for every piece 820, conversions where the codes come instead of between the MFMAs 756.
template <typename T, int D, Kind kKind>
__device__ __forceinline__ void attend(const Attend8Args& a, const Rows& rows, int n_rows, int row0, const Keys<keys_of(kKind)>& keys, int u0, int u1,
                                       const int32_t* pages, bool whole, int64_t part, char* lds_array)
{
    constexpr bool kWide = kKind == kWideRows;
    constexpr int kCols = columns(kKind), kTile = keys_of(kKind);
    constexpr int kSharers = kKind == kFewRows ? kWaves : 1;
    typedef Lds<D, kCols> L;
    // (weights of bfloat16 are 2^-20, or 2^-12 where the maximum lags, so that sums of values as large as the type's largest stay in range; of
    // values near its smallest number, 2^-126, the sums still have steps of 2^-129)
    typedef Softmax<T, D, kCols, std::is_same_v<T, F16> ? 7 : -20> State;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                        // (what is made of it is made for every item, not kept from one to the next)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds = (uint32_t)reinterpret_cast<uintptr_t>((LdsBytes)lds_array);
    const float c = a.rate;

    // the wavefront's rows
    const int row_first = row0 + (kWide ? wave * kCols : 0), row_here = min(row_first + lane % kCols, n_rows - 1);
    const bool idle = row_first >= n_rows;
    const int n = rows.keys(row_here), from = a.window ? n - a.window : 0;
    // what all rows of the wavefront see needs no look
    const int n_least = rows.keys(min(row_first, n_rows - 1)), from_most = a.window ? rows.keys(min(row_first + kCols, n_rows) - 1) - a.window : 0;
    State x;
    {
        // Few rows: a lane's 16 bytes of a key are the elements of two fragments, so that those of a query are taken in the same order.
        const uint16_t* q = a.q + rows.token(row_here) * a.q_stride + (int64_t)rows.head(row_here) * D;
#pragma unroll
        for (int f = 0; f < D * kCols / 512; ++f)
        {
            uint4 w = *reinterpret_cast<const uint4*>(q + (kWide ? f * 16 + lane / kCols * 8 : f / 2 * 64 + lane / kCols * 16 + f % 2 * 8));
            if constexpr (std::is_same_v<T, Bf16>) {
                auto times = [&](uint32_t y) { return T::pack(T::up((uint16_t)y) * a.q_power, T::up((uint16_t)(y >> 16)) * a.q_power); };
                w = make_uint4(times(w.x), times(w.y), times(w.z), times(w.w));
            }
            x.q[f] = __builtin_bit_cast(typename T::x8, w);
        }
    }

    // What a lane's places are is made anew from `anew()`: kept, they hold registers that the loop needs.
    auto anew = [&] { int l = lane; asm volatile("" : "+v"(l)); return l; };
    // Where keys lie.  A wavefront loads kLoadRows rows of a tile; 64 of them are a set, those of two or four tiles, a lane each: the page id
    // comes first, then the offset goes to LDS, and the scales' bytes, when they are here, as powers of two.
    constexpr int kLoadRows = kWide ? 16 : 32, kTilesASet = 64 / kLoadRows;
    const uint32_t offsets = lds + Lds8<kKind, D>::kTiles + wave * 2048, powers = offsets + 1024;
    const int mine = kKind == kFewRows ? wave : 0, tiles = (u1 - u0 - mine + kSharers - 1) / kSharers;
    auto tile_of = [&](int t) { return u0 + t * kSharers + mine; };
    const uint8_t* gk = static_cast<const uint8_t*>(a.c.k) + rows.kv * a.c.head_stride;
    const uint8_t* gv = static_cast<const uint8_t*>(a.c.v) + rows.kv * a.c.head_stride;
    int32_t id;
    uint8_t k_byte, v_byte;
    auto key_of = [&](int set) {
        const int l = anew(), u = min(tile_of(set * kTilesASet + l / kLoadRows), u1 - 1);
        return keys.seen(keys.first(u) + (kWide ? wave * 16 : 0) + l % kLoadRows);
    };
    auto ask_ids = [&](int set) { id = pages[key_of(set) >> a.page_shift]; };
    auto make_offsets = [&](int set) {
        const int slot = key_of(set) & (a.c.page_size - 1);
        const uint64_t page = (uint64_t)(uint32_t)within(id, 0, (int32_t)a.c.n_pages - 1);
        *reinterpret_cast<LdsOffset>(lds_at(offsets + (set & 1) * 512 + anew() * 8)) = page * (uint32_t)a.c.page_stride + (uint64_t)(uint32_t)slot * (uint32_t)a.c.slot_stride;
        const uint64_t at = page * (uint32_t)a.c.scale_page_stride + (uint64_t)(uint32_t)rows.kv * (uint32_t)a.c.scale_head_stride +
                            (uint64_t)(uint32_t)(slot >> a.block_shift) * (uint32_t)a.c.scale_block_stride;
        k_byte = a.c.k_scale[at];
        v_byte = a.c.v_scale[at];
    };
    auto make_powers = [&](int set) {
        *reinterpret_cast<LdsPair>(lds_at(powers + (set & 1) * 512 + anew() * 8)) = f32x2{power_of(scale_byte<T>(k_byte)), power_of(scale_byte<T>(v_byte))};
    };
    auto offset_at = [&](int t, int r) { return *reinterpret_cast<LdsOffset>(lds_at(offsets + (t / kTilesASet & 1) * 512 + ((t % kTilesASet) * kLoadRows + r) * 8)); };
    auto power_at = [&](int t, int r, bool value) {
        return (*reinterpret_cast<LdsPair>(lds_at(powers + (t / kTilesASet & 1) * 512 + ((t % kTilesASet) * kLoadRows + r) * 8)))[value];
    };
    // Values: a lane has 16 codes of a row, kLanes lanes a row.
    constexpr int kLanes = D / 16, kRowsAtOnce = 64 / kLanes, kLoads = kLoadRows / kRowsAtOnce;
    // Rows of values that no row of queries sees become zeros (their weights are 0, but 0 times NaN is not); with `clean`, NaN does everywhere.
    bool clean = false;
    auto fit = [&](uint4 w, int first, int r) {
        if (!keys.all_seen(first)) {
            const int j = first + r;
            if (keys.seen(j) != j) w = make_uint4(0, 0, 0, 0);
        }
        return clean ? without_nan(w) : w;
    };
    auto put = [&](uint32_t tile, int r, int piece, uint32_t order, uint4 w, float power) {
        const uint32_t at = tile + r * L::kRow + ((2 * piece) ^ order) * 16;
        *reinterpret_cast<LdsWide>(lds_at(at)) = eight_numbers<T>(w.x, w.y, power);
        *reinterpret_cast<LdsWide>(lds_at(at ^ 16)) = eight_numbers<T>(w.z, w.w, power);
    };
    // Scores of keys that a row does not see.
    typedef typename State::Block Block;
    auto hide = [&](Block (&s)[2], int first) {
        if (first + kTile <= n_least && (first >= from_most || first + kTile <= a.sinks)) return;
        const int l = anew();
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < State::kInBlock; ++i) {
                const int j = first + b * kCols + State::in_block(i, l);
                if (j >= n || (j < from && j >= a.sinks)) s[b][i] = -INFINITY;
            }
    };

    auto pass = [&] {
        x.start();
        if (tiles <= 0) return;
        if constexpr (!kWide) {
            const uint32_t v = lds + wave * 64 * D;
            Fragments<T, D, kCols> fragments(v, lane);
            uint4 kw[2][D / 64], vw[kLoads];
            auto load_k = [&](int t) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int l = anew();
                    const uint8_t* at = gk + offset_at(t, b * 16 + l % 16) + l / 16 * 16;
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) kw[b][h] = *reinterpret_cast<const uint4*>(at + h * 64);
                }
            };
            auto load_v = [&](int t) {
                const int l = anew();
#pragma unroll
                for (int y = 0; y < kLoads; ++y) vw[y] = *reinterpret_cast<const uint4*>(gv + offset_at(t, y * kRowsAtOnce + l / kLanes) + l % kLanes * 16);
            };
            ask_ids(0);
            make_offsets(0);
            if (tiles > kTilesASet) ask_ids(1);
            load_k(0);
            load_v(0);
            make_powers(0);
            for (int t = 0; t < tiles; ++t) {
                const bool more = t + 1 < tiles;
                const int first = keys.first(tile_of(t));
                if (t % 2 == 0 && t + 2 < tiles) {
                    make_offsets(t / 2 + 1);
                    if (t + 4 < tiles) ask_ids(t / 2 + 2);
                }
                f32x4 s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float power = power_at(t, b * 16 + anew() % 16, false);
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) {
                        s[b] = mfma(__builtin_bit_cast(typename T::x8, eight_numbers<T>(kw[b][h].x, kw[b][h].y, power)), x.q[2 * h], s[b]);
                        s[b] = mfma(__builtin_bit_cast(typename T::x8, eight_numbers<T>(kw[b][h].z, kw[b][h].w, power)), x.q[2 * h + 1], s[b]);
                        keep_order();                      // (a fragment's registers, not all fragments': four workgroups a unit)
                    }
                }
                if (more) load_k(t + 1);
                const int l = anew();
#pragma unroll
                for (int y = 0; y < kLoads; ++y) {
                    const int r = y * kRowsAtOnce + l / kLanes;
                    put(v, r, l % kLanes, L::fv(r), fit(vw[y], first, r), power_at(t, r, true));
                    keep_order();
                }
                if (more) load_v(t + 1);
                if (t % 2 == 1 && more) make_powers(t / 2 + 1);
                hide(s, first);
                float top = s[0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i / 4][i % 4]);
                x.grow(top_of_row<kCols>(top), c);
                const float zero = x.zero_point();
                uint32_t p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = x.weigh_from(s[e / 2][2 * e % 4], s[e / 2][2 * e % 4 + 1], c, zero);
                wait_lds();
                asm volatile("" : "+v"(fragments.v));
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
                    x.o[d] = mfma(fragments.of_v(0, d), State::fragment(p), x.o[d]);
                    if (d % 4 == 3) keep_order();
                }
                wait_lds();
            }
        } else {
            // While tile t's scores become weights (vector unit), the matrix cores make those of tile t + 1, and the codes of K of t + 2 and V of
            // t + 1 become numbers in LDS; those of K of t + 3 and V of t + 2 are asked for behind that.  Scores are made less the maximum: the
            // products' sum starts with it.
            constexpr uint32_t kHalf = kTile * L::kRow;
            constexpr int kSteps = D / 8;                   // MFMAs of the scores, and as many with the values
            constexpr int kAhead = 4;                       // fragments read ahead of their MFMA
            constexpr int kPairsBeside = D == 128 ? 10 : 8; // of 16 pairs of weights, those beside the scores' MFMAs; the rest are beside the first half of the values'
            Fragments<T, D, kCols> fragments(lds, lane);
            typename T::x8 ahead[kAhead];
            auto k_of = [&](auto odd, int y) { return fragments.of_k(odd * kHalf + y % 2 * 32 * L::kRow, y / 2); };
            auto v_of = [&](auto odd, int y) { return fragments.of_v((2 + odd) * kHalf + y / (D / 32) * 16 * L::kRow, y % (D / 32)); };
            u32x4 kw[kLoads], vw[kLoads];
            auto load = [&](u32x4 (&w)[kLoads], const uint8_t* from, int t) {
                const int l = anew(), to = min(t, tiles - 1);
#pragma unroll
                for (int y = 0; y < kLoads; ++y) w[y] = *reinterpret_cast<const u32x4*>(from + offset_at(to, y * kRowsAtOnce + l / kLanes) + l % kLanes * 16);
            };
            // powers of two of the lane's rows of tile t; half a lane's codes of a row into tile `odd` of K (V)
            auto powers_of = [&](float (&w)[kLoads], int t, bool value) {
                const int l = anew(), of = min(t, tiles - 1);
#pragma unroll
                for (int y = 0; y < kLoads; ++y) w[y] = power_at(of, y * kRowsAtOnce + l / kLanes, value);
            };
            float kp[kLoads], vp[kLoads];
            // (rows y kRowsAtOnce further down have another order of pieces, in bits that the lane's own leave alone)
            const uint32_t my_row = wave * 16 + lane / kLanes;
            uint32_t k_at = lds + my_row * L::kRow + ((2 * (lane % kLanes)) ^ L::fk(my_row)) * 16, v_at = lds + 2 * kHalf + my_row * L::kRow + ((2 * (lane % kLanes)) ^ L::fv(my_row)) * 16;
            auto made_here = [&](uint32_t lo, uint32_t hi, float power) {       // (not where the codes come: the numbers take twice their registers)
                asm volatile("" : "+v"(lo), "+v"(hi));
                return eight_numbers<T>(lo, hi, power);
            };
            auto put_k = [&](uint32_t odd, int e) {
                const int y = e / 2;
                *reinterpret_cast<LdsWide>(lds_at(k_at ^ ((L::fk(y * kRowsAtOnce) ^ e % 2) * 16)) + odd * kHalf + y * kRowsAtOnce * L::kRow) =
                    made_here(kw[y][e % 2 * 2], kw[y][e % 2 * 2 + 1], kp[y]);
            };
            auto put_v = [&](uint32_t odd, int e) {
                const int y = e / 2;
                *reinterpret_cast<LdsWide>(lds_at(v_at ^ ((L::fv(y * kRowsAtOnce) ^ e % 2) * 16)) + odd * kHalf + y * kRowsAtOnce * L::kRow) =
                    made_here(vw[y][e % 2 * 2], vw[y][e % 2 * 2 + 1], vp[y]);
            };
            auto fit_v = [&](int t) {
                const int first = keys.first(u0 + t);
                if (!keys.all_seen(first) || clean) {
#pragma unroll
                    for (int y = 0; y < kLoads; ++y) vw[y] = __builtin_bit_cast(u32x4, fit(__builtin_bit_cast(uint4, vw[y]), first, wave * 16 + y * kRowsAtOnce + anew() / kLanes));
                }
            };
            f32x16 minus;
#pragma unroll
            for (int i = 0; i < 16; ++i) minus[i] = 0.0f;
            float top = -INFINITY;
            auto tops = [&](const f32x16 (&s)[2], int e) { top = fmaxf(top, s[e / 16][e % 16]); };
            auto step = [&](f32x16 (&now)[2], f32x16 (&next)[2], int t, auto here, auto other) {      // (here: t modulo 2)
                __syncthreads();                            // K of t + 1 and V of t are here; K of t and V of t - 1 are done with
                powers_of(kp, t + 2, false);
                powers_of(vp, t + 1, true);
                fit_v(t + 1);
                if (idle) {
#pragma unroll
                    for (int e = 0; e < 2 * kLoads; ++e) put_k(here, e), put_v(other, e);
                } else {
                    asm volatile("" : "+v"(fragments.k), "+v"(fragments.v), "+v"(k_at), "+v"(v_at));        // (one register each, not one for every fragment)
#pragma unroll
                    for (int y = 0; y < kAhead; ++y) ahead[y] = k_of(other, y);
                    // a larger maximum, if the one in use lags behind by more than kSlack, or there has been none
                    if (__any((x.m == -INFINITY ? top + INFINITY : top * c) > kSlack)) {
                        // (exactly as much as the tile's scores exceed it: the maximum may be off by half an ulp then, which the next tile's scores show)
                        const bool none = x.m == -INFINITY;
                        const float more = none ? top == -INFINITY ? 0.0f : top : fmaxf(top, 0.0f), old = __builtin_amdgcn_exp2f(-more * c);
                        x.l *= none ? 1.0f : old;
                        x.l1 *= none ? 1.0f : old;
#pragma unroll
                        for (int d = 0; d < D / kCols; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) x.o[d][i] *= none ? 1.0f : old;
                        x.m = none ? top : x.m + more;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            now[0][i] -= more;
                            now[1][i] -= more;
                            minus[i] = -x.zero_point();
                        }
                    }
                    uint32_t p[16];
                    auto pair = [&](int e) {
                        p[e] = x.weigh_from(now[e / 8][2 * e % 16], now[e / 8][2 * e % 16 + 1], c, 0.0f);
                        asm volatile("" : "+v"(p[e]), "+v"(x.l), "+v"(x.l1));             // (made here, not where they are used)
                    };
                    keep_order();
#pragma unroll
                    for (int y = 0; y < kSteps; ++y) {          // (behind the last tile: of what lies there, not used)
                        next[y % 2] = mfma(ahead[y % kAhead], x.q[y / 2], y < 2 ? minus : next[y % 2]);
                        ahead[y % kAhead] = y + kAhead < kSteps ? k_of(other, y + kAhead) : v_of(here, y + kAhead - kSteps);
#pragma unroll
                        for (int e = y * kPairsBeside / kSteps; e < (y + 1) * kPairsBeside / kSteps; ++e) pair(e);
                        if (y % 2 == 0) {
                            if (y / 2 < 2 * kLoads) put_k(here, y / 2);
                            else put_v(other, y / 2 - 2 * kLoads);
                        }
                        keep_order();
                    }
                    hide(next, keys.first(u0 + t + 1));
                    top = -INFINITY;
                    keep_order();
                    // (in front of the tiles' loads: the compiler waits for those behind a load that may not have been asked for)
                    if (t % kTilesASet == 0) {
                        make_offsets(t / kTilesASet + 1);
                        ask_ids(t / kTilesASet + 2);
                    } else if (t % kTilesASet == 1) {
                        make_powers(t / kTilesASet + 1);
                    }
                    load(kw, gk, t + 3);
                    load(vw, gv, t + 2);
                    keep_order();
                    __builtin_amdgcn_s_setprio(1);              // (first to the matrix cores: the other workgroup's wavefront has weights to make)
#pragma unroll
                    for (int y = 0; y < kSteps; ++y) {
                        constexpr int kFirst = kSteps / 2, kRest = 16 - kPairsBeside;
                        const int f = y / (D / 32), d = y % (D / 32);
                        x.o[d] = mfma(ahead[y % kAhead], State::fragment(p + 4 * f), x.o[d]);
                        if (y + kAhead < kSteps) ahead[y % kAhead] = v_of(here, y + kAhead);
                        if (y < kFirst) {
#pragma unroll
                            for (int e = y * kRest / kFirst; e < (y + 1) * kRest / kFirst; ++e) pair(kPairsBeside + e);
                        } else {
#pragma unroll
                            for (int e = (y - kFirst) * 32 / kFirst; e < (y - kFirst + 1) * 32 / kFirst; ++e) tops(next, e);
                        }
                        keep_order();
                    }
                    __builtin_amdgcn_s_setprio(0);
                    top = top_of_row<kCols>(top);
                    return;
                }
                if (t % kTilesASet == 0) {
                    make_offsets(t / kTilesASet + 1);
                    ask_ids(t / kTilesASet + 2);
                } else if (t % kTilesASet == 1) {
                    make_powers(t / kTilesASet + 1);
                }
                load(kw, gk, t + 3);
                load(vw, gv, t + 2);
            };
            const std::integral_constant<uint32_t, 0> even{};
            const std::integral_constant<uint32_t, 1> odd{};
            ask_ids(0);
            make_offsets(0);
            ask_ids(1);
            load(kw, gk, 0);
            load(vw, gv, 0);
            make_powers(0);
            powers_of(kp, 0, false);
            powers_of(vp, 0, true);
#pragma unroll
            for (int e = 0; e < 2 * kLoads; ++e) put_k(even, e);
            load(kw, gk, 1);
            powers_of(kp, 1, false);
            fit_v(0);
#pragma unroll
            for (int e = 0; e < 2 * kLoads; ++e) put_v(even, e);
            load(vw, gv, 1);
#pragma unroll
            for (int e = 0; e < 2 * kLoads; ++e) put_k(odd, e);
            load(kw, gk, 2);
            __syncthreads();
            f32x16 s0[2], s1[2];
            if (!idle) {
#pragma unroll
                for (int y = 0; y < kSteps; ++y) s0[y % 2] = mfma(k_of(even, y), x.q[y / 2], y < 2 ? minus : s0[y % 2]);
                hide(s0, keys.first(u0));
#pragma unroll
                for (int e = 0; e < 32; ++e) tops(s0, e);
                top = top_of_row<kCols>(top);
            }
            for (int t = 0;; t += 2) {
                step(s0, s1, t, even, odd);
                if (t + 1 >= tiles) break;
                step(s1, s0, t + 1, odd, even);
                if (t + 2 >= tiles) break;
            }
        }
    };
    // A weight of 0 for a key that a row does not see, times NaN, is NaN: where rows see different keys and one of the results is NaN, the pass
    // is made again without the values' NaN, and then it is given to the rows that see it.
    for (;;) {
        pass();
        if (clean || n_rows <= a.group) break;
        bool bad = false;
#pragma unroll
        for (int d = 0; d < D / kCols; ++d)
#pragma unroll
            for (int i = 0; i < State::kInBlock; ++i) bad |= x.o[d][i] != x.o[d][i];
        bad &= !idle;
        clean = kWide ? (bool)__syncthreads_or(bad) : (bool)__any(bad);
        if (!clean) break;
    }
    if (__builtin_expect(clean, 0)) {
        for (int t = 0; t < tiles; ++t) {
            const int first = keys.first(tile_of(t)), j = first + lane;
            bool any = false;
            auto place = [&](int j) {
                const uint64_t page = (uint64_t)(uint32_t)within(pages[j >> a.page_shift], 0, (int32_t)a.c.n_pages - 1);
                return gv + page * (uint32_t)a.c.page_stride + (uint64_t)(uint32_t)(j & (a.c.page_size - 1)) * (uint32_t)a.c.slot_stride;
            };
            if (lane < kTile && keys.seen(j) == j) {
                const uint4* w = reinterpret_cast<const uint4*>(place(j));
#pragma unroll 1
                for (int e = 0; e < D / 16; ++e) any |= (nan_codes(w[e].x) | nan_codes(w[e].y) | nan_codes(w[e].z) | nan_codes(w[e].w)) != 0;
            }
#pragma unroll 1
            for (uint64_t left = __ballot(any); left; left &= left - 1) {
                const int y = first + __ffsll((unsigned long long)left) - 1;
                if (y >= n || (y < from && y >= a.sinks)) continue;
                const uint8_t* at = place(y);
#pragma unroll
                for (int d = 0; d < D / kCols; ++d)
#pragma unroll
                    for (int i = 0; i < State::kInBlock; ++i)
                        if ((at[d * kCols + State::in_block(i, lane)] & 0x7f) == 0x7f) x.o[d][i] = NAN;
            }
        }
    }
    x.l = sum_of_row<kCols>(x.l + x.l1);

    // results through LDS, so that rows are written whole: a wavefront's rows of D floats, 16-byte chunk c of row r at c ^ r
    constexpr uint32_t kFloatRow = D * 4, kFloatChunks = D / 4, kRegion = kCols * kFloatRow;
    static_assert(kWaves * kRegion <= Lds8<kKind, D>::kTiles, "");
    __syncthreads();                                              // tiles are done with
    const uint32_t region = lds + wave * kRegion, mls = lds + Lds8<kKind, D>::kTiles;
    auto ml = [&](int wv, int r) { return reinterpret_cast<LdsPair>(lds_at(mls + (wv * kCols + r) * 8)); };
    const float m2 = x.reference(c);                     // (-infinity stays: c is positive)
    float mine_of = 1.0f;
    if (lane < kCols) *ml(wave, lane) = f32x2{m2, x.l};
    if constexpr (kKind == kFewRows) {
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int y = 0; y < kWaves; ++y) top = fmaxf(top, (*ml(y, lane % kCols))[0]);
        mine_of = __builtin_amdgcn_exp2f(m2 - (top == -INFINITY ? 0.0f : top));
    }
#pragma unroll
    for (int d = 0; d < D / kCols; ++d)
#pragma unroll
        for (int i = 0; i < State::kInBlock; i += 4) {
            const uint32_t r = lane % kCols, chunk = (d * kCols + State::in_block(i, lane)) / 4;
            *reinterpret_cast<LdsFloats>(lds_at(region + r * kFloatRow + (chunk ^ (r & (kFloatChunks - 1))) * 16)) =
                f32x4{x.o[d][i] * mine_of, x.o[d][i + 1] * mine_of, x.o[d][i + 2] * mine_of, x.o[d][i + 3] * mine_of};
        }
    __syncthreads();
    // a thread takes eight elements of a row: two chunks, neighbours for a result of 16 bits, head_dim / 2 apart for a part (so that
    // neighbouring threads write neighbouring chunks)
    constexpr int kPieces = D / 8, kOutRows = rows_of(kKind);
    for (int y = tid; y < kOutRows * kPieces; y += kThreads) {
        const int r = y / kPieces, piece = y % kPieces, to = row0 + r;
        if (to >= n_rows) break;
        f32x4 lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
        float top, sum;
        const int in = r % kCols;
        auto chunk = [&](int wv, int e) {
            return *reinterpret_cast<LdsFloats>(lds_at(lds + wv * kRegion + in * kFloatRow + ((uint32_t)(whole ? 2 * piece + e : piece + e * kPieces) ^ (in & (kFloatChunks - 1))) * 16));
        };
        if constexpr (kKind != kFewRows) {
            const int wv = r / kCols;
            lo = chunk(wv, 0), hi = chunk(wv, 1);
            top = (*ml(wv, in))[0], sum = (*ml(wv, in))[1];
        } else {
            top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int wv = 0; wv < kWaves; ++wv) top = fmaxf(top, (*ml(wv, in))[0]);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int wv = 0; wv < kWaves; ++wv) {
                lo += chunk(wv, 0), hi += chunk(wv, 1);
                sum += (*ml(wv, in))[1] * __builtin_amdgcn_exp2f((*ml(wv, in))[0] - base);
            }
        }
        if (whole) {
            const int64_t token = rows.token(to), head = rows.head(to);
            const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
            *reinterpret_cast<uint4*>(a.out + token * a.out_stride + head * D + piece * 8) =
                make_uint4(T::pack(lo[0] * f, lo[1] * f), T::pack(lo[2] * f, lo[3] * f), T::pack(hi[0] * f, hi[1] * f), T::pack(hi[2] * f, hi[3] * f));
            if (a.lse && piece == 0) a.lse[token * a.n_q_heads + head] = sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2;
        } else {
            const int64_t at = part * kOutRows + r;
            *reinterpret_cast<f32x4*>(a.part_o + at * D + piece * 4) = lo;
            *reinterpret_cast<f32x4*>(a.part_o + at * D + D / 2 + piece * 4) = hi;
            if (piece == 0) a.part_ml[at] = make_float2(top, sum);
        }
    }
}

// The sequence that comes at a place in the order of falling lengths (64 sequences at most; equal ones in their own order).
__device__ __forceinline__ int by_length(const Attend8Args& a, int place, int lane)
{
    const int len = lane < a.n_seqs && a.max_len ? within(a.lens[lane], 0, a.max_len) : -1;
    int longer = 0;
    for (int e = 0; e < a.n_seqs; ++e) {
        const int y = __builtin_amdgcn_readlane(len, e);
        longer += y > len || (y == len && e < lane);
    }
    return __ffsll((unsigned long long)__ballot(lane < a.n_seqs && longer == place)) - 1;
}

// Workgroups are dealt round-robin over the XCDs.  Those that read the same keys (the row tiles of a group: one sequence, one key head, one
// run of keys) follow one another on one XCD, through its L2; groups go round the XCDs, the first parts of all sequences before the second
// ones, so that every XCD has the same mixture of sequences and of parts that short ones do not have.
template <typename T, int D, Kind kKind>
__global__ __launch_bounds__(kThreads, kKind == kWideRows ? 2 : 4) void k_attend8(Attend8Args a)
{
    constexpr int kRows = rows_of(kKind), kTile = keys_of(kKind);
    __shared__ __align__(1024) char lds[Lds8<kKind, D>::kTiles + Lds8<kKind, D>::kTable];
    const int unit = a.first_unit + blockIdx.x / kXcds, xcd = blockIdx.x % kXcds;
    const int tile = a.row_tiles - 1 - unit % a.row_tiles;             // (the last rows, which see the most keys, first)
    const int group = unit / a.row_tiles * kXcds + xcd;
    if (group >= a.groups) return;
    const int whole = a.n_seqs * a.c.n_kv_heads, split = group / whole, of = group % whole, kv = of % a.c.n_kv_heads;
    int b = of / a.c.n_kv_heads;
    // Many rows: the longest sequences first, so that what runs last is short.
    if (kKind == kWideRows && a.n_seqs > 1 && a.n_seqs <= 64) b = by_length(a, b, threadIdx.x & 63);
    const Sequence s(a, b);
    const int n_rows = s.tokens * a.group, row0 = tile * kRows;
    if (row0 >= n_rows) return;
    const Keys<kTile> keys(a, s.n0, row0 / a.group, (min(n_rows, row0 + kRows) - 1) / a.group);
    const int u0 = (int)min((int64_t)split * a.split_len, (int64_t)keys.tiles), u1 = (int)min((int64_t)u0 + a.split_len, (int64_t)keys.tiles);
    if (u0 >= u1 && split) return;                                     // (the first part is always there)
    const Rows rows{a, kv, s.token0, s.n0};
    attend<T, D, kKind>(a, rows, n_rows, row0, keys, u0, u1, a.pages + b * a.pages_stride, a.splits == 1, (((int64_t)b * a.c.n_kv_heads + kv) * a.splits + split) * a.row_tiles + tile, lds);
}

// How the tiles of a key head's items (a sequence, 16 of its rows) are dealt out among workers: all items one behind the other, `length` tiles each.
// Where no item has more than twice that, by whole items: nothing has to be joined then.  It is so where a call has room for long sequences (max_len) and
// they are short: with 16 sequences of up to 65536 tokens, all of which have up to 450, 25 -> 18 us, equal ones of 450 21 -> 18, of 512 17.4 -> 18.4.
// Eight tiles at least, two a wavefront: 4 cost such sequences of up to 200 and 400 tokens 24 and 20 us instead of 15 and 18, 16 those of up to 1000 27
// instead of 22; long ones do not care.  An item's weight is its tiles, 1 if it has rows that see nothing.  Every wavefront finds this out for itself,
// 64 items at a time.
struct Share {
    int32_t length, before, weight;        // tiles of a worker; tiles before an item, and its own
    int32_t item;
    bool by_items;
    static __device__ __forceinline__ int weigh(const Attend8Args& a, int item)
    {
        const Sequence s(a, item / a.row_tiles);
        const int n_rows = s.tokens * a.group, row0 = item % a.row_tiles * rows_of(kFewRows);
        if (row0 >= n_rows) return 0;
        return max(1, Keys<keys_of(kFewRows)>(a, s.n0, row0 / a.group, (min(n_rows, row0 + rows_of(kFewRows)) - 1) / a.group).tiles);
    }
    // of an item, or (item < 0) of the one in which worker ~item begins
    __device__ __forceinline__ Share(const Attend8Args& a, int lane, int of)
    {
        const int items = a.n_seqs * a.row_tiles;
        int all = 0, most = 0;
        for (int i0 = 0; i0 < items; i0 += 64) {
            const int w = i0 + lane < items ? weigh(a, i0 + lane) : 0;
            int sum = w, top = w;
#pragma unroll
            for (int e = 1; e < 64; e *= 2) sum += __shfl_xor(sum, e), top = max(top, __shfl_xor(top, e));
            all += sum;
            most = max(most, top);
        }
        length = max((all + a.workers - 1) / a.workers, 8);
        by_items = (int64_t)most * ((items + a.workers - 1) / a.workers) <= (int64_t)length * 2;
        item = items, before = all, weight = 0;
        const int64_t from = of < 0 ? (int64_t)~of * length : 0;
        int at = 0;
        for (int i0 = 0; i0 < items; i0 += 64) {
            const int w = i0 + lane < items ? weigh(a, i0 + lane) : 0;
            int sum = w;
#pragma unroll
            for (int e = 1; e < 64; e *= 2) {
                const int y = __shfl_up(sum, e);
                if (lane >= e) sum += y;
            }
            const uint64_t found = __ballot(of < 0 ? at + sum > from : i0 + lane == of);
            if (found) {
                const int l = __ffsll((unsigned long long)found) - 1;
                weight = __shfl(w, l);
                before = at + __shfl(sum, l) - weight;
                item = i0 + l;
                return;
            }
            at += __shfl(sum, 63);
        }
    }
};

// A worker goes through its tiles, item by item: results of whole items go where they belong, of others they are parts, at most two a worker.
template <typename T, int D> __global__ __launch_bounds__(kThreads, 4) void k_attend8_dealt(Attend8Args a)
{
    constexpr int kRows = rows_of(kFewRows);
    __shared__ __align__(1024) char lds[Lds8<kFewRows, D>::kTiles + Lds8<kFewRows, D>::kTable];
    const int kv = blockIdx.x % a.c.n_kv_heads, worker = blockIdx.x / a.c.n_kv_heads, items = a.n_seqs * a.row_tiles;
    const Share share(a, threadIdx.x & 63, ~worker);
    const bool by_items = __builtin_amdgcn_readfirstlane(share.by_items);
    int item = __builtin_amdgcn_readfirstlane(by_items ? worker : share.item);
    int u0 = __builtin_amdgcn_readfirstlane(by_items ? 0 : worker * share.length - share.before);
    int left = __builtin_amdgcn_readfirstlane(by_items ? 0x7fffffff : share.length);
    for (bool first = true; item < items && left > 0; first = false) {
        const int tile = item % a.row_tiles, b = item / a.row_tiles;
        const Sequence s(a, b);
        const int n_rows = s.tokens * a.group, row0 = tile * kRows;
        if (row0 < n_rows) {
            const Keys<keys_of(kFewRows)> keys(a, s.n0, row0 / a.group, (min(n_rows, row0 + kRows) - 1) / a.group);
            const int u1 = min(keys.tiles, u0 + min(left, keys.tiles));
            if (!first) __syncthreads();                   // (the results before are out of LDS)
            attend<T, D, kFewRows>(a, Rows{a, kv, s.token0, s.n0}, n_rows, row0, keys, u0, u1, a.pages + b * a.pages_stride, u0 == 0 && u1 == keys.tiles,
                                   ((int64_t)kv * a.workers + worker) * 2 + !first, lds);
            if (!by_items) left -= max(u1 - u0, 1);
        }
        item += by_items ? a.workers : 1;
        u0 = 0;
    }
}

// Joins the parts of a row: twice four elements a thread, kLanes threads for every eight, each with every kLanes-th part, eight of them in one
// go.  Bound by latency: the launch, the sequence's length, then all parts.
template <typename T, int D, Kind kKind, int kLanes>
__global__ __launch_bounds__(kThreads) void k_attend8_join(Attend8Args a, int64_t first)
{
    constexpr int kRows = rows_of(kKind), kPieces = D / 8, kRowsHere = kThreads / kPieces / kLanes, kBlocks = (kRows + kRowsHere - 1) / kRowsHere;
    const int64_t id = first + blockIdx.x;
    const int tile = (int)(id / kBlocks % a.row_tiles), of = (int)(id / kBlocks / a.row_tiles), kv = of % a.c.n_kv_heads, b = of / a.c.n_kv_heads;
    const int r = (int)(id % kBlocks) * kRowsHere + threadIdx.x / kPieces / kLanes, mine = threadIdx.x / kPieces % kLanes, piece = threadIdx.x % kPieces;
    const Sequence s(a, b);
    const int n_rows = s.tokens * a.group, row0 = tile * kRows;
    bool there = r < kRows && row0 + r < n_rows;
    const Keys<keys_of(kKind)> keys(a, s.n0, row0 / a.group, max(0, min(n_rows, row0 + kRows) - 1) / a.group);
    int parts = there ? max(1, (keys.tiles + a.split_len - 1) / a.split_len) : 0;
    constexpr int kAtOnce = 8;
    int64_t step = (int64_t)a.row_tiles * kRows, at0 = ((int64_t)of * a.splits * a.row_tiles + tile) * kRows + r, at_first = 0;
    if constexpr (kKind == kFewRows) {
        if (a.workers) {
            const Share share(a, threadIdx.x & 63, b * a.row_tiles + tile);
            const int w0 = share.before / share.length, w1 = (share.before + max(share.weight, 1) - 1) / share.length;
            if (share.by_items || w0 == w1) there = false;     // (nothing to join)
            parts = there ? w1 - w0 + 1 : 0;
            step = 2 * kRows;
            at0 = ((int64_t)kv * a.workers + w0) * 2 * kRows + r;
            at_first = share.before % share.length ? kRows : 0;        // the first part's, if it is not the first of its worker
        }
    }
    float top = -INFINITY, base, sum = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    for (int y0 = mine; y0 < parts; y0 += kAtOnce * kLanes) {
        float2 ml[kAtOnce];
        float4 lo[kAtOnce], hi[kAtOnce];
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
            const int y = min(y0 + x * kLanes, parts - 1);
            const int64_t at = at0 + y * step + (y ? 0 : at_first);
            const float4* p = reinterpret_cast<const float4*>(a.part_o + at * D) + piece;
            ml[x] = a.part_ml[at];
            lo[x] = p[0];
            hi[x] = p[kPieces];
        }
        const float before = top;
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x)
            if (y0 + x * kLanes < parts) top = fmaxf(top, ml[x].x);
        base = top == -INFINITY ? 0.0f : top;
        const float g = __builtin_amdgcn_exp2f(before - base);
        sum *= g;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= g;
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
            if (y0 + x * kLanes >= parts) continue;
            const float f = __builtin_amdgcn_exp2f(ml[x].x - base);
            sum = fmaf(ml[x].y, f, sum);
            o[0] = fmaf(lo[x].x, f, o[0]), o[1] = fmaf(lo[x].y, f, o[1]), o[2] = fmaf(lo[x].z, f, o[2]), o[3] = fmaf(lo[x].w, f, o[3]);
            o[4] = fmaf(hi[x].x, f, o[4]), o[5] = fmaf(hi[x].y, f, o[5]), o[6] = fmaf(hi[x].z, f, o[6]), o[7] = fmaf(hi[x].w, f, o[7]);
        }
    }
    if constexpr (kLanes > 1) {
        __shared__ float all[10][kThreads];
#pragma unroll
        for (int e = 0; e < 8; ++e) all[e][threadIdx.x] = o[e];
        all[8][threadIdx.x] = sum;
        all[9][threadIdx.x] = top;
        __syncthreads();
        if (mine) return;
        for (int y = 1; y < kLanes; ++y) top = fmaxf(top, all[9][threadIdx.x + y * kPieces]);
        base = top == -INFINITY ? 0.0f : top;
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
        for (int y = 0; y < kLanes; ++y) {
            const int x = threadIdx.x + y * kPieces;
            const float f = __builtin_amdgcn_exp2f(all[9][x] - base);
            sum = fmaf(all[8][x], f, sum);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(all[e][x], f, o[e]);
        }
    }
    if (!there) return;
    const int64_t token = s.token0 + (row0 + r) / a.group, head = kv * a.group + (row0 + r) % a.group;
    const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t* out = a.out + token * a.out_stride + head * D + piece * 4;
    *reinterpret_cast<uint2*>(out) = make_uint2(T::pack(o[0] * f, o[1] * f), T::pack(o[2] * f, o[3] * f));
    *reinterpret_cast<uint2*>(out + D / 2) = make_uint2(T::pack(o[4] * f, o[5] * f), T::pack(o[6] * f, o[7] * f));
    if (a.lse && piece == 0) a.lse[token * a.n_q_heads + head] = sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

bool sizes_ok(const fr_attend_kv8_desc& d)
{
    if (!kv8_pages_shape_ok(d.cache) || d.n_tokens < 0 || d.n_seqs < 0 || d.max_q < 1) return false;
    if (d.n_q_heads < 1 || d.n_q_heads > 1024 || d.n_q_heads % d.cache.n_kv_heads) return false;
    if ((int64_t)d.n_tokens * d.n_q_heads > 0x7fffffff - 4096) return false;
    return d.max_len >= 0 && d.max_len <= 0x7fffffff - 8191 && d.window >= 0 && d.sinks >= 0;
}

int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

// How a call is cut.
struct Plan {
    Kind kind = kFewRows;
    int64_t row_tiles = 1, base = 0, splits = 1, split_len = 1;        // base: sequences x key heads x row tiles
    int64_t workers = 0;                   // of a key head; 0: every item has the same number of parts
};
// Rows of a sequence and key head that are few: up to three items of 16, each of which goes through the keys, against 128 rows of which some are none.
// us by items of 16 and by 128 rows, head_dim 128, sequences x key heads:
//                                  24 rows        32        40        48        64        96
//   64 x 8, up to 4000 keys       92   114   99   116  111  111  119  121  131  121  179  135
//   8 x 8, up to 4000             26    46   26    45   30   50   32   50   35   46   43   53
//   33 x 5, window 1000           24    48   24    49   26   51   26   50   28   54   33   55
//   128 x 8, up to 500            31    51   30    49   43   56   42   55   49   55   66   58
//   1 x 8, 40000                  35    50   36    51   46   55   48   56   54   58   64   63
//   8 x 8, up to 40000           135   155  151   158  177  173  176  167  235  171  341  189
constexpr int64_t kMostFew = 48;
constexpr int64_t kMostDealt = 512;        // items of a key head that are dealt out evenly: each worker looks at all of them
// Parts of a row, at most: what the join's threads read in one go (32, 64, 128 and 256: two sequences of 30000 keys with one key head 22, 16, 13.3, 13.3 us, one of
// 60000 33, 22, 16, 14.5, one of 60000 with 8 key heads 35, 29, 30, 32).
constexpr int64_t kMostParts = 128;
constexpr int64_t kMostBlocks = 0x7fffffff;

// Parts are no more than give so many items in all: four a unit, which are on it at once.  Of few rows three times as many, where there are few sequences
// and heads: they even out lengths that differ (8 sequences of up to 65536 tokens with 8 key heads 125 -> 114 us; with more sequences than that there is
// no gain, and of equal lengths they begin and end more often: 128 windows of 4096 tokens 185 us in one part, 197 in two).
int64_t most_items(Kind k, int64_t base, int64_t cus) { return (k == kFewRows && 2 * base <= cus ? 12 : 4) * cus; }

int64_t rows_a_seq(const fr_attend_kv8_desc& d) { return (int64_t)std::min(d.max_q, d.n_tokens) * (d.n_q_heads / d.cache.n_kv_heads); }
int64_t row_tiles_of(int64_t rows) { return rows > kMostFew ? up(rows, rows_of(kWideRows)) : up(rows, rows_of(kFewRows)); }

Plan plan(const fr_attend_kv8_desc& d, int cus)
{
    Plan p;
    cus = std::min(cus, kUnits);
    const int64_t rows = rows_a_seq(d), group = d.n_q_heads / d.cache.n_kv_heads;
    p.kind = rows > kMostFew ? kWideRows : kFewRows;
    p.row_tiles = row_tiles_of(rows);
    p.base = (int64_t)d.n_seqs * d.cache.n_kv_heads * p.row_tiles;
    const int64_t tile = keys_of(p.kind);
    // tiles of keys that a row tile sees, at most
    int64_t keys = d.max_len;
    if (d.window) keys = std::min<int64_t>(keys, (int64_t)d.window + std::min<int64_t>(up(rows_of(p.kind), group), d.max_q) + d.sinks + 3 * tile);
    // A part has two tiles a wavefront at least where rows are few, and two tiles of 128 rows.  Few rows, 4 and 8 tiles, 32 heads, 8 key heads of 128: 8 sequences of
    // 4000 keys 24.9, 20.6 us, 16 of 2000 23.3, 20.4, 3 of up to 9000 19.5, 17.8, 4 of 3000 15.0, 15.2, one of 1000 10.1, 11.7 (16 tiles 14.0), two of 700 9.8, 12.1.
    // Many, 1, 2, 4 and 8 tiles: 300 tokens behind as many 47, 34, 30, 30, 300 alone 29, 24, 25, 20, 2 x 64 behind 2000 50, 35, 34, 32, 20 behind 1000 with 16 heads of
    // 64 16.2, 16.5, 18, 22.
    const int64_t tiles = std::max<int64_t>(up(keys, tile), 1), least = p.kind == kWideRows ? 2 : 8;
    const int64_t want = std::max<int64_t>(1, std::min({up(tiles, least), most_items(p.kind, p.base, cus) / p.base, kMostParts}));
    p.split_len = up(tiles, want);
    p.splits = up(tiles, p.split_len);
    // Some long sequences: tiles dealt out evenly.  Against parts of one length, 8 key heads, lengths up to these: 4 sequences of 65536 88 -> 78 us, 8
    // 164 -> 151, 16 of 32768 134 -> 126, of equal lengths 206 -> 204; with more items the units even themselves out better (32 of 8000 equal ones
    // 103, dealt out 114), with fewer there are enough parts (2 of 65536 57 and 60).
    if (p.kind == kFewRows && d.n_seqs > 1 && d.n_seqs * p.row_tiles <= kMostDealt && 8 * p.base >= cus && 2 * p.base <= cus && p.base * tiles >= 128 * (int64_t)cus &&
        d.n_seqs * p.row_tiles * tiles < 1 << 30)
        p.workers = 4 * cus / d.cache.n_kv_heads;
    return p;
}

// Rows of results in parts that a call has room for; no call with smaller sizes, of whatever window, has more.
int64_t most_part_rows(const fr_attend_kv8_desc& d)
{
    const int64_t rows = rows_a_seq(d), kind_rows = rows > kMostFew ? rows_of(kWideRows) : rows_of(kFewRows), most = most_items(rows > kMostFew ? kWideRows : kFewRows, 1, kUnits);
    const int64_t base = (int64_t)d.n_seqs * d.cache.n_kv_heads * row_tiles_of(rows), parts = up(d.max_len, 128);
    return parts < 2 ? 0 : std::min(base * parts, most) * kind_rows;
}
uint64_t part_bytes(const fr_attend_kv8_desc& d) { return (uint64_t)most_part_rows(d) * (d.cache.head_dim * 4 + 8); }

template <typename T, int D, Kind kKind> int launch(Attend8Args a, const Plan& p, hipStream_t stream)
{
    constexpr int kBlocksALaunch = kMostThreads / kThreads;
    a.groups = (int)((int64_t)a.n_seqs * a.c.n_kv_heads * p.splits);
    a.units = (int)(up(a.groups, kXcds) * a.row_tiles);
    if (p.workers) {
        if constexpr (kKind == kFewRows)
            hipLaunchKernelGGL((k_attend8_dealt<T, D>), dim3((unsigned)(p.workers * a.c.n_kv_heads)), dim3(kThreads), 0, stream, a);
    } else for (a.first_unit = 0; a.first_unit < a.units; a.first_unit += kBlocksALaunch / kXcds)
        hipLaunchKernelGGL((k_attend8<T, D, kKind>), dim3((unsigned)std::min(a.units - a.first_unit, kBlocksALaunch / kXcds) * kXcds), dim3(kThreads), 0, stream, a);
    auto join = [&](auto lanes) {
        constexpr int kRowsHere = kThreads / (D / 8) / lanes, kBlocks = (rows_of(kKind) + kRowsHere - 1) / kRowsHere;
        const int64_t all = p.base * kBlocks;
        for (int64_t first = 0; first < all; first += kBlocksALaunch)
            hipLaunchKernelGGL((k_attend8_join<T, D, kKind, lanes>), dim3((unsigned)std::min<int64_t>(all - first, kBlocksALaunch)), dim3(kThreads), 0, stream, a, first);
    };
    // Threads of the join for every eight elements, 1, 4 and 16: one sequence of 60000 keys, 128 parts, 45, 33, 30 us, two of 8000, 32 parts, 18.1, 15.5, 15.9, 4 of
    // 3000, 12 parts, 14.2, 14.7, 15.5, 64 of up to 4000, 2 parts, 73, 79, 90; dealt out, 8 of up to 65536, 131, 128, 130.
    if (p.workers || (p.splits > 8 && p.splits <= 32)) join(std::integral_constant<int, 4>{});
    else if (p.splits > 32) join(std::integral_constant<int, 16>{});
    else if (p.splits > 1) join(std::integral_constant<int, 1>{});
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}

template <typename T, int D> int launch(const Attend8Args& a, const Plan& p, hipStream_t stream)
{
    return p.kind == kWideRows ? launch<T, D, kWideRows>(a, p, stream) : launch<T, D, kFewRows>(a, p, stream);
}

}  // namespace

extern "C" {

int fr_attend_kv8_workspace_bytes(const fr_attend_kv8_desc* d, uint64_t* bytes_out)
{
    if (!d || !bytes_out || !sizes_ok(*d)) return FR_ERR_ARG;
    *bytes_out = 0;
    if (d->n_tokens == 0 || d->n_seqs == 0) return FR_OK;
    if (plan(*d, kUnits).base > kMostBlocks / 16) return FR_ERR_ARG;
    *bytes_out = part_bytes(*d);
    return FR_OK;
}

int fr_attend_kv8(const fr_attend_kv8_desc* d, void* stream)
{
    if (!d || !sizes_ok(*d) || !kv8_pages_ok(d->cache)) return FR_ERR_ARG;
    if (!(d->scale > 0.0f && d->scale <= 0x1p120f)) return FR_ERR_ARG;
    if (d->n_tokens == 0 || d->n_seqs == 0) return FR_OK;
    const fr_kv8_pages& c = d->cache;
    const int64_t width = (int64_t)d->n_q_heads * c.head_dim, most = (int64_t)1 << 45;
    if (!d->q || !d->out || d->q == d->out || (((uintptr_t)d->q | (uintptr_t)d->out) & 15)) return FR_ERR_ARG;
    for (int64_t s : {d->q_stride, d->out_stride})
        if (s % 8 || s > most || s < 0 || (d->n_tokens > 1 && s < width)) return FR_ERR_ARG;
    if (!d->q_begin && d->n_tokens != d->n_seqs) return FR_ERR_ARG;
    if (d->max_len && (!d->pages || !d->lens || d->pages_stride < ((int64_t)d->max_len + c.page_size - 1) / c.page_size || d->pages_stride > most)) return FR_ERR_ARG;
    fr_attend_kv8_desc sizes = *d;
    if (!d->q_begin) sizes.max_q = 1;                              // (a token each, whatever a program's other calls have)
    const Plan p = plan(sizes, (int)fr_stream_cus((hipStream_t)stream));
    if (p.base > kMostBlocks / 16) return FR_ERR_ARG;
    const uint64_t need = part_bytes(sizes);
    if (need && (!d->workspace || ((uintptr_t)d->workspace & 255) || d->workspace_bytes < need)) return FR_ERR_ARG;
    const int64_t part_rows = p.workers ? p.workers * c.n_kv_heads * 2 * rows_of(p.kind) : p.splits > 1 ? p.base * p.splits * rows_of(p.kind) : 0;
    if (part_rows > most_part_rows(sizes)) return FR_ERR_ARG;        // (the plan keeps to it)
    Attend8Args a = {c, (const uint16_t*)d->q, (uint16_t*)d->out, d->lse, d->q_stride, d->out_stride, d->pages_stride, d->q_begin, d->pages, d->lens,
                     d->n_tokens, d->n_seqs, d->n_q_heads, sizes.max_q, d->max_len, d->window, d->sinks,
                     __builtin_ctz(c.page_size), __builtin_ctz(c.block), d->n_q_heads / c.n_kv_heads};
    // With queries and keys as far apart as bfloat16 lets them be, a product of 32 bits would be beyond its range before a scale below 1 brings it back.
    // Not more of it than 2^-64 goes into the queries: those down to 2^-62 lose nothing then, and sums up to 2^192 are in range.  A scale above 1 makes
    // scores larger than the products, which need no help; into the queries it could take them beyond the type's range.
    int e = 0;
    if (c.dtype == FR_DTYPE_BF16) {
        std::frexp(d->scale, &e);
        e = std::max(-64, std::min(0, e));
    }
    a.q_power = std::ldexp(1.0f, e);
    a.rate = std::ldexp(d->scale, -e) * kLog2e;
    a.row_tiles = (int)p.row_tiles;
    a.splits = (int)p.splits;
    a.split_len = (int)std::min<int64_t>(p.split_len, 0x7fffffff);
    a.part_o = (float*)d->workspace;
    a.part_ml = (float2*)((char*)d->workspace + (uint64_t)part_rows * c.head_dim * 4);
    a.workers = (int)p.workers;
    hipStream_t s = (hipStream_t)stream;
    if (c.dtype == FR_DTYPE_BF16) return c.head_dim == 64 ? launch<Bf16, 64>(a, p, s) : launch<Bf16, 128>(a, p, s);
    return c.head_dim == 64 ? launch<F16, 64>(a, p, s) : launch<F16, 128>(a, p, s);
}

}  // extern "C"
