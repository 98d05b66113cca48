// Attention of a batch of sequences behind a shared prefix, keys and values in a cache of pages.
//
// A query row q (a token, a head) that sees keys k_j with values v_j gets  out = sum_j w_j v_j / sum_j w_j,  w_j = exp(s_j - m),
// s_j = scale q . k_j,  and lse = m + log sum_j w_j, for whatever m: the largest score seen so far.  Where m rises, the sums so far
// are multiplied by exp(m_before - m), so that one pass over the keys is enough, and parts of the keys, each with its own m, are
// joined in the same way.  Scores, m, both sums and the parts' results are of 32 bits; weights are rounded to the type for the
// product with the values, and the result is, once.
//
// The heads that share a key head, and all tokens of a sequence, are rows of one matrix product with its keys; against the prefix
// the rows of all sequences are, so the prefix is read once for 128 of them.
// What bounds it:
//   Decoding from long caches, the reading: 8 sequences of 20000 to 65536 tokens, 1.62 GB in 285 us, 5.7 TB/s (a kernel that only
//     reads reaches 6.5).
//   Prompts, the matrix cores: 16 questions of 300 to 700 tokens about 8192, 32 heads, 1.03 TFLOP in 1.04 to 1.08 ms, 0.95 to 0.99
//     PFLOP/s (a library product of 8192 x 8192 matrices 1.25), 4 prompts of 4096 by themselves 0.55 in 0.62 ms; beside them the vector
//     units make 2 exps and 5 other operations of every two weights.
//   Decoding behind a prefix, neither: 64 sequences behind 16384 keys take 63 us in a kernel trace, the prefix' workgroups by
//     themselves 33 and the own keys' 36: the two kinds slow one another down; then the parts are joined, 7 us.
//   A few short sequences, the launch: 5 us.

#include <algorithm>
#include <cmath>

#include "attend_tiles.h"
#include "common.h"

namespace {

struct Segment {                           // the work of one of the two kinds of workgroups
    int32_t row_tiles, splits, split_len, first_part, items, groups, units;      // (a group: what follows one another on an XCD, its row tiles)
};

typedef std::integral_constant<uint32_t, 0> Even;
typedef std::integral_constant<uint32_t, 1> Odd;

// What a workgroup's four wavefronts do.  kWideRows: 128 rows, 32 a wavefront, which share tiles of 64 keys.  kFewRows: 16 rows, and
// every wavefront takes every fourth tile of 32 keys for itself, the four results being joined at the end.  kWaveRows: every
// wavefront has an item of its own, 16 rows and all of its keys in tiles of 32, and meets no barrier.
enum Kind { kNone, kFewRows, kWaveRows, kWideRows };
constexpr int columns(Kind k) { return k == kWideRows ? 32 : 16; }                     // rows of a wavefront: columns of its MFMA blocks
constexpr int rows_of(Kind k) { return k == kWideRows ? kWaves * 32 : 16; }            // rows of a workgroup (kWaveRows: of a wavefront)

struct AttendArgs {
    fr_kv_pages c;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_stride, out_stride, pages_stride;
    const int32_t *q_begin, *prefix_pages, *pages, *own_len;
    int32_t n_tokens, n_seqs, n_q_heads, max_q, prefix_len, max_own_len, page_shift, group;
    float scale;
    int32_t own_from;                      // the sequences' workgroups take keys from here on: 0, or prefix_len
    int32_t first_unit;                    // of this launch
    Segment prefix, own;
    int32_t parts;                         // 1: results go to `out`, else to part_*
    float* part_o;                         // [parts][n_tokens * n_q_heads][head_dim], relative to 2^m
    float2* part_ml;                       // [parts][n_tokens * n_q_heads]: m in powers of 2, sum
};

template <int kLeft> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(kLeft) : "memory"); }
// Global memory to LDS without passing through registers, 16 bytes (or 4) a lane: lane l's go to LDS address lds + 16 l (4 l).
// Written as assembly so that the compiler does not wait for every load in flight before each read of LDS; which loads have to be
// here is counted by hand.  (m0 is reserved and cannot be named as overwritten; no instruction of these kernels but the two uses it.)
__device__ __forceinline__ void load16_to_lds(uint32_t lds, const void* g)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(g) : "memory");
}
__device__ __forceinline__ void load4_to_lds(uint32_t lds, const void* g)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(g) : "memory");
}

// Whether a token is one of the first max_q of a sequence.
__device__ __forceinline__ bool is_computed(const AttendArgs& a, int token)
{
    int b = 0, end = a.n_seqs;
    while (end - b > 1) {
        const int middle = b + (end - b) / 2;
        if (within(a.q_begin[middle], 0, a.n_tokens) <= token) b = middle;
        else end = middle;
    }
    const int t0 = within(a.q_begin[b], 0, a.n_tokens), t1 = within(a.q_begin[b + 1], t0, a.n_tokens);
    return token >= t0 && token < t1 && token - t0 < a.max_q;
}

// What a workgroup works on: query rows (token and head of a group, the group's heads side by side) against a run of keys.
struct Item {
    int32_t kv, token0, rows, row0;        // key head; first token; rows there are; first row of this workgroup
    int32_t k0, k1;                        // keys, counted through the prefix and then the sequence's own
    int32_t seen0, seen_step;              // a row of token i sees the keys below max(prefix, seen0 + i * seen_step)
    int32_t part;
    const int32_t* own_pages;
    bool of_all;                           // rows of all tokens, also of those that are in no sequence
};

// Where a row's result goes.
template <int D> struct Rows {
    const AttendArgs& a;
    const Item& w;
    __device__ __forceinline__ int32_t token(int r) const { return w.token0 + r / a.group; }
    __device__ __forceinline__ int32_t head(int r) const { return w.kv * a.group + r % a.group; }
    __device__ __forceinline__ int32_t seen(int r) const { return max(a.prefix_len, w.seen0 + r / a.group * w.seen_step); }
};

// The work of one workgroup (kWaveRows: of one wavefront).
//
// kWideRows: a wavefront's 32 rows are the columns of 32 x 32 x 16 blocks; scores and results stand in its registers, transposed, and
// weights go from the one product to the next without passing through LDS.  Tiles of 64 keys come to LDS, two of K and two of V.
// A tile is 32 MFMAs a wavefront (head_dim 128), 0.5 us, and takes 1.43 us where the workgroup is alone on its unit, 2.0 where there
// are two: there is a barrier to wait for, 64 fragments are read, and the weights' vector operations take as long as the MFMAs beside
// which they are issued.  Measured at the 16 questions above, 1.013 ms in a graph: fragments read 6 MFMAs ahead instead of 4 1.021;
// 8 or 12 pairs of weights beside the scores' MFMAs instead of 10 1.009 and 1.028; loads asked for between the MFMAs instead of before
// them 1.11; the MFMAs with the values at the usual priority 5 % more.
//
// kFewRows and kWaveRows: 16 rows, blocks of 16 x 16 x 32, tiles of 32 keys that pass through LDS (where the values are transposed)
// into registers while the next ones are on their way: with so few rows the MFMAs are next to nothing, and what counts is the number
// of bytes asked for ahead, 16 KB a wavefront and 128 KB a unit at head_dim 128.
template <typename T, int D, Kind kKind>
__device__ __forceinline__ void attend(const AttendArgs& a, const Item& w, char* lds_array, int32_t* ids_array)
{
    constexpr bool kWide = kKind == kWideRows, kAlone = kKind == kWaveRows;
    constexpr int kCols = columns(kKind);
    constexpr int kSharers = kAlone ? 1 : kWaves;           // wavefronts that deal tiles of 32 keys out among themselves
    typedef Lds<D, kCols> L;
    typedef Softmax<T, D, kCols> State;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds = (uint32_t)reinterpret_cast<uintptr_t>((LdsBytes)lds_array), ids = (uint32_t)reinterpret_cast<uintptr_t>((LdsBytes)(char*)ids_array);
    asm volatile("" ::"s"(lds), "s"(ids) : "memory");       // (both arrays are written behind the compiler's back)
    const Rows<D> rows{a, w};
    const float c = a.scale * kLog2e;

    // the wavefront's rows
    const int row_first = w.row0 + (kWide ? wave * kCols : 0), row = row_first + lane % kCols;
    const bool idle = row_first >= w.rows;
    const int row_here = min(row, w.rows - 1);
    const int end = min(rows.seen(row_here), w.k1);
    State x;
    x.start();
    {
        const uint16_t* q = a.q + rows.token(row_here) * a.q_stride + (int64_t)rows.head(row_here) * D + lane / kCols * 8;
#pragma unroll
        for (int f = 0; f < D * kCols / 512; ++f) x.q[f] = __builtin_bit_cast(typename T::x8, *reinterpret_cast<const uint4*>(q + f * (512 / kCols)));
    }

    // What a lane loads is made anew from `anew(lane)` for every tile: kept, it holds registers that the loop needs.
    auto anew = [](int x) { asm volatile("" : "+v"(x)); return (uint32_t)x; };

    // A wavefront loads kLoadRows rows of a tile.  Where 64 of them (a set: those of two or four tiles) lie is worked out at once, a
    // lane each: page ids come to LDS, offsets go back there.  Keys behind the last stand for the last.
    constexpr int kLoadRows = kWide ? 16 : 32, kTilesASet = 64 / kLoadRows, kLoads = kLoadRows / L::kRowsALoad;
    const uint32_t my_ids = ids + wave * 1536, my_offsets = my_ids + 512;
    auto key_of = [&](int set) {
        const int l = (int)anew(lane), tile = set * kTilesASet + l / kLoadRows;
        return min(w.k0 + (kWide ? tile * 64 + wave * 16 : (kAlone ? tile : tile * kWaves + wave) * 32) + l % kLoadRows, w.k1 - 1);
    };
    auto ask_ids = [&](int set) {
        const int j = key_of(set), own = j - a.prefix_len;
        load4_to_lds(my_ids + (set & 1) * 256, own < 0 ? a.prefix_pages + (j >> a.page_shift) : w.own_pages + (own >> a.page_shift));
    };
    typedef __attribute__((address_space(3))) uint64_t* LdsOffset;
    auto make_offsets = [&](int set) {
        const int j = key_of(set), in = j < a.prefix_len ? j : j - a.prefix_len;
        const int32_t id = *reinterpret_cast<const __attribute__((address_space(3))) int32_t*>(lds_at(my_ids + (set & 1) * 256 + anew(lane) * 4));
        const uint32_t page = (uint32_t)within(id, 0, (int32_t)a.c.n_pages - 1);
        *reinterpret_cast<LdsOffset>(lds_at(my_offsets + (set & 1) * 512 + anew(lane) * 8)) =
            (uint64_t)page * (uint32_t)a.c.page_stride + (uint64_t)(uint32_t)(in & (a.c.page_size - 1)) * (uint32_t)a.c.slot_stride;
    };
    // tile t's rows of K (V) to LDS
    auto ask = [&](int t, const uint16_t* from, uint32_t to, auto piece) {
        const uint32_t l = anew(lane), at = my_offsets + (t / kTilesASet & 1) * 512 + (t % kTilesASet) * (kLoadRows * 8) + l / L::kChunks * 8;
        uint64_t row[kLoads];
#pragma unroll
        for (int y = 0; y < kLoads; ++y) row[y] = *reinterpret_cast<LdsOffset>(lds_at(at) + y * (int)L::kRowsALoad * 8);
#pragma unroll
        for (int y = 0; y < kLoads; ++y) load16_to_lds(to + y * 1024, from + piece(l, y) * 8 + row[y]);
    };
    // Rows of V that came to LDS for a wavefront, from key `first` on: those behind the last key (which stand for it) become zeros.  Their
    // weights are 0, but 0 times a value that is not finite is not.
    typedef __attribute__((address_space(3))) f32x4* LdsFloats;
    auto blank = [&](uint32_t at, int first) {
        if (first + kLoadRows <= w.k1) return;
        const uint32_t l = anew(lane);
        const float zero = __uint_as_float(anew(0));
#pragma unroll
        for (int y = 0; y < kLoads; ++y)
            if (first + y * (int)L::kRowsALoad + (int)(l / L::kChunks) >= w.k1) *reinterpret_cast<LdsFloats>(lds_at(at + l * 16) + y * 1024) = f32x4{zero, zero, zero, zero};
        wait_lds();
    };
    auto k_piece = [](uint32_t l, int y) { return L::k_piece(l, y); };
    auto v_piece = [](uint32_t l, int y) { return L::v_piece(l, y); };
    const uint16_t* gk = static_cast<const uint16_t*>(a.c.k) + w.kv * a.c.head_stride;
    const uint16_t* gv = static_cast<const uint16_t*>(a.c.v) + w.kv * a.c.head_stride;
    if (w.k0 < w.k1) {
        if constexpr (kWide) {
            // While tile t's scores become weights (vector unit), the matrix cores make those of tile t + 1: K runs a tile ahead of V.
            constexpr int kTile = 64;
            constexpr uint32_t kHalf = kTile * L::kRow;
            const int tiles = (w.k1 - w.k0 + kTile - 1) / kTile;
            auto ask_k = [&](int t, auto odd) { ask(t, gk, lds + odd * kHalf + wave * 16 * L::kRow, k_piece); };
            auto ask_v = [&](int t, auto odd) { ask(t, gv, lds + (2 + odd) * kHalf + wave * 16 * L::kRow, v_piece); };
            constexpr int kSteps = D / 8;                   // MFMAs of the scores, and as many with the values
            constexpr int kAhead = 4;                       // fragments read ahead of their MFMA
            // 16 pairs of weights: as many beside the scores' MFMAs as they take time, the rest beside the first half of the values'
            constexpr int kPairsBeside = D == 128 ? 10 : 8;
            const Even even{};
            const Odd odd{};
            Fragments<T, D, kCols> fragments(lds, lane);
            typename T::x8 ahead[kAhead];
            auto k_of = [&](auto odd, int y) { return fragments.of_k(odd * kHalf + y % 2 * 32 * L::kRow, y / 2); };
            auto v_of = [&](auto odd, int y) { return fragments.of_v((2 + odd) * kHalf + y / (D / 32) * 16 * L::kRow, y % (D / 32)); };
            const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            float top = -INFINITY;
            auto step = [&](f32x16 (&now)[2], f32x16 (&next)[2], int t, auto here, auto other) {      // (here: t modulo 2)
                wait_loads<0>();
                if (t + 1 == tiles) blank(lds + (2 + here) * kHalf + wave * 16 * L::kRow, w.k0 + t * kTile + wave * 16);
                __syncthreads();                            // K of t + 1 and V of t are here; K of t and V of t - 1 are done with
                if (!idle) {
                    asm volatile("" : "+v"(fragments.k), "+v"(fragments.v));        // (one register each, not one for every fragment)
#pragma unroll
                    for (int y = 0; y < kAhead; ++y) ahead[y] = k_of(other, y);
                }
                if (t + 1 < tiles) ask_v(t + 1, other);
                if (t + 2 < tiles) ask_k(t + 2, here);
                // offsets of set s are there when step 4 s - 2 asks for K of tile 4 s
                if (t % kTilesASet == 0 && t + kTilesASet < tiles) ask_ids(t / kTilesASet + 1);
                if (t % kTilesASet == 1 && t + kTilesASet - 1 < tiles) make_offsets(t / kTilesASet + 1);
                if (idle) return;
                x.grow(top, c);
                const float base = x.base(c);
                uint32_t p[16];
                auto pair = [&](int e) {
                    p[e] = x.weigh(now[e / 8][2 * e % 16], now[e / 8][2 * e % 16 + 1], c, base);
                    asm volatile("" : "+v"(p[e]), "+v"(x.l), "+v"(x.l1));             // (made here, not where they are used)
                };
                keep_order();
#pragma unroll
                for (int y = 0; y < kSteps; ++y) {          // (behind the last tile: of what lies there, not used)
                    next[y % 2] = mfma(ahead[y % kAhead], x.q[y / 2], y < 2 ? zero : next[y % 2]);
                    ahead[y % kAhead] = y + kAhead < kSteps ? k_of(other, y + kAhead) : v_of(here, y + kAhead - kSteps);
#pragma unroll
                    for (int e = y * kPairsBeside / kSteps; e < (y + 1) * kPairsBeside / kSteps; ++e) pair(e);
                    keep_order();
                }
                State::hide(next, w.k0 + (t + 1) * kTile, end, lane);
                top = -INFINITY;
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
                        for (int e = (y - kFirst) * 32 / kFirst; e < (y - kFirst + 1) * 32 / kFirst; ++e) top = fmaxf(top, next[e / 16][e % 16]);
                    }
                    keep_order();
                }
                __builtin_amdgcn_s_setprio(0);
                top = top_of_row<kCols>(top);
            };
            ask_ids(0);
            wait_loads<0>();
            make_offsets(0);
            ask_k(0, even);
            wait_loads<0>();
            __syncthreads();
            ask_v(0, even);
            if (tiles > 1) ask_k(1, odd);
            f32x16 s0[2], s1[2];
            if (!idle) {
#pragma unroll
                for (int y = 0; y < kSteps; ++y) s0[y % 2] = mfma(k_of(even, y), x.q[y / 2], y < 2 ? zero : s0[y % 2]);
                State::hide(s0, w.k0, end, lane);
#pragma unroll
                for (int e = 0; e < 32; ++e) top = fmaxf(top, s0[e / 16][e % 16]);
                top = top_of_row<kCols>(top);
            }
            for (int t = 0; t < tiles; t += 2) {
                step(s0, s1, t, even, odd);
                if (t + 1 < tiles) step(s1, s0, t + 1, odd, even);
            }
        } else {
            constexpr int kTile = 32;
            constexpr uint32_t kHalf = kTile * L::kRow;
            const int all = (w.k1 - w.k0 + kTile - 1) / kTile, mine = kAlone ? 0 : wave, tiles = (all - mine + kSharers - 1) / kSharers;
            const uint32_t k = lds + wave * 2 * kHalf, v = k + kHalf;
            auto first_of = [&](int t) { return w.k0 + (t * kSharers + mine) * kTile; };
            const Fragments<T, D, kCols> fragments(k, lane);
            // LDS is where tiles pass through: K and V of a tile go on into registers as soon as they are here, and the next one's are
            // asked for, so that every load has a whole round to arrive.
            typename T::x8 kf[2][D / 32], vf[D / 16];
            auto take_k = [&] {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int f = 0; f < D / 32; ++f) kf[b][f] = fragments.of_k(b * 16 * L::kRow, f);
                wait_lds();
            };
            if (tiles > 0) {
                ask_ids(0);
                ask_ids(1);
                wait_loads<0>();
                make_offsets(0);
                ask(0, gk, k, k_piece);
                ask(0, gv, v, v_piece);
                wait_loads<kLoads>();
                take_k();
                if (tiles > 1) ask(1, gk, k, k_piece);
            }
            for (int t = 0; t < tiles; ++t) {
                // K of tile t is in registers; in flight are V of tile t, K of t + 1 and, for odd t, page ids, in this order
                const bool more = t + 1 < tiles;
                f32x4 s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int f = 0; f < D / 32; ++f)
#pragma unroll
                    for (int b = 0; b < 2; ++b) s[b] = mfma(kf[b][f], x.q[f], s[b]);
                if (more) {
                    wait_loads<kLoads>();
                } else {
                    wait_loads<0>();
                    blank(v, first_of(t));
                }
#pragma unroll
                for (int d = 0; d < D / 16; ++d) vf[d] = fragments.of_v(kHalf, d);
                wait_lds();
                if (more) ask(t + 1, gv, v, v_piece);
                State::hide(s, first_of(t), end, lane);
                float top = s[0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i / 4][i % 4]);
                x.grow(top_of_row<kCols>(top), c);
                const float base = x.base(c);
                uint32_t p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = x.weigh(s[e / 2][2 * e % 4], s[e / 2][2 * e % 4 + 1], c, base);
                if (more) {
                    wait_loads<kLoads>();
                    take_k();
                    if (t + 2 < tiles) {
                        if (t % 2 == 0) make_offsets(t / 2 + 1);
                        ask(t + 2, gk, k, k_piece);
                        if (t % 2 == 0) ask_ids(t / 2 + 2);
                    }
                }
#pragma unroll
                for (int d = 0; d < D / 16; ++d) x.o[d] = mfma(vf[d], State::fragment(p), x.o[d]);
            }
        }

        // A weight of 0 for a key that a row does not see, times a value that is not finite, is not 0.  Keys from `hidden` on are not
        // seen by every row of the workgroup: where a result is not finite and one of them has such a value, the sums are made again,
        // with zeros for these values, and what they are to the rows that see them is added.  Fragments come straight from memory, V an
        // element at a time, with a third of the pace: 4 questions of 300 tokens about 4096, 67 us, one NaN in a question 213; in the
        // document, where every row sees it and nothing is made again, 68.
        const int hidden = w.seen_step ? max(w.k0, min(rows.seen(w.row0), w.k1)) : w.k1;
        auto place_of = [&](int j) {                        // (of a key behind the last: that of the last)
            j = min(j, w.k1 - 1);
            const int in = j < a.prefix_len ? j : j - a.prefix_len;
            const int32_t id = within(j < a.prefix_len ? a.prefix_pages[in >> a.page_shift] : w.own_pages[in >> a.page_shift], 0, (int32_t)a.c.n_pages - 1);
            return (uint64_t)(uint32_t)id * (uint32_t)a.c.page_stride + (uint64_t)(uint32_t)(in & (a.c.page_size - 1)) * (uint32_t)a.c.slot_stride;
        };
        // keys of j .. j + 63 from `hidden` on with values that are not finite, a bit each
        auto spoilt = [&](int j) {
            j += (int)anew(lane);
            bool any = false;
            if (j < w.k1) {
                const uint16_t* y = gv + place_of(j);
#pragma unroll 1
                for (int e = 0; e < D; e += 8) {
                    const uint4 b = *reinterpret_cast<const uint4*>(y + e);
                    any |= !T::both_finite(b.x) || !T::both_finite(b.y) || !T::both_finite(b.z) || !T::both_finite(b.w);
                }
            }
            return __ballot(any);
        };
        bool bad = false;
        if (hidden < w.k1 && !idle) {
#pragma unroll
            for (int d = 0; d < D / kCols; ++d)
#pragma unroll
                for (int i = 0; i < State::kInBlock; ++i) bad |= !(fabsf(x.o[d][i]) < INFINITY);
        }
        if (__builtin_expect(__any(bad), 0)) {
            bad = false;
            for (int j = hidden; j < w.k1; j += 64) bad |= spoilt(j) != 0;
        }
        if (__builtin_expect(__any(bad), 0)) {
            const float base = x.base(c);
            x.clear();
            constexpr int kBlocks = 32 / kCols, kInRow = 512 / kCols;       // blocks of 32 keys; keys of a fragment of weights
#pragma unroll 1
            for (int j0 = w.k0; j0 < w.k1; j0 += 32) {
                if (kKind == kFewRows && (j0 - w.k0) / 32 % kWaves != wave) continue;
                typename State::Block s[kBlocks];
                uint32_t p[8];
#pragma unroll
                for (int y = 0; y < kBlocks; ++y) {
#pragma unroll
                    for (int i = 0; i < State::kInBlock; ++i) s[y][i] = 0.0f;
                    const uint16_t* k = gk + place_of(j0 + y * kCols + lane % kCols) + lane / kCols * 8;
#pragma unroll
                    for (int f = 0; f < D / kInRow; ++f) s[y] = mfma(__builtin_bit_cast(typename T::x8, *reinterpret_cast<const uint4*>(k + f * kInRow)), x.q[f], s[y]);
#pragma unroll
                    for (int i = 0; i < State::kInBlock; i += 2) {
                        float wt[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) wt[e] = j0 + y * kCols + State::in_block(i + e, lane) < end ? __builtin_amdgcn_exp2f(fmaf(s[y][i + e], c, -base)) : 0.0f;
                        p[(y * State::kInBlock + i) / 2] = T::pack(wt[0], wt[1]);
                    }
                }
#pragma unroll
                for (int f = 0; f < 32 / kInRow; ++f) {
                    uint64_t at[8];
                    int j[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int r = f * 8 + e;                            // the score's register, through the blocks
                        j[e] = j0 + r / State::kInBlock * kCols + State::in_block(r % State::kInBlock, lane);
                        at[e] = place_of(j[e]) + lane % kCols;
                    }
#pragma unroll
                    for (int d = 0; d < D / kCols; ++d) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const uint32_t y = (uint32_t)gv[at[e] + d * kCols] | (uint32_t)gv[at[e + 1] + d * kCols] << 16;
                            v[e / 2] = T::finite_or_0(y, j[e] >= hidden, j[e + 1] >= hidden);
                        }
                        x.o[d] = mfma(State::fragment(v), State::fragment(p + 4 * f), x.o[d]);
                    }
                }
            }
            const int mine = min(row_first + (int)(anew(lane) % kCols), w.rows - 1);
            const uint16_t* q = a.q + rows.token(mine) * a.q_stride + (int64_t)rows.head(mine) * D;
#pragma unroll 1
            for (int j0 = hidden; j0 < w.k1; j0 += 64) {
#pragma unroll 1
                for (uint64_t left = spoilt(j0); left; left &= left - 1) {
                    const int j = j0 + __ffsll((unsigned long long)left) - 1;
                    if (kKind == kFewRows && (j - w.k0) / 32 % kWaves != wave) continue;
                    const uint64_t at = place_of(j);
                    float s = 0.0f;
                    for (int e = 0; e < D; ++e) s = fmaf(T::up(q[e]), T::up(gk[at + e]), s);
                    const float p = __builtin_amdgcn_exp2f(fmaf(s, c, -base));
#pragma unroll
                    for (int d = 0; d < D / kCols; ++d)
#pragma unroll
                        for (int i = 0; i < State::kInBlock; ++i) {
                            const float y = T::up(gv[at + d * kCols + State::in_block(i, lane)]);
                            if (!(fabsf(y) < INFINITY) && j < end) x.o[d][i] = fmaf(p, y, x.o[d][i]);
                        }
                }
            }
        }
    }
    x.l = sum_of_row<kCols>(x.l + x.l1);

    // results through LDS, so that rows are written whole: a wavefront's rows of D floats, 16-byte chunk c of row r at c ^ r
    __shared__ float2 row_ml[kWaves][kCols];
    __shared__ bool left_out[rows_of(kKind)];
    constexpr uint32_t kFloatRow = D * 4, kFloatChunks = D / 4;
    auto meet = [] {
        if constexpr (!kAlone) __syncthreads();
        else wait_lds();
    };
    meet();                                              // tiles are done with
    const float m2 = x.reference(c);                     // (-infinity stays: c is positive)
    float mine = 1.0f;
    if (lane < kCols) row_ml[wave][lane] = make_float2(m2, x.l);
    // (without q_begin every token has a sequence; of parts the join leaves out rows that have none)
    const bool may_leave_out = !kAlone && w.of_all && a.parts == 1 && a.q_begin;
    if constexpr (!kAlone)
        if (may_leave_out && tid < rows_of(kKind)) left_out[tid] = !is_computed(a, rows.token(w.row0 + tid));
    if constexpr (kKind == kFewRows) {
        meet();
        float top = -INFINITY;
#pragma unroll
        for (int y = 0; y < kWaves; ++y) top = fmaxf(top, row_ml[y][lane % kCols].x);
        mine = __builtin_amdgcn_exp2f(m2 - (top == -INFINITY ? 0.0f : top));
    }
    constexpr uint32_t kRegion = 128 * D;                // (what the wavefront's own tiles take: others may still be at theirs)
    static_assert(kCols * kFloatRow <= kRegion, "");
    const uint32_t region = lds + wave * kRegion;
#pragma unroll
    for (int d = 0; d < D / kCols; ++d)
#pragma unroll
        for (int i = 0; i < State::kInBlock; i += 4) {
            const uint32_t r = lane % kCols, chunk = (d * kCols + State::in_block(i, lane)) / 4;
            *reinterpret_cast<LdsFloats>(lds_at(region + r * kFloatRow + (chunk ^ (r & (kFloatChunks - 1))) * 16)) =
                f32x4{x.o[d][i] * mine, x.o[d][i + 1] * mine, x.o[d][i + 2] * mine, x.o[d][i + 3] * mine};
        }
    meet();
    // a thread takes eight elements of a row: two chunks, neighbours for a result of 16 bits, head_dim / 2 apart for a part (so that
    // neighbouring threads write neighbouring chunks)
    const bool whole = a.parts == 1;
    constexpr int kPieces = D / 8, kOutRows = rows_of(kKind);
    for (int y = kAlone ? lane : tid; y < kOutRows * kPieces; y += kAlone ? 64 : kThreads) {
        const int r = y / kPieces, piece = y % kPieces, from = w.row0 + r;
        if (from >= w.rows) {
            if (kWide) continue;
            break;
        }
        if constexpr (!kAlone)
            if (may_leave_out && left_out[r]) continue;
        f32x4 lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
        float top, sum;
        const int in = r % kCols;
        auto chunk = [&](int wv, int e) { return *reinterpret_cast<LdsFloats>(lds_at(lds + wv * kRegion + in * kFloatRow + ((uint32_t)(whole ? 2 * piece + e : piece + e * kPieces) ^ (in & (kFloatChunks - 1))) * 16)); };
        if constexpr (kKind != kFewRows) {
            const int wv = kAlone ? wave : r / kCols;
            lo = chunk(wv, 0), hi = chunk(wv, 1);
            top = row_ml[wv][in].x, sum = row_ml[wv][in].y;
        } else {
            top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int wv = 0; wv < kWaves; ++wv) top = fmaxf(top, row_ml[wv][in].x);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int wv = 0; wv < kWaves; ++wv) {
                lo += chunk(wv, 0), hi += chunk(wv, 1);
                sum += row_ml[wv][in].y * __builtin_amdgcn_exp2f(row_ml[wv][in].x - base);
            }
        }
        const int64_t token = rows.token(from), head = rows.head(from);
        if (whole) {
            const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
            *reinterpret_cast<uint4*>(a.out + token * a.out_stride + head * D + piece * 8) =
                make_uint4(T::pack(lo[0] * f, lo[1] * f), T::pack(lo[2] * f, lo[3] * f), T::pack(hi[0] * f, hi[1] * f), T::pack(hi[2] * f, hi[3] * f));
            if (a.lse && piece == 0) a.lse[token * a.n_q_heads + head] = sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2;
        } else {
            const int64_t to = ((int64_t)w.part * a.n_tokens + token) * a.n_q_heads + head;
            *reinterpret_cast<f32x4*>(a.part_o + to * D + piece * 4) = lo;
            *reinterpret_cast<f32x4*>(a.part_o + to * D + D / 2 + piece * 4) = hi;
            if (piece == 0) a.part_ml[to] = make_float2(top, sum);
        }
    }
}

// Workgroups are dealt round-robin over the XCDs.  Those that read the same keys (the row tiles of a group: one key head, one run
// of keys) follow one another on one XCD, through its L2; groups go round the XCDs, so that long sequences spread.  `unit` counts
// rounds of eight workgroups, one on every XCD.
__device__ __forceinline__ bool group_of(const Segment& s, int unit, int xcd, int& group, int& tile)
{
    tile = unit % s.row_tiles;
    group = unit / s.row_tiles * kXcds + xcd;
    return group < s.groups;
}

// Rows of all tokens against a part of the prefix.
template <typename T, int D, Kind kKind>
__device__ __forceinline__ void attend_prefix(const AttendArgs& a, int unit, int xcd, char* lds, int32_t* ids)
{
    int group, tile;
    if (!group_of(a.prefix, unit, xcd, group, tile)) return;
    Item w;
    w.kv = group / a.prefix.splits;
    w.part = group % a.prefix.splits;
    w.token0 = 0;
    w.rows = a.n_tokens * a.group;
    w.row0 = tile * rows_of(kKind);
    w.k0 = w.part * a.prefix.split_len;
    w.k1 = (int)min((uint32_t)a.prefix_len, (uint32_t)w.k0 + (uint32_t)a.prefix.split_len);
    w.seen0 = a.prefix_len;
    w.seen_step = 0;
    w.own_pages = nullptr;
    w.of_all = true;
    attend<T, D, kKind>(a, w, lds, ids);
}

// Rows of one sequence against a part of its keys, or of the prefix and its keys.
template <typename T, int D, Kind kKind>
__device__ __forceinline__ void attend_own(const AttendArgs& a, int unit, int xcd, char* lds, int32_t* ids)
{
    int rest, tile;
    if (!group_of(a.own, unit, xcd, rest, tile)) return;
    if constexpr (kKind == kWaveRows) {                    // (four items a workgroup)
        rest = rest * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (rest >= a.own.items) return;
    }
    const int split = rest % a.own.splits;
    rest /= a.own.splits;
    Item w;
    w.kv = rest % a.c.n_kv_heads;
    const int b = rest / a.c.n_kv_heads;
    const int t0 = a.q_begin ? within(a.q_begin[b], 0, a.n_tokens) : b, t1 = a.q_begin ? within(a.q_begin[b + 1], t0, a.n_tokens) : b + 1;
    const int t = t1 - t0, own = a.max_own_len ? within(a.own_len[b], 0, a.max_own_len) : 0;
    w.token0 = t0;
    w.rows = min(t, a.max_q) * a.group;
    w.row0 = tile * rows_of(kKind);
    if (w.row0 >= w.rows) return;
    w.seen0 = a.prefix_len + own - t + 1;
    w.seen_step = t > 1 ? 1 : 0;
    const int last = min(w.rows, w.row0 + rows_of(kKind)) - 1;
    const int seen = max(a.prefix_len, w.seen0 + last / a.group);
    w.k0 = a.own_from + split * a.own.split_len;
    w.k1 = (int)min((uint32_t)seen, (uint32_t)w.k0 + (uint32_t)a.own.split_len);
    if (w.k0 >= w.k1 && a.parts > 1) return;
    w.part = a.own.first_part + split;
    w.own_pages = a.pages + b * a.pages_stride;
    w.of_all = false;
    attend<T, D, kKind>(a, w, lds, ids);
}

// Both kinds of work in one launch.  The prefix' workgroups come first, one a compute unit: they keep its matrix cores busy while the
// sequences' workgroups, in the room that is left beside each, keep the memory busy.  (Two a unit at first, or both kinds mixed evenly,
// take 10 to 15 % longer: 256 sequences with 64 heads behind 4096 keys 96 us, 122 and 114.)
template <typename T, int D, Kind kPrefix, Kind kOwn>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void k_attend(AttendArgs a)
{
    __shared__ __align__(1024) char lds[Lds<D, 32>::kBytes];
    __shared__ __align__(1024) int32_t ids[kWaves * 384];      // a wavefront: two sets of 64 page ids, two of 64 offsets
    const int unit = a.first_unit + blockIdx.x / kXcds, xcd = blockIdx.x % kXcds;
    if constexpr (kPrefix != kNone) {
        if (unit < a.prefix.units) attend_prefix<T, D, kPrefix>(a, unit, xcd, lds, ids);
        else attend_own<T, D, kOwn>(a, unit - a.prefix.units, xcd, lds, ids);
    } else {
        attend_own<T, D, kOwn>(a, unit, xcd, lds, ids);
    }
}

// Joins the parts of a row: twice four elements a thread, kLanes threads for every eight, each with every kLanes-th part.  Bound by
// latency (the launch, the sequence's length, then all parts in one go): 33 sequences of up to 6 tokens with 15 heads 5 us of 21, 64
// sequences with 32 heads and 22 parts, 23 MB, 7 of 70.  (With the parts' maxima first and then the parts, four at once, by 16 threads
// from 17 parts on, 1.5 to 2 us more.)
template <typename T, int D, int kLanes>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a, int row_blocks, int first_block)
{
    constexpr int kPieces = D / 8, kRowsHere = kThreads / kPieces / kLanes;
    const int piece = threadIdx.x % kPieces, mine = threadIdx.x / kPieces % kLanes;
    const int block = first_block + blockIdx.x, b = block / row_blocks, r = block % row_blocks * kRowsHere + threadIdx.x / kPieces / kLanes;
    const int t0 = a.q_begin ? within(a.q_begin[b], 0, a.n_tokens) : b, t1 = a.q_begin ? within(a.q_begin[b + 1], t0, a.n_tokens) : b + 1;
    const int t = t1 - t0, i = r / a.n_q_heads, own = a.max_own_len ? within(a.own_len[b], 0, a.max_own_len) : 0;
    const bool there = i < min(t, a.max_q);
    const int seen = max(a.prefix_len, a.prefix_len + own - t + 1 + i);
    const int of_own = seen > a.own_from ? (int)(((uint32_t)(seen - a.own_from) + (uint32_t)a.own.split_len - 1) / (uint32_t)a.own.split_len) : 0, parts = there ? a.own.first_part + of_own : 0;
    const int64_t token = t0 + i, head = r % a.n_q_heads, row = token * a.n_q_heads + head, pitch = (int64_t)a.n_tokens * a.n_q_heads;
    constexpr int kAtOnce = 8;
    float top = -INFINITY, base, sum = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    for (int y0 = mine; y0 < parts; y0 += kAtOnce * kLanes) {    // (nearly always all there are)
        float2 ml[kAtOnce];
        float4 lo[kAtOnce], hi[kAtOnce];
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
            const int64_t at = min(y0 + x * kLanes, parts - 1) * pitch + row;
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
        __shared__ float of[10][kThreads];
#pragma unroll
        for (int e = 0; e < 8; ++e) of[e][threadIdx.x] = o[e];
        of[8][threadIdx.x] = sum;
        of[9][threadIdx.x] = top;
        __syncthreads();
        if (mine) return;
        for (int y = 1; y < kLanes; ++y) top = fmaxf(top, of[9][threadIdx.x + y * kPieces]);
        base = top == -INFINITY ? 0.0f : top;
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
        for (int y = 0; y < kLanes; ++y) {
            const int x = threadIdx.x + y * kPieces;
            const float f = __builtin_amdgcn_exp2f(of[9][x] - base);
            sum = fmaf(of[8][x], f, sum);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(of[e][x], f, o[e]);
        }
    }
    if (!there) return;
    const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t* out = a.out + token * a.out_stride + head * D + piece * 4;
    *reinterpret_cast<uint2*>(out) = make_uint2(T::pack(o[0] * f, o[1] * f), T::pack(o[2] * f, o[3] * f));
    *reinterpret_cast<uint2*>(out + D / 2) = make_uint2(T::pack(o[4] * f, o[5] * f), T::pack(o[6] * f, o[7] * f));
    if (a.lse && piece == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

bool sizes_ok(const fr_attend_desc& d)
{
    if (!kv_pages_shape_ok(d.cache) || d.n_tokens < 0 || d.n_seqs < 0 || d.max_q < 1) return false;
    if (d.n_q_heads < 1 || d.n_q_heads > 1024 || d.n_q_heads % d.cache.n_kv_heads) return false;
    if ((int64_t)d.n_tokens * d.n_q_heads > 0x7fffffff - 4096) return false;
    return d.prefix_len >= 0 && d.max_own_len >= 0 && (int64_t)d.prefix_len + d.max_own_len < 0x7fffffff - 4096;
}

// How a call is cut: which keys the prefix' workgroups take, and in how many parts.
struct Plan {
    Kind of_prefix = kNone, of_own = kFewRows;
    Segment prefix{}, own{};
    int parts = 1;
    int64_t blocks = 0;                    // of the attention or the join, whichever are more
};
constexpr int64_t kMostBlocks = 0x7fffffff;            // (they are counted in 32 bits)

// What a call takes, roughly, in microseconds: enough to tell ways to cut it from one another.  A workgroup with tiles of 128 rows
// needs `one` for a tile of 64 keys where it has a unit to itself and `all` where as many are on the unit as fit, and kStart to begin
// and end; results of several parts are written, read and joined.  (1.43 and 2.0 are measured; those of head_dim 64 are about half of
// that: with 0.7 and 1.1 three of 36 calls take 6 to 17 % longer, none is faster.)
// Tiles of 128 rows, against parts of 128 to 2048 keys, as many as four workgroups a unit ask for, and the prefix gone through by every
// sequence from 128 rows a sequence on, of 32 heads with 8 key heads: one sequence's 640 rows behind 8192 keys 70 -> 44 us, 2800 rows behind 512
// 63 -> 34; 64 sequences' 96 rows against 250 keys 46 -> 24; 8 sequences' 160 rows behind 2048 shared keys 53 -> 33, 32 sequences'
// 640 rows 322 -> 217; where the prefix is short it stays with the sequences (32 of 640 rows behind 512 keys 84; taken apart 134).
struct Cost {
    double one, all;
    int at_once, dim;
    explicit Cost(int D) : one(D == 128 ? 1.43 : 0.9), all(D == 128 ? 2.0 : 1.6), at_once(D == 128 ? 2 : 3), dim(D) {}
    static constexpr double kStart = 4.0, kJoin = 4.0, kBytesAUs = 4e6, kRound = 0.6, kStartFew = 3.0, kBytesAgain = 12e6;
    double tile(double a_unit) const { return a_unit <= 1 ? one : one + (all - one) * (std::min(std::ceil(a_unit), (double)at_once) - 1) / (at_once - 1); }
    double workgroups(double blocks, double tiles, int cus) const
    {
        const double a_unit = blocks / cus, full = std::floor(a_unit / at_once), rest = a_unit - full * at_once;
        return tiles * (full * all + (rest > 0 ? tile(rest) : 0)) + kStart * std::ceil(a_unit / at_once);
    }
    // two kinds of workgroups in one launch
    double both(double blocks0, double tiles0, double blocks1, double tiles1, int cus) const
    {
        const double a_unit = (blocks0 + blocks1) / cus, work = (blocks0 * tiles0 + blocks1 * tiles1) * all / at_once / cus;
        return std::max(work + 0.25 * all * tiles1, tile(a_unit) * std::max(tiles0, tiles1)) + kStart * std::ceil(a_unit / at_once);
    }
    // Workgroups of four wavefronts with 16 rows, which take 32 keys each in a round: kRound us where a unit's memory keeps up, and no
    // faster than memory is, or the caches for keys that every sequence reads again.
    double few(double blocks, double tiles, double own_keys, double again, int cus) const
    {
        const double rounds = tiles / 2 * kRound;
        return kStartFew + 0.5 * rounds + std::max(rounds * std::ceil(blocks / (at_once * cus)), reading(own_keys, cus) + again * dim * 4 / kBytesAgain);
    }
    double reading(double keys, int cus) const { return keys * dim * 4 / std::min(5.7e6, cus * 40e3); }
    static double join(int64_t parts, const fr_attend_desc& d)
    {
        return parts < 2 ? 0 : kJoin + (double)parts * d.n_tokens * d.n_q_heads * d.cache.head_dim * (2 * sizeof(float)) / kBytesAUs;
    }
};

// Threads of the join for eight elements of a row, one where it has all parts in one go, else four; rows of its workgroups.
int join_lanes(int parts) { return parts <= 8 ? 1 : 4; }
int join_rows(int parts, int head_dim) { return kThreads / (head_dim / 8) / join_lanes(parts); }

int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

// Rows of results in parts that a call has room for; no call with smaller sizes has more, so that a program can ask once for its
// largest.  `plan` makes no more than four workgroups a unit by cutting keys (16 where a wavefront takes an item), and two where few
// rows' prefix is taken apart; what is not cut has one part of every row, of the prefix and of the own keys.
constexpr int64_t kMostFew = 32;           // rows of a sequence that are few
constexpr int64_t kMostShared = 1 << 21;   // many rows are not taken apart from there on (2 GB of results; one in a hundred such calls would be)
int64_t most_part_rows(const fr_attend_desc& d)
{
    const int64_t group = d.n_q_heads / d.cache.n_kv_heads, rows = (int64_t)d.n_tokens * d.n_q_heads, parts = up(d.prefix_len, 128) + up(d.max_own_len, 128);
    const bool few = d.max_q * group <= kMostFew;
    const int64_t own = few ? 16 * kUnits * std::min<int64_t>(16, d.max_q * group) : 4 * kUnits * 128;
    const int64_t prefix = few ? 2 * kUnits * std::min<int64_t>(128, d.n_tokens * group) : 4 * kUnits * 128;
    if (parts < 2) return 0;
    if (d.prefix_len == 0) return std::min(rows * parts, own);
    const int64_t of_few = group <= kMostFew ? std::min<int64_t>(d.n_tokens, d.n_seqs * (kMostFew / group)) * d.n_q_heads : 0;
    const int64_t shared = std::max(of_few, std::min(rows, kMostShared));
    return std::min(rows * parts, std::max(shared, own) + std::max(shared, prefix));
}

// `whole`: in one part
Plan plan(const fr_attend_desc& d, int cus, bool whole = false)
{
    Plan p;
    const int64_t group = d.n_q_heads / d.cache.n_kv_heads, heads = d.cache.n_kv_heads;
    const int64_t tokens_a_seq = std::min(d.max_q, d.n_tokens), seq_rows = tokens_a_seq * group, all_rows = d.n_tokens * group;
    // Rows of a sequence up to which tiles of 16 are taken, above, tiles of 128: several of those read the same keys, but do not wait
    // for one another.  8 key heads, in tiles of 16 and of 128: 32 rows, 256 sequences of 64 keys 23 and 36 us, 4 of 1000 13.5 and
    // 15.4, 16 of 4000 52 and 52; 64 rows, 64 sequences of 250 keys 21.5 and 22, of 1000 79 and 49, 16 of 1000 28 and 25.
    cus = std::min(cus, kUnits);
    const Cost cost(d.cache.head_dim);
    auto finish = [&](Segment& s, int64_t items, int64_t at_once) {
        const int64_t groups = up(items, at_once), units = up(groups, kXcds) * s.row_tiles;
        s.items = (int)std::min<int64_t>(items, 0x7fffffff);
        s.groups = (int)std::min<int64_t>(groups, 0x7fffffff);
        s.units = (int)std::min<int64_t>(units, 0x7fffffff);
        p.blocks += units * kXcds;
    };
    // `keys` in parts of a whole number of tiles, two at least: as many as cost(parts, tiles of a part) is least for, of powers of two,
    // the numbers that give every unit up to four workgroups, and parts of two tiles
    auto cut = [&](Segment& s, int64_t keys, int64_t blocks, auto cost) {
        double least = INFINITY;
        const int64_t most = whole ? 1 : std::max<int64_t>(up(keys, 128), 1);
        auto consider = [&](int64_t n) {
            if (n < 1 || n > most) return;
            const int64_t len = std::max<int64_t>(up(up(keys, n), 64), 1) * 64, parts = std::max<int64_t>(up(keys, len), 1);
            const double t = cost(parts, len / 64);
            if (t < least) { least = t; s.split_len = (int)std::min<int64_t>(len, 0x7fffffc0); s.splits = (int)parts; }
        };
        for (int64_t n = 1; n == 1 || n * blocks <= 4 * cus; n *= 2) consider(n);
        for (int a_unit = 1; a_unit <= 4; ++a_unit) consider(a_unit * cus / blocks);
        if (most * blocks <= cus) consider(most);
        return least;
    };
    p.of_own = seq_rows > kMostFew ? kWideRows : kFewRows;
    Segment &s = p.own, &shared = p.prefix;
    s.row_tiles = (int)up(seq_rows, rows_of(p.of_own));
    shared.row_tiles = (int)up(all_rows, rows_of(all_rows > kMostFew ? kWideRows : kFewRows));
    bool share = d.prefix_len > 0 && d.n_seqs > 1 && !whole && (p.of_own == kFewRows || (int64_t)d.n_tokens * d.n_q_heads <= kMostShared);
    const int64_t base = (int64_t)d.n_seqs * heads * s.row_tiles;
    if (p.of_own == kWideRows) {
        // row tiles that hold rows, half of a sequence's last one being empty
        const double tiles = std::min((double)d.n_seqs * s.row_tiles, all_rows / 128.0 + 0.5 * d.n_seqs) * heads;
        auto alone = [&](int64_t parts, int64_t t) { return cost.workgroups(tiles * parts, (double)t, cus) + cost.join(parts, d); };
        double together = INFINITY;
        if (share) {
            if (d.max_own_len) cut(s, d.max_own_len, base, alone);
            together = cut(shared, d.prefix_len, shared.row_tiles * heads, [&](int64_t parts, int64_t t) {
                return cost.both((double)shared.row_tiles * heads * parts, (double)t, tiles * s.splits, s.split_len / 64.0, cus) +
                       cost.join(parts + s.splits, d);
            });
        }
        const Segment own = s;
        if (cut(s, (int64_t)d.prefix_len + d.max_own_len, base, alone) <= together) {
            share = false;
        } else {
            s = own;
        }
    } else if (share) {
        // (one workgroup a unit leaves room for the sequences' own; two, 64 sequences behind 12000 keys 47 instead of 37 us.  Without
        // own keys two: 256 sequences behind 16384 keys 151 instead of 166)
        const int64_t most = up(d.prefix_len, 256), want = (d.max_own_len ? 1 : 2) * cus / (shared.row_tiles * heads);
        const int64_t splits = std::max<int64_t>(1, std::min(most, want));
        shared.split_len = (int)(up(up(d.prefix_len, splits), 64) * 64);
        shared.splits = (int)up(d.prefix_len, shared.split_len);
        // Few rows a sequence: taken apart, the prefix is read once, but there are parts to join.  The estimate against 8192 or more keys
        // in all, 32 heads with 8 key heads and 8 with one: 32 sequences behind 300 keys 15.5 -> 8.6 and 13.5 -> 8.3 us, 128 behind 300
        // 22.5 either way and 14.5 -> 8.4, 4 behind 2000 11.7 -> 10.3 and 9.8 either way; of 64 behind 5000 (taken apart) 26 and 18, by
        // every sequence 67 and 22.
        const double tiles = shared.split_len / 64.0, own = (double)base * d.max_own_len;
        const double together = (all_rows > kMostFew ? Cost::kStart + tiles * cost.tile((double)shared.row_tiles * heads * shared.splits / cus)
                                                     : cost.few((double)heads * shared.row_tiles * shared.splits, tiles, (double)heads * d.prefix_len, 0, cus)) +
                                cost.reading(own, cus) + cost.join(shared.splits + (own > 0 ? 1 : 0), d);
        share = together < cut(s, (int64_t)d.prefix_len + d.max_own_len, base, [&](int64_t parts, int64_t t) {
            return cost.few((double)base * parts, (double)t, own, (double)base * d.prefix_len, cus) + cost.join(parts, d);
        });
    }
    if (share) {
        p.of_prefix = all_rows > kMostFew ? kWideRows : kFewRows;
        finish(shared, heads * shared.splits, 1);
    } else {
        shared = {};
    }
    const int64_t keys = (share ? 0 : d.prefix_len) + (int64_t)d.max_own_len;
    s.first_part = shared.splits;
    if (keys || !share) {
        if (p.of_own == kFewRows) {
            // (Against parts that give four workgroups a unit, of 128 keys at least: 8 sequences of 200 to 300 keys 8.9 -> 6.6 us, 12 of 2000
            // 25 -> 21, 1 of 60000 47 -> 43, 128 of 4000 278 -> 261.)
            cut(s, keys, base, [&](int64_t parts, int64_t t) {
                return cost.few((double)base * parts, (double)t, (double)base * d.max_own_len, share ? 0 : (double)base * d.prefix_len, cus) +
                       cost.join(parts + shared.splits, d);
            });
            // Short caches: a wavefront an item.  By themselves, where each unit has four of up to 256 keys: 256 sequences of 64 keys with 8 key
            // heads 12 us, a workgroup an item 20, 128 of 200 17 and 19; of 400 50 either way, 64 of 200 12 and 10, of 800 28 and 25.
            // Behind a prefix, whose workgroups take half of a unit, items of 256 keys (128 where they are few, more where they are many),
            // if there are enough, of up to 2048 keys, 512 where there are many.  A wavefront and a workgroup an item, up to so many own keys
            // behind 4096: 64 sequences, 32 heads: 300 24 and 26, 512 27 and 31, 1500 48 and 53, 2000 73 and 71; 128, 64 heads: 300 39 and 41,
            // 512 43 and 46, 600 52 and 50, 1100 86 and 77; 256, 32 heads: 100 38 and 44, 400 60 either way, 512 71 either way, 600 93 and 86;
            // 64 heads: 400 74 and 76, 512 86 and 88, 600 104 and 98.  64 of up to 1500 behind 16384: 73.5; in parts of 512 77.1.
            int64_t wave_len = base < cus ? 128 : 256;
            while (base * up(keys, wave_len) > (base < cus ? 4 : 16) * cus && wave_len < keys) wave_len *= 2;
            const bool enough = !whole && base >= cus / 2 && base * up(keys, wave_len) >= (base < cus ? 4 : 3) * cus / 2;
            if (share ? p.of_prefix == kWideRows && enough && keys <= (base < 4 * cus ? 2048 : 512) : base >= 4 * cus && keys <= 256) {
                p.of_own = kWaveRows;
                s.split_len = (int)wave_len;
                s.splits = (int)std::max<int64_t>(1, up(keys, wave_len));
            }
        }
        finish(s, (int64_t)d.n_seqs * heads * s.splits, p.of_own == kWaveRows ? kWaves : 1);
    } else {
        s.splits = 0;
        s.split_len = 1;
    }
    p.parts = p.prefix.splits + s.splits;
    if (p.parts * (int64_t)d.n_tokens * d.n_q_heads > most_part_rows(d) && p.parts > 1) return plan(d, cus, true);     // (most tokens in no sequence)
    if (p.parts > 1) p.blocks = std::max(p.blocks, d.n_seqs * up(tokens_a_seq * d.n_q_heads, join_rows(p.parts, d.cache.head_dim)));
    return p;
}

uint64_t part_bytes(const fr_attend_desc& d) { return (uint64_t)most_part_rows(d) * (d.cache.head_dim * 4 + 8); }

template <typename T, int D>
int launch(AttendArgs a, const Plan& p, hipStream_t stream)
{
    constexpr int kBlocksALaunch = kMostThreads / kThreads;
    auto go = [&](auto kernel) {
        const int units = a.prefix.units + a.own.units;
        for (a.first_unit = 0; a.first_unit < units; a.first_unit += kBlocksALaunch / kXcds)
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(units - a.first_unit, kBlocksALaunch / kXcds) * kXcds), dim3(kThreads), 0, stream, a);
    };
    if (p.of_prefix == kNone) {
        if (p.of_own == kFewRows) go(k_attend<T, D, kNone, kFewRows>);
        else if (p.of_own == kWaveRows) go(k_attend<T, D, kNone, kWaveRows>);
        else go(k_attend<T, D, kNone, kWideRows>);
    } else if (p.of_prefix == kFewRows) {              // (few rows in all: few of a sequence, and few sequences)
        go(k_attend<T, D, kFewRows, kFewRows>);
    } else {
        if (p.of_own == kFewRows) go(k_attend<T, D, kWideRows, kFewRows>);
        else if (p.of_own == kWaveRows) go(k_attend<T, D, kWideRows, kWaveRows>);
        else go(k_attend<T, D, kWideRows, kWideRows>);
    }
    if (p.parts > 1) {
        const int rows = join_rows(p.parts, D), blocks = (int)((std::min<int64_t>(a.max_q, a.n_tokens) * a.n_q_heads + rows - 1) / rows);
        const int64_t all = (int64_t)a.n_seqs * blocks;
        for (int64_t first = 0; first < all; first += kBlocksALaunch) {
            const dim3 joins((unsigned)std::min<int64_t>(all - first, kBlocksALaunch));
            if (join_lanes(p.parts) == 1) hipLaunchKernelGGL((k_attend_join<T, D, 1>), joins, dim3(kThreads), 0, stream, a, blocks, (int)first);
            else hipLaunchKernelGGL((k_attend_join<T, D, 4>), joins, dim3(kThreads), 0, stream, a, blocks, (int)first);
        }
    }
    return hipGetLastError() == hipSuccess ? FR_OK : FR_ERR_HIP;
}

}  // namespace

extern "C" {

int fr_attend_shared_workspace_bytes(const fr_attend_desc* d, uint64_t* bytes_out)
{
    if (!d || !bytes_out || !sizes_ok(*d)) return FR_ERR_ARG;
    *bytes_out = 0;
    if (d->n_tokens == 0 || d->n_seqs == 0) return FR_OK;
    const Plan p = plan(*d, kUnits);
    if (p.blocks > kMostBlocks) return FR_ERR_ARG;
    *bytes_out = part_bytes(*d);
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
                    d->pages, d->own_len, d->n_tokens, d->n_seqs, d->n_q_heads, d->q_begin ? d->max_q : 1, d->prefix_len, d->max_own_len,
                    __builtin_ctz(c.page_size), d->n_q_heads / c.n_kv_heads, d->scale};
    // cut for the units that the stream may use, in no more parts than the workspace was asked for
    const Plan whole = plan(*d, kUnits);
    const int cus = (int)fr_stream_cus((hipStream_t)stream);
    Plan p = cus < kUnits ? plan(*d, cus) : whole;
    if (whole.blocks > kMostBlocks) return FR_ERR_ARG;
    if (p.parts > whole.parts || p.blocks > kMostBlocks) p = whole;
    if (whole.parts > 1 && (!d->workspace || ((uintptr_t)d->workspace & 255) || d->workspace_bytes < part_bytes(*d))) return FR_ERR_ARG;
    a.own_from = p.of_prefix == kNone ? 0 : d->prefix_len;
    a.prefix = p.prefix;
    a.own = p.own;
    a.parts = p.parts;
    a.part_o = (float*)d->workspace;
    a.part_ml = (float2*)((char*)d->workspace + (uint64_t)p.parts * d->n_tokens * d->n_q_heads * c.head_dim * 4);
    hipStream_t s = (hipStream_t)stream;
    if (c.dtype == FR_DTYPE_BF16) return c.head_dim == 64 ? launch<Bf16, 64>(a, p, s) : launch<Bf16, 128>(a, p, s);
    return c.head_dim == 64 ? launch<F16, 64>(a, p, s) : launch<F16, 128>(a, p, s);
}

}  // extern "C"
