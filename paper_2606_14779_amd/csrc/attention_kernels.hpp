// Kernels of attention over the paged cache, for gfx950 (MI355X): attention.hip, whose first lines have the formulas,
// launches them on 16-bit pages, attention_tree.hip with a mask among the new tokens, attention_e4m3.hip on 8-bit pages.
//
// With a mask a new token sees all keys before the new ones (as far as its window goes) and the new ones whose bit is set in
// its row, words of 64 bits: tiles of keys before the new tokens are as under a causal mask without an edge, and the
// others' bits are shifted to where the tile begins.
// Of 8-bit pages the elements become 16-bit floats on their way to the products: exact, one instruction for two of them with
// their power of two (e4m3.hpp), so that all that follows is the same.
#ifndef KVP_ATTENTION_KERNELS_HPP
#define KVP_ATTENTION_KERNELS_HPP

#include <type_traits>

#include "e4m3.hpp"

namespace kvp {

namespace {

// What a kernel reads: 16-bit pages under a causal mask, the same with a mask among the new tokens, or 8-bit pages with
// either mask.
enum PageKind { kCausal16, kTree16, kEight };

// Row of a cached token: of the cache, or with 8-bit pages of its slot; kNoRow where the slot is none of the cache's.
template <int KIND>
__device__ __forceinline__ uint32_t row_in(const CacheView &c, int32_t slot, uint32_t kv_head, uint32_t token)
{
    if constexpr (KIND != kEight) return row_of(c, slot, kv_head, token);
    const uint32_t row = kv_head * c.block + token - block_of(c, token) * c.block;
    return (uint32_t)slot < c.num_slots ? row : kNoRow;
}
// Where a row of 8-bit pages begins, and its exponents; row 0 of the cache in the place of one that is not there.
template <class Offset>
__device__ __forceinline__ Offset elements_at(const AttentionArgs &a, int32_t slot, uint32_t row)
{
    return row == kNoRow ? 0 : (Offset)slot * (Offset)a.slot_bytes + (Offset)row * a.c.head_dim;
}
template <class Offset>
__device__ __forceinline__ Offset exponents_at(const AttentionArgs &a, int32_t slot, uint32_t row)
{
    return (row == kNoRow ? 0 : (Offset)slot * (Offset)a.slot_bytes + (Offset)row * a.row_exponents) + a.exponents;
}

// Eight elements of a cache's row, from element d on; r counts rows of a head over all slots.
template <class T, int KIND>
__device__ __forceinline__ w4 eight_at(const AttentionArgs &a, const uint16_t *cache, uint32_t r, uint32_t d)
{
    if constexpr (KIND == kEight) {
        const uint32_t rows = a.c.kv_heads * a.c.block, slot = r / rows;
        const uint8_t *p = (const uint8_t *)cache + (uint64_t)slot * a.slot_bytes;
        const uint64_t row = r - slot * rows;
        const uint32_t word = (uint32_t)load4g((const int32_t *)(p + a.exponents + row * a.row_exponents) + d / 128);
        return widen<T>(load8g((const uint16_t *)(p + row * a.c.head_dim + d)), power_of(word, d / 32 % 4 * 8));
    } else {
        return load16g(cache + (uint64_t)r * a.c.head_dim + d);
    }
}

// The new tokens `from` to from + 63 of its sequence that a new token sees.
__device__ __forceinline__ uint64_t tree_bits(const AttentionArgs &a, const Seq &s, int32_t token, int32_t from)
{
    const uint64_t *row = a.tree + (uint64_t)(s.q_begin + token) * a.tree_words;
    const int32_t word = from >> 6, shift = from & 63, words = (int32_t)a.tree_words;
    const uint64_t low = word >= 0 && word < words ? row[word] : 0;
    const uint64_t high = shift && word + 1 >= 0 && word + 1 < words ? row[word + 1] : 0;
    return low >> shift | high << (63 - shift) << 1;
}

// How many new tokens it sees.
__device__ __forceinline__ int32_t tree_depth(const AttentionArgs &a, const Seq &s, int32_t token)
{
    const uint64_t *row = a.tree + (uint64_t)(s.q_begin + token) * a.tree_words;
    int32_t depth = 0;
    for (int32_t from = 0; from < s.n_q; from += 64) {
        const uint64_t x = row[from / 64];
        depth += __popcll(s.n_q - from < 64 ? x & ((1ull << (s.n_q - from)) - 1) : x);
    }
    return depth;
}

// Sum of a row's weights with the sink's, and its logarithm: what a finished row needs.
struct RowEnd {
    float scale_o;   // of the accumulated output
    float lse;
};
__device__ __forceinline__ RowEnd finish_row(float m, float l, const float *sinks, uint32_t head)
{
    float f = 1.0f;
    if (sinks) {
        const float s = sinks[head] * kLog2e;
        const float top = fmaxf(m, s);
        f = exp2_fast(m - top);
        l = l * f + exp2_fast(s - top);
        m = top;
    }
    // an empty row has l = 0 (and no sink): output 0, lse -inf
    return {l == 0.0f ? 0.0f : f / l, l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2};
}

struct Split {
    int32_t begin, end;   // keys
};
// Keys of one workgroup: what its rows can see, cut into the launch's parts of split_keys.
__device__ __forceinline__ Split keys_of(const AttentionArgs &a, const Seq &s, int32_t first_token, int32_t last_token,
                                         uint32_t split, uint32_t split_keys)
{
    const int32_t shift = s.kv - s.n_q;
    int32_t lo = 0;
    if (a.window) lo = (int32_t)max((int64_t)0, (int64_t)(shift + first_token) + 1 - (int64_t)a.window);
    lo &= ~(int32_t)(kTileKeys - 1);
    const int32_t hi = min(shift + last_token + 1, s.kv);
    const int64_t begin = (int64_t)lo + (int64_t)split * split_keys;
    const int64_t end = split + 1 == a.splits ? (int64_t)hi : min((int64_t)hi, begin + (int64_t)split_keys);
    return {(int32_t)min(begin, (int64_t)max(hi, 0)), (int32_t)max(end, (int64_t)0)};
}

// Keys of a part where the lengths of a batch decide, which the host does not know: lane i has sequence i's span of keys and
// its row tiles (0: none), and every workgroup finds the same.  The parts of a call are at most a.splits.
__device__ __forceinline__ uint32_t lowest_of(uint32_t x)
{
    for (int d = 1; d < 64; d *= 2) x = min(x, (uint32_t)__shfl_xor(x, d));
    return (uint32_t)__builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ uint32_t longest_of(uint32_t x) { return ~lowest_of(~x); }
// Workgroups of row tiles, one to a CU: of 1 to 64 parts to the longest sequence that number for which the rounds of the chip,
// each as long as a part's tiles of keys (2.1 us each at head_dim 128) and about five more to begin and end, take least.
// Trees of 16 x 32 over up to 8K (32, 8, 128): 123 us by sizes alone, 94 so; of 64 x 4 over 32K (32, 4, 128) 220 and 175.
// Where max_kv is far above the lengths, as in a graph for all of them (2 x 8 tokens over 4K, max_kv 128K), 116 and 28; where
// it is not and all parts run at once, 1 to 2 us more.
__device__ __forceinline__ uint32_t keys_of_rounds(const AttentionArgs &a, uint32_t span, uint32_t tiles)
{
    const uint32_t lane = threadIdx.x & 63, longest = longest_of(tiles ? span : 0);
    const uint32_t n = min(lane + 1, a.splits), keys = max((longest + n - 1) / n + 63 & ~63u, 64u);
    const float per_key = 1.0f / (float)keys;
    uint32_t count = 0;
    for (uint32_t s = 0; s < a.c.n_seq; ++s)
        count += (uint32_t)__builtin_amdgcn_readlane(tiles, s) *
                 (uint32_t)ceilf((float)(uint32_t)__builtin_amdgcn_readlane(span, s) * per_key);
    const uint32_t rounds = (count * a.c.kv_heads + 255) / 256;
    const uint32_t best = lowest_of(min(rounds * (keys / 64 + 5), (1u << 26) - 1) << 6 | lane) & 63;
    return (uint32_t)__builtin_amdgcn_readlane(keys, best);
}

// A row must not meet the infinities and NaN of values that it does not see, but a weight of 0 times them is NaN, and in a
// product every row meets every value of a tile.  So both kernels look at the values of the tiles that not all of their
// rows see, and hand the product 0 in the place of those that are not finite.  Where there was one, these tiles are gone
// over once more before a row ends, key by key: what each row that sees such a key lacks of its output is added here.
// 256 new tokens over 64K (32 heads, 8 KV heads, 128) take 0.34 ms with an infinity among the newest values or without;
// going over all keys of the rows once more took 140 ms.

// The weight of a key, row r of the cache, in this lane's row: q[i] are the row's elements from at(i) on, and add sums a
// value over the lanes that have the others.
template <class T, int KIND, int Q, class At, class Add>
__device__ __forceinline__ float weight_of(const AttentionArgs &a, const w4 (&q)[Q], uint32_t r, float m, At at, Add add)
{
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        if (at(i) >= a.c.head_dim) continue;
        const w4 y = eight_at<T, KIND>(a, a.k, r, at(i));
#pragma unroll
        for (int e = 0; e < 8; ++e) x = __builtin_fmaf(T::unpack(q[i][e / 2], e & 1), T::unpack(y[e / 2], e & 1), x);
    }
    return exp2_fast(__builtin_fmaf(add(x), a.scale_log2, -m));
}
// Four elements of a value's row.
template <class T, int KIND>
__device__ __forceinline__ w2 four_at(const AttentionArgs &a, uint32_t r, uint32_t d)
{
    if constexpr (KIND == kEight) {
        const w4 v = eight_at<T, KIND>(a, a.v, r, d & ~7u);
        return d & 4 ? w2{v[2], v[3]} : w2{v[0], v[1]};
    } else {
        return load8g(a.v + (uint64_t)r * a.c.head_dim + d);
    }
}
// What a row lacks of element e of four: the products left out.
template <class T>
__device__ __forceinline__ float unbounded_part(w2 v, int e, float weight)
{
    const float x = T::unpack(v[e / 2], e & 1);
    return __builtin_isfinite(x) ? 0.0f : weight * x;
}
// Whether a value's row has an element that is not finite.
template <class T, int KIND>
__device__ __forceinline__ bool unbounded_row(const AttentionArgs &a, uint32_t r)
{
    bool all = true;
    for (uint32_t d = 0; d < a.c.head_dim; d += 8) all &= T::finite(eight_at<T, KIND>(a, a.v, r, d));
    return !all;
}

// ---- many rows

// 32 rows to a wave, two waves to a SIMD that work in turns: while one feeds the matrix cores (the products of tile
// t with K and of tile t - 1 with V), the other's vector unit turns its logits into weights; a barrier ends each
// stage.  A tile of 64 keys at head_dim 128 is 32 products of 32 cycles, and beside them about 140 vector
// instructions for the softmax alone (a maximum, a scaled difference, an exponential, a sum and half a rounding per
// logit), so the rest is kept off the vector unit: 32-bit offsets from scalar bases where a buffer has less than
// 2^32 bytes (Offset), buffers of LDS known at compile time (the loop is written for two tiles), masks and zeros
// only in the tiles that need them.
//
// Stages: the first half of the waves has products(t) in stage 2t and softmax(t) in 2t + 1, the second half one
// stage later.  What the products of stage 2t read, K(t) and V(t - 1), is stored by the first half in stage 2t - 1
// and by the second in 2t - 2; the buffers' last readers are done at the end of stage 2t - 3.
//
// 512 new tokens over 128K (32 heads, 8 KV heads, 128): 1074 us, 1022 TFLOP/s, where a bf16 matrix product of 16384^3
// reaches 1370.  Matrix cores busy for 51 % of the cycles, no LDS bank conflicts, 87 % of the L2 reads hit; the clock
// falls to about 2.0 GHz of 2.4 under it.  Without turns (four waves, two such workgroups to a CU) 1218 us.
// The same over 8-bit pages: 1055 to 1097 us by card where 16-bit ones take 1050 to 1090: an eighth more vector
// instructions, for widening what a lane has loaded, and half the bytes.  64 drafts over 128K (32, 4, 128) in 8 bits: 163 to
// 172 us with the join, 800 to 840 TFLOP/s, 67 tiles to each of 248 workgroups.  Two tiles ahead instead of one: 2 % more for 8-bit pages, 1 % less for
// 16-bit ones.
template <class T, int DP, class Offset, int KIND = kCausal16>
__global__ __launch_bounds__(row_waves(DP) * 64, row_waves(DP) / 4) void attention_rows(const AttentionArgs a)
{
    constexpr int TK = kTileKeys, NW = row_waves(DP), TR = NW * 32;
    constexpr bool E8 = KIND == kEight;
    constexpr int XW = E8 ? (DP + 127) / 128 : 1;    // words of exponents to a row of 8-bit pages
    constexpr int CH = DP / 8;                       // 16-byte pieces of a row
    constexpr int PASS = NW * 64 / CH;               // rows that the workgroup loads at once
    constexpr int N = TK / PASS;
    constexpr uint32_t BUF = TK * DP * 2;            // bytes of a tile: buffers K0, K1, V0, V1
    __shared__ __align__(16) char lds[4 * BUF];

    const CacheView &c = a.c;
    const uint32_t kv_head = blockIdx.x % c.kv_heads;
    const uint32_t rest = blockIdx.x / c.kv_heads;
    // the tiles of a part of the keys run side by side, so that its keys come from L2 for all but one of them;
    // under a causal mask later tiles have more keys
    uint32_t split, seq, row0, split_keys = a.split_keys;
    Seq s;
    if (c.n_seq > 1 && c.n_seq <= 64) {
        const Tile t = tile_by_length(c, rest, a.splits, TR, TK);
        if (t.tile == kNoTile) return;
        if (a.uneven) split_keys = keys_of_rounds(a, t.mine.kv, t.tiles);
        split = t.split;
        seq = t.seq;
        s = t.s;
        row0 = t.tile * TR;
    } else {
        split = rest / a.tiles;
        const uint32_t tile = a.tiles - 1 - rest % a.tiles;
        seq = seq_of_tile(c, tile, TR);
        s = load_seq(c, seq);
        row0 = (tile - first_tile(c, seq, TR)) * TR;
    }
    // the same for all lanes, whichever way they came
    split = __builtin_amdgcn_readfirstlane(split);
    seq = __builtin_amdgcn_readfirstlane(seq);
    row0 = __builtin_amdgcn_readfirstlane(row0);
    s = {__builtin_amdgcn_readfirstlane(s.q_begin), __builtin_amdgcn_readfirstlane(s.n_q), __builtin_amdgcn_readfirstlane(s.kv)};
    const uint32_t rows = (uint32_t)s.n_q * c.group;
    if (row0 >= rows) return;
    const uint32_t rows_here = min(rows - row0, (uint32_t)TR);

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const bool second = wave >= NW / 2;
    const uint32_t wave_row = wave * 32;
    const bool wave_live = wave_row < rows_here;
    const int32_t shift = s.kv - s.n_q;
    const uint32_t row = row0 + min(wave_row + col, rows_here - 1);   // rows past the end repeat the last one
    const int32_t token = (int32_t)token_of(c, row);
    const uint32_t head = kv_head * c.group + row - (uint32_t)token * c.group;
    // with a tree: what is said here of the keys that a row sees holds for those before the new tokens
    const bool tree = KIND != kCausal16 && a.tree;
    const int32_t limit = tree ? shift - 1 : min(shift + token, s.kv - 1);   // last key that this row sees
    const int64_t place = tree && a.window ? (int64_t)shift + tree_depth(a, s, token) : (int64_t)limit + 1;
    const int32_t floor_key = a.window ? (int32_t)max(place - (int64_t)a.window, (int64_t)0) : 0;

    const Split keys = keys_of(a, s, tree ? -1 : (int32_t)token_of(c, row0),
                               tree ? s.n_q - 1 : (int32_t)token_of(c, row0 + rows_here - 1), split, split_keys);
    if (a.uneven && keys.begin >= keys.end) {      // of no weight: its output is not looked at
        const uint64_t part = (uint64_t)split * c.total_q * c.heads + (uint64_t)(s.q_begin + token) * c.heads + head;
        if (half == 0 && wave_row + col < rows_here) *(v2f *)(a.part_ml + 2 * part) = v2f{kLowest, 0.0f};
        return;
    }
    const int32_t tiles_n = keys.end > keys.begin ? (keys.end - keys.begin + TK - 1) / TK : 0;
    // all of the wave's rows see the keys of [wave_full, wave_first]
    const int32_t wave_first = tree ? shift - 1 : shift + (int32_t)token_of(c, row0 + min(wave_row, rows_here - 1));
    const int32_t wave_last = !wave_live ? -1
                              : tree     ? shift + s.n_q - 1
                                         : shift + (int32_t)token_of(c, row0 + min(wave_row + 31, rows_here - 1));
    const int32_t wave_full = a.window ? (int32_t)max((int64_t)wave_last + 1 - (int64_t)a.window, (int64_t)0) : 0;

    // and all of the workgroup's rows those of [all_full, all_first]
    const int32_t all_first = tree ? shift - 1 : shift + (int32_t)token_of(c, row0);
    const int32_t all_last = shift + (tree ? s.n_q - 1 : (int32_t)token_of(c, row0 + rows_here - 1));
    const int32_t all_full = a.window ? (int32_t)max((int64_t)all_last + 1 - (int64_t)a.window, (int64_t)0) : 0;
    bool bounded = true;                             // the values of tiles that not all rows see are finite

    w4 q[DP / 16];
    {
        const uint16_t *p = a.q + (uint64_t)(s.q_begin + token) * a.q_stride + (uint64_t)head * c.head_dim;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const uint32_t at = 16 * i + 8 * half;
            q[i] = load16g(p + (at < c.head_dim ? at : 0));
            if (c.head_dim != DP && at >= c.head_dim) q[i] = w4{0, 0, 0, 0};
        }
    }
    v16f o[DP / 32], z[2];
    w4 p[4];                                         // weights of 16 keys each
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = v16f{};
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = w4{0, 0, 0, 0};
    float m = kLowest, l = 0.0f;

    // loading: thread -> row load_row + i * PASS of a tile, piece load_piece
    const int load_piece = tid % CH, load_row = tid / CH;
    const bool piece_live = (uint32_t)load_piece * 8 < c.head_dim;
    const Offset piece_at = piece_live ? load_piece * (E8 ? 8 : 16) : 0;
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    std::conditional_t<E8, w2, w4> rk[N], rv[N];     // 8 elements each
    uint32_t xk[XW], xv[XW];                         // exponents of this lane's key in 8-bit pages

    auto slot_at = [&](int32_t t) __attribute__((always_inline)) {   // table entry of this lane's key of tile t
        return load4g(table + block_of(c, min(keys.begin + t * TK + lane, keys.end - 1)));
    };
    auto row_at = [&](int32_t t, int32_t slot) __attribute__((always_inline)) {
        const int32_t key = keys.begin + t * TK + lane;
        return row_in<KIND>(c, key < keys.end ? slot : -1, kv_head, key);
    };
    // where a row begins, and the exponents of one in 8-bit pages; not there: a row that is
    auto offset_of = [&](uint32_t r, int32_t slot) __attribute__((always_inline)) {
        if constexpr (E8)
            return elements_at<Offset>(a, slot, r);
        else
            return (Offset)(r == kNoRow ? 0 : r) * (c.head_dim * 2);
    };
    auto exponents_of = [&](uint32_t r, int32_t slot) __attribute__((always_inline)) {
        if constexpr (E8)
            return exponents_at<Offset>(a, slot, r);
        else
            return (Offset)0;
    };
    auto load = [&](const uint16_t *cache, Offset at, auto (&to)[N]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint16_t *p = (const uint16_t *)((const char *)cache + (lane_value(at, load_row + i * PASS) + piece_at));
            if constexpr (E8)
                to[i] = load8g(p);
            else
                to[i] = load16g(p);
        }
    };
    auto load_exponents = [&](const uint16_t *cache, Offset at, uint32_t (&to)[XW]) __attribute__((always_inline)) {
        if constexpr (E8) {
#pragma unroll
            for (int w = 0; w < XW; ++w) to[w] = (uint32_t)load4g((const int32_t *)((const char *)cache + at) + w);
        }
    };
    // hands out the rows of what was loaded of 8-bit pages as 16-bit floats: all are widened first, or one after the other
    // where that does not fit the registers
    auto each_wide = [&](const auto &from, const uint32_t (&exponents)[XW], auto out) __attribute__((always_inline)) {
        w4 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t word = lane_value(exponents[0], load_row + i * PASS);
            if constexpr (XW > 1) {
                const uint32_t other = lane_value(exponents[1], load_row + i * PASS);
                word = load_piece >= 16 ? other : word;
            }
            x[i] = widen<T>(from[i], power_of(word, load_piece / 4 % 4 * 8));
            if constexpr (DP > 128) {
                out(i, x[i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (DP <= 128) {
#pragma unroll
            for (int i = 0; i < N; ++i) out(i, x[i]);
        }
    };
    // Rows of 64 elements lie two to 64 banks of LDS, longer ones fill them: the pieces of a row change places with
    // its number, so that 16 rows read at one place of K, and four at four places of V, meet different banks.  PASS
    // and the steps between the rows that a lane reads leave the number's low bits as they are: one place to a lane.
    auto k_place = [&](int r) __attribute__((always_inline)) { return DP >= 128 ? r & (PASS >= 16 ? 15 : 7) : (r >> 1) & 7; };
    auto v_place = [&](int r) __attribute__((always_inline)) { return DP >= 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2; };
    const uint32_t k_store = load_row * DP * 2 + (load_piece ^ k_place(load_row)) * 16;
    const uint32_t v_store = load_row * DP * 2 + (load_piece ^ v_place(load_row)) * 16;
    uint32_t k_read[DP / 16], v_read[DP / 32];
    {
        const int ti = lane & 15, r = 4 * half + ti / 4;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) k_read[i] = col * DP * 2 + ((2 * i + half) ^ k_place(col)) * 16;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
            v_read[i] = r * DP * 2 + ((4 * i + 2 * (lane >> 4 & 1) + (ti % 4) / 2) ^ v_place(r)) * 16 + (ti & 1) * 8;
    }
    auto store_k = [&](uint32_t buffer) __attribute__((always_inline)) {
        if constexpr (E8) {
            each_wide(rk, xk, [&](int i, w4 x) __attribute__((always_inline)) {
                if (__builtin_expect(c.head_dim != DP, 0) && !piece_live) x = w4{0, 0, 0, 0};
                *(w4 *)(lds + (k_store + buffer) + i * PASS * DP * 2) = x;
            });
        } else {
            if (__builtin_expect(c.head_dim != DP, 0) && !piece_live) {
#pragma unroll
                for (int i = 0; i < N; ++i) rk[i] = w4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < N; ++i) *(w4 *)(lds + (k_store + buffer) + i * PASS * DP * 2) = rk[i];
        }
    };
    auto store_v = [&](int32_t t, uint32_t buffer, uint64_t seen) __attribute__((always_inline)) {
        const int32_t k0 = keys.begin + t * TK;
        if constexpr (E8) {
            const bool edge = k0 + TK - 1 > all_first || k0 < all_full;
            each_wide(rv, xv, [&](int i, w4 x) __attribute__((always_inline)) {
                if (__builtin_expect(c.head_dim != DP || seen != ~0ull, 0))   // what is not there must be finite: its weight is 0
                    if (!piece_live || !(seen >> (load_row + i * PASS) & 1)) x = w4{0, 0, 0, 0};
                if (__builtin_expect(edge, 0)) bounded &= T::bound(x);
                *(w4 *)(lds + (v_store + buffer) + i * PASS * DP * 2) = x;
            });
        } else {
            if (__builtin_expect(c.head_dim != DP || seen != ~0ull, 0)) {
#pragma unroll
                for (int i = 0; i < N; ++i)          // what is not there must be finite: its weight is 0
                    if (!piece_live || !(seen >> (load_row + i * PASS) & 1)) rv[i] = w4{0, 0, 0, 0};
            }
            if (__builtin_expect(k0 + TK - 1 > all_first || k0 < all_full, 0)) {
#pragma unroll
                for (int i = 0; i < N; ++i) bounded &= T::bound(rv[i]);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) *(w4 *)(lds + (v_store + buffer) + i * PASS * DP * 2) = rv[i];
        }
    };

    auto product_k = [&](uint32_t buffer, int j) __attribute__((always_inline)) {
        const w4 k = *(const w4 *)(lds + k_read[j / 2] + (buffer + (j & 1) * 32 * DP * 2));
        z[j & 1] = T::mma32(k, q[j / 2], j < 2 ? v16f{} : z[j & 1]);
    };
    auto product_v = [&](uint32_t buffer, int j) __attribute__((always_inline)) {
        const int db = j % (DP / 32), i = j / (DP / 32);
        const char *v = lds + v_read[db] + (buffer + i * 16 * DP * 2);
        const w2 x = read_down((const uint16_t *)v), y = read_down((const uint16_t *)(v + 8 * DP * 2));
        o[db] = T::mma32(w4{x[0], x[1], y[0], y[1]}, p[i], o[db]);
    };
    // V(t - 1) and K(t): always both, so that the registers of o stay where they are.  Weights that are not there are
    // 0, and logits that are not there are not looked at.
    auto products = [&](uint32_t ks, uint32_t vs) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < DP / 8; ++j) product_v(vs, j);
#pragma unroll
        for (int j = 0; j < DP / 8; ++j) product_k(ks, j);
        __builtin_amdgcn_s_setprio(0);
    };
    auto softmax = [&](int32_t t, uint64_t seen) __attribute__((always_inline)) {
        const int32_t k0 = keys.begin + t * TK;
        if (__builtin_expect(!(k0 + TK - 1 <= wave_first && k0 >= wave_full && seen == ~0ull), 0)) {
            const uint64_t mine = seen >> (4 * half);
            const uint64_t drafted = tree ? (tree_bits(a, s, token, k0 - shift) & seen) >> (4 * half) : 0;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = kb * 32 + 8 * (r / 4) + r % 4;
                    const int32_t key = k0 + at + 4 * half;
                    bool sees = key <= limit && key >= floor_key && (mine >> at & 1);
                    if constexpr (KIND != kCausal16) sees |= drafted >> at & 1;
                    z[kb][r] = sees ? z[kb][r] : -INFINITY;
                }
        }
        float top = z[0][0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, z[0][r]);
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, z[1][r]);
        top = fmaxf(top, other_half(top)) * a.scale_log2;
        // m moves only when the maximum has passed it by 2^8, and then to the maximum: weights up to 2^8 lose nothing in
        // 32 bits, nor when rounded to 16 (their sum and the output keep the same factor), and rescaling becomes rare.
        // A 16-bit float ends at 2^-25, where weights would still be in the sum and no longer in the output, and has
        // room up to 2^16: m stays 2^7 below the maximum, so that weights run from 2^-32 of the largest to 2^15.
        if (__builtin_expect(__any(top > m + (8.0f + T::kLift)), 0)) {
            const float to = fmaxf(m, top - T::kLift);
            const float f = exp2_fast(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= f;
        }
        // The weights are rounded to the type of the values, as the matrix cores take them; their sum is not.
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 8 * (i & 1) + 2 * j;
                const float x = exp2_fast(__builtin_fmaf(z[i / 2][r], a.scale_log2, -m));
                const float y = exp2_fast(__builtin_fmaf(z[i / 2][r + 1], a.scale_log2, -m));
                l += x;
                l += y;
                p[i][j] = T::pack(x, y);
            }
    };

    if (tiles_n) {
        // which keys of tiles t to t + 2 are there; the first half of the waves does not use the last
        uint64_t seen0, seen1, seen2 = 0;
        const int32_t slot0 = slot_at(0), slot1 = slot_at(1);
        uint32_t r0 = row_at(0, slot0), r1 = row_at(1, slot1);
        int32_t slot = slot_at(2);
        seen0 = __ballot(r0 != kNoRow);
        seen1 = __ballot(r1 != kNoRow);
        Offset at_v = offset_of(r0, slot0), at_k = offset_of(r1, slot1);
        Offset exponents_v = exponents_of(r0, slot0), exponents_k = exponents_of(r1, slot1);
        load(a.k, at_v, rk);
        load(a.v, at_v, rv);
        load_exponents(a.k, exponents_v, xk);
        load_exponents(a.v, exponents_v, xv);
        store_k(0);
#pragma unroll
        for (int i = 0; i < N; ++i) *(w4 *)(lds + (v_store + 3 * BUF) + i * PASS * DP * 2) = w4{0, 0, 0, 0};   // "V(-1)"
        load(a.k, at_k, rk);
        load_exponents(a.k, exponents_k, xk);
        int32_t next = 2;                            // tile of the next K to load; slot is its table entry
        // stores the pair that was loaded to the buffers of parity odd and starts the next one's loads
        auto pass_on = [&](int32_t t, bool odd, uint64_t seen) __attribute__((always_inline)) {   // t: V's tile
            const uint32_t r = row_at(next, slot);   // before the loads: so that it does not wait for them
            at_v = at_k;
            at_k = offset_of(r, slot);
            exponents_v = exponents_k;
            exponents_k = exponents_of(r, slot);
            store_v(t, odd ? 3 * BUF : 2 * BUF, seen);
            store_k(odd ? 0 : BUF);
            load(a.v, at_v, rv);                     // past the last tile: some row
            load(a.k, at_k, rk);
            load_exponents(a.v, exponents_v, xv);
            load_exponents(a.k, exponents_k, xk);
            ++next;
            slot = slot_at(next);
            return __ballot(r != kNoRow);
        };
        if (second) seen2 = pass_on(0, false, seen0);
        __syncthreads();
        if (second) __syncthreads();
        auto iteration = [&](int32_t t, auto buffer) __attribute__((always_inline)) {
            constexpr int buf = decltype(buffer)::value;
            products(buf * BUF, (3 - buf) * BUF);
            __syncthreads();
            softmax(t, seen0);
            const uint64_t after = pass_on(second ? t + 1 : t, second != (buf == 1), second ? seen1 : seen0);
            seen0 = seen1;
            seen1 = second ? seen2 : after;
            seen2 = after;
            __syncthreads();
        };
        for (int32_t t = 0;; t += 2) {
            iteration(t, std::integral_constant<int, 0>());
            if (t + 1 >= tiles_n) break;
            iteration(t + 1, std::integral_constant<int, 1>());
            if (t + 2 >= tiles_n) break;
        }
        const uint32_t last = tiles_n & 1 ? 2 * BUF : 3 * BUF;
#pragma unroll
        for (int j = 0; j < DP / 8; ++j) product_v(last, j);
        if (!second) __syncthreads();                // the second half's last stage
        if (__builtin_expect(__syncthreads_or(!bounded), 0) && wave_live) {
            for (int32_t t = 0; t < tiles_n; ++t) {
                const int32_t k0 = keys.begin + t * TK;
                if (k0 + TK - 1 <= all_first && k0 >= all_full) continue;
                const int32_t key = k0 + lane;
                const uint32_t r = row_of(c, key < keys.end ? slot_at(t) : -1, kv_head, key);
                const bool found = r != kNoRow && unbounded_row<T, KIND>(a, r);
                const uint64_t drafted = tree ? tree_bits(a, s, token, k0 - shift) : 0;
                for (uint64_t left = __ballot(found); left; left &= left - 1) {
                    const int j = __ffsll((unsigned long long)left) - 1;
                    const uint32_t at = (uint32_t)__builtin_amdgcn_readlane(r, j);
                    const float weight = weight_of<T, KIND>(a, q, at, m, [&](int i) { return 16u * i + 8 * half; },
                                                            [](float x) { return x + other_half(x); });
                    if ((k0 + j > limit || k0 + j < floor_key) && !(drafted >> j & 1)) continue;
#pragma unroll
                    for (int i = 0; i < DP / 8; ++i) {
                        const uint32_t d = 8 * i + 4 * half;
                        if (d >= c.head_dim) continue;
                        const w2 v = four_at<T, KIND>(a, at, d);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[i / 4][4 * (i % 4) + e] += unbounded_part<T>(v, e, weight);
                    }
                }
            }
        }
    }

    if (!wave_live) return;
    const bool live = wave_row + col < rows_here;
    l += other_half(l);
    const uint64_t out_row = (uint64_t)(s.q_begin + token);
    if (a.splits == 1) {
        const RowEnd e = finish_row(m, l, a.sinks, head);
        if (!live) return;
        uint16_t *p = a.out + out_row * a.out_stride + (uint64_t)head * c.head_dim;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t at = db * 32 + 8 * j + 4 * half;
                if (at < c.head_dim)
                    *(w2 *)(p + at) = w2{T::pack(o[db][4 * j] * e.scale_o, o[db][4 * j + 1] * e.scale_o),
                                         T::pack(o[db][4 * j + 2] * e.scale_o, o[db][4 * j + 3] * e.scale_o)};
            }
        if (a.lse && half == 0) a.lse[(uint64_t)head * c.total_q + out_row] = e.lse;
    } else if (live) {
        const uint64_t part = (uint64_t)split * c.total_q * c.heads + out_row * c.heads + head;
        if (half == 0) *(v2f *)(a.part_ml + 2 * part) = v2f{m, l};
        float *p = a.part_o + part * c.head_dim;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t at = db * 32 + 8 * j + 4 * half;
                if (at < c.head_dim)
                    *(v4f *)(p + at) = v4f{o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]};
            }
    }
}

// ---- up to 16 rows, the waves split the keys

constexpr int kFewWaves = 4;
constexpr int kFewKeys = 32;    // to a wave at a time

// Bound by reading the cache: 16 KB in flight to a wave (head_dim 128), each loaded as soon as its registers are free.
// One token over 128K (64 heads, 8 KV heads, 64): 55 us with its join, 4.8 TB/s, where inputs change from call to call
// (41 and 5 on the same 268 MB again and again, part of which the cache behind L2 still holds); 32 tokens over ragged
// contexts of up to 16K (32, 8, 128): 190 us, 5.1 TB/s, where a copy moves 6.1.
// Short contexts are bound by what has to be known before the first key can be asked for, so the block table's
// entries are asked for together with the sequence's length wherever they do not depend on it.
// Two waves to a SIMD: three would have 168 registers, and what does not fit them costs more (276 us for those 32 tokens).
// Of 8-bit pages a lane's load is 16 elements and half the registers do, so there are three.  One token over 128K (32, 8, 128):
// 51.7 to 52.8 us by card with its join, 5.2 TB/s; 32 over ragged 16K 113 us, 4.4 TB/s (116 if the values, each line one load's, stay in the
// caches; 119 if keys go past them as well, whose lines are two loads').  64 keys at a time and two waves: 61 and 129.
template <class T, int DP, int KIND = kCausal16>
__global__ __launch_bounds__(kFewWaves * 64, KIND == kEight && DP <= 128 ? 3 : 2) void attention_few(const AttentionArgs a)
{
    constexpr bool E8 = KIND == kEight;
    constexpr int XW = E8 ? (DP + 127) / 128 : 1;    // words of exponents to a row of 8-bit pages
    constexpr int NW = kFewWaves, TK = kFewKeys;
    constexpr int EL = E8 ? 16 : 8;                  // elements of a load
    constexpr int CH = DP / EL;
    constexpr int PASS = 64 / CH;                    // rows that a wave loads at once
    constexpr int N = TK / PASS;
    constexpr int KS = DP / 32;
    // each wave's values, and at the end its part of the output: [wave][16 rows][DP] in 32 bits
    __shared__ __align__(16) uint16_t lds_v[NW][TK * DP];
    __shared__ float lds_ml[NW][2][16];
    static_assert(sizeof(lds_v) == NW * 16 * DP * sizeof(float), "the parts reuse the values' space");

    const CacheView &c = a.c;
    const uint32_t kv_head = blockIdx.x % c.kv_heads;
    const uint32_t rest = blockIdx.x / c.kv_heads;
    const uint32_t split = rest % a.splits;
    const uint32_t seq = rest / a.splits;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    int32_t slot0 = -1, slot1 = -1;                  // table entries of this lane's first two keys
    if (!a.window && c.max_kv) {
        const int64_t key = (int64_t)split * a.split_keys + wave * TK + (lane & 31);
        slot0 = load4g(table + block_of(c, (uint32_t)min(key, (int64_t)c.max_kv - 1)));
        slot1 = load4g(table + block_of(c, (uint32_t)min(key + NW * TK, (int64_t)c.max_kv - 1)));
    }
    const Seq s = load_seq(c, seq);
    const uint32_t rows = (uint32_t)s.n_q * c.group;   // at most 16
    if (!rows) return;

    const int col = lane & 15, quad = lane >> 4;
    const uint32_t row = min((uint32_t)col, rows - 1);
    const int32_t token = (int32_t)(row / c.group);
    const uint32_t head = kv_head * c.group + row % c.group;
    // with a tree: what is said here of the keys that a row sees holds for those before the new tokens
    const bool tree = KIND != kCausal16 && a.tree;
    const int32_t shift = s.kv - s.n_q;
    const int32_t limit = tree ? shift - 1 : min(shift + token, s.kv - 1);
    const int64_t place = tree && a.window ? (int64_t)shift + tree_depth(a, s, token) : (int64_t)limit + 1;
    const int32_t floor_key = a.window ? (int32_t)max(place - (int64_t)a.window, (int64_t)0) : 0;
    const Split keys = keys_of(a, s, tree ? -1 : 0, s.n_q - 1, split, a.split_keys);
    const int32_t all_first = tree ? shift - 1 : shift;   // last key that every row sees
    const int64_t all_full = a.window ? (int64_t)s.kv - (int64_t)a.window : 0;   // first key that every row sees

    // a product's 32 elements, 8 to a lane: neighbours, or for 8-bit pages those that two products' lanes load as 16
    auto element_of = [&](int i) __attribute__((always_inline)) {
        return E8 ? 64u * (i / 2) + 16 * quad + 8 * (i & 1) : 32u * i + 8 * quad;
    };
    w4 q[KS];
    {
        const uint16_t *p = a.q + (uint64_t)(s.q_begin + token) * a.q_stride + (uint64_t)head * c.head_dim;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const uint32_t at = element_of(i);
            q[i] = load16g(p + (at < c.head_dim ? at : 0));
            if (c.head_dim != DP && at >= c.head_dim) q[i] = w4{0, 0, 0, 0};
        }
    }
    v4f o[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i] = v4f{};
    float m = kLowest, l = 0.0f;

    const int load_piece = lane % CH, load_row = lane / CH;
    const bool piece_live = (uint32_t)load_piece * EL < c.head_dim;
    const uint32_t piece_at = piece_live ? load_piece * EL : 0;
    const int32_t mine = keys.begin + wave * TK;     // this wave's first keys; then every NW * TK
    const int32_t steps = keys.end > mine ? (keys.end - mine + NW * TK - 1) / (NW * TK) : 0;

    bool bounded = true;                             // the values of tiles that not all rows see are finite
    w4 rk[2][KS * 8 / EL], rv[N];
    uint32_t exponents[XW];                          // lane i: of key i, and lane i + 32 of value i
    uint32_t seen_next = 0;
    auto slot_at = [&](int32_t t) {
        const int32_t key = mine + t * (NW * TK) + (lane & 31);
        return load4g(table + block_of(c, min(key, keys.end - 1)));
    };
    auto load_tile = [&](int32_t t, int32_t slot) {
        const int32_t key = mine + t * (NW * TK) + (lane & 31);
        const uint32_t r = row_in<KIND>(c, key < keys.end ? slot : -1, kv_head, key);
        const uint32_t ok = (uint32_t)__ballot(r != kNoRow);
        if constexpr (E8) {
            const uint64_t at_row = elements_at<uint64_t>(a, slot, r);
            const uint8_t *x = (const uint8_t *)(lane < 32 ? a.k : a.v) + exponents_at<uint64_t>(a, slot, r);
#pragma unroll
            for (int w = 0; w < XW; ++w) exponents[w] = (uint32_t)load4g((const int32_t *)x + w);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint8_t *p = (const uint8_t *)a.k + lane_value(at_row, b * 16 + col);
#pragma unroll
                for (int i = 0; i < KS / 2; ++i) {
                    const uint32_t at = 64 * i + 16 * quad;
                    const uint8_t *from = p + (at < c.head_dim ? at : 0);   // past the end: q is 0 there
                    rk[b][i] = KS > 2 ? load16g_by8(from) : stream16g_by8(from);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                rv[i] = stream16g_by8((const uint8_t *)a.v + lane_value(at_row, load_row + i * PASS) + piece_at);
            return ok;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t from = __shfl(r, b * 16 + col);
            from = from == kNoRow ? 0 : from;
            const uint16_t *p = a.k + (uint64_t)from * c.head_dim;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint32_t at = 32 * i + 8 * quad;
                if constexpr (!E8) rk[b][i] = load16g(p + (at < c.head_dim ? at : 0));   // past the end: q is 0 there
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t from = __shfl(r, load_row + i * PASS);
            from = from == kNoRow ? 0 : from;
            rv[i] = load16g(a.v + (uint64_t)from * c.head_dim + piece_at);
        }
        return ok;
    };

    int32_t slot_next = -1;
    if (steps) {
        if (a.window) {
            slot0 = slot_at(0);
            slot1 = slot_at(1);
        }
        slot_next = slot1;
        loads_arrived();
        seen_next = load_tile(0, slot0);
    }
    uint16_t *vs = lds_v[wave];

    for (int32_t t = 0; t < steps; ++t) {
        const uint32_t seen = seen_next;
        const int32_t k0 = mine + t * (NW * TK);
        const bool edge = !(k0 + TK - 1 <= all_first && (int64_t)k0 >= all_full);   // not all rows see these keys
        const bool partial = edge || seen != ~0u || c.head_dim != DP;   // there may be values to leave out
        v4f z[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            z[b] = v4f{};
            uint32_t word[XW];
            if constexpr (E8) {
#pragma unroll
                for (int w = 0; w < XW; ++w) word[w] = lane_value(exponents[w], b * 16 + col);
            }
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                w4 k;
                if constexpr (E8) {
                    const w4 x = rk[b][i / 2];
                    const float power = power_of(word[i / 4 % XW], i / 2 % 2 * 16 + quad / 2 * 8);   // 32 elements: two quads
                    k = widen<T>(i & 1 ? w2{x[2], x[3]} : w2{x[0], x[1]}, power);
                } else {
                    k = rk[b][i];
                }
                if (E8 ? __builtin_expect(c.head_dim != DP, 0) && element_of(i) >= c.head_dim
                       : c.head_dim != DP && element_of(i) >= c.head_dim)
                    k = w4{0, 0, 0, 0};
                z[b] = T::mma16(k, q[i], z[b]);
            }
        }
        if constexpr (E8) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = load_row + i * PASS;
                uint32_t word = lane_value(exponents[0], 32 + r);
                if constexpr (XW > 1) {
                    const uint32_t other = lane_value(exponents[XW - 1], 32 + r);
                    word = load_piece >= 8 ? other : word;
                }
                const float power = power_of(word, load_piece / 2 % 4 * 8);
                w4 v[2] = {widen<T>(w2{rv[i][0], rv[i][1]}, power), widen<T>(w2{rv[i][2], rv[i][3]}, power)};
                if (__builtin_expect(partial, 0)) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (16u * load_piece + 8 * j >= c.head_dim || !(seen >> r & 1)) v[j] = w4{0, 0, 0, 0};
                        if (edge) bounded &= T::bound(v[j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *(w4 *)&vs[r * DP + ((2 * load_piece + j) ^ (DP >= 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2)) * 8] = v[j];
            }
        }
#pragma unroll
        for (int i = 0; i < (E8 ? 0 : N); ++i) {
            const int r = load_row + i * PASS;
            const bool there = piece_live && (seen >> r & 1);
            const int vp = load_piece ^ (DP >= 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2);
            w4 v = there ? rv[i] : w4{0, 0, 0, 0};
            if (__builtin_expect(edge, 0)) bounded &= T::bound(v);
            *(w4 *)&vs[r * DP + vp * 8] = v;
        }
        if (t + 1 < steps) {
            seen_next = load_tile(t + 1, slot_next);
            slot_next = slot_at(t + 2);
        }
        if (edge || seen != ~0u) {
            const uint32_t here = seen >> (4 * quad);
            const uint32_t drafted = tree ? ((uint32_t)tree_bits(a, s, token, k0 - shift) & seen) >> (4 * quad) : 0;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int32_t key = k0 + b * 16 + 4 * quad + r;
                    bool sees = key <= limit && key >= floor_key && (here >> (b * 16 + r) & 1);
                    if constexpr (KIND != kCausal16) sees |= drafted >> (b * 16 + r) & 1;
                    z[b][r] = sees ? z[b][r] : -INFINITY;
                }
        }
        float top = z[0][0];
#pragma unroll
        for (int r = 1; r < 4; ++r) top = fmaxf(top, z[0][r]);
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, z[1][r]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, other_half(top)) * a.scale_log2;
        if (__any(top > m + (8.0f + T::kLift))) {    // as in attention_rows
            const float to = fmaxf(m, top - T::kLift);
            const float f = exp2_fast(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= f;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                z[b][r] = exp2_fast(__builtin_fmaf(z[b][r], a.scale_log2, -m));
                l += z[b][r];
            }
        const w4 p = {T::pack(z[0][0], z[0][1]), T::pack(z[0][2], z[0][3]), T::pack(z[1][0], z[1][1]),
                      T::pack(z[1][2], z[1][3])};
        // the wave's own values: LDS keeps a wave's accesses in order
        wave_lds_order();
        const int r = 4 * quad + col / 4;
#pragma unroll
        for (int db = 0; db < DP / 16; ++db) {
            const int piece = db * 2 + (col % 4) / 2;
            const int at = (piece ^ (DP >= 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2)) * 8 + (col & 1) * 4;
            const w2 x = read_down(&vs[r * DP + at]), y = read_down(&vs[(r + 16) * DP + at]);
            o[db] = T::mma16(w4{x[0], x[1], y[0], y[1]}, p, o[db]);
        }
        wave_lds_order();
    }

    if (__builtin_expect(__any(!bounded), 0)) {
        for (int32_t t = 0; t < steps; ++t) {
            const int32_t k0 = mine + t * (NW * TK), key = k0 + (lane & 31);
            if (k0 + TK - 1 <= all_first && (int64_t)k0 >= all_full) continue;
            const uint32_t r = row_of(c, key < keys.end ? slot_at(t) : -1, kv_head, key);
            const bool found = r != kNoRow && unbounded_row<T, KIND>(a, r);
            const uint32_t drafted = tree ? (uint32_t)tree_bits(a, s, token, k0 - shift) : 0;
            for (uint32_t left = (uint32_t)__ballot(found); left; left &= left - 1) {
                const int j = __ffs(left) - 1;
                const uint32_t at = (uint32_t)__builtin_amdgcn_readlane(r, j);
                const float weight = weight_of<T, KIND>(a, q, at, m, element_of, [](float x) {
                    x += __shfl_xor(x, 16);
                    return x + other_half(x);
                });
                if ((k0 + j > limit || k0 + j < floor_key) && !(drafted >> j & 1)) continue;
#pragma unroll
                for (int db = 0; db < DP / 16; ++db) {
                    const uint32_t d = 16 * db + 4 * quad;
                    if (d >= c.head_dim) continue;
                    const w2 v = four_at<T, KIND>(a, at, d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[db][e] += unbounded_part<T>(v, e, weight);
                }
            }
        }
    }

    // join the waves: scale each part to the common maximum, then add
    l += __shfl_xor(l, 16);
    l += other_half(l);
    if (quad == 0) {
        lds_ml[wave][0][col] = m;
        lds_ml[wave][1][col] = l;
    }
    __syncthreads();
    float top = lds_ml[0][0][col];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, lds_ml[w][0][col]);
    const float f = exp2_fast(m - top);
    float *parts = (float *)&lds_v[0][0];
#pragma unroll
    for (int db = 0; db < DP / 16; ++db)
        *(v4f *)&parts[(wave * 16 + col) * DP + db * 16 + 4 * quad] =
            v4f{o[db][0] * f, o[db][1] * f, o[db][2] * f, o[db][3] * f};
    __syncthreads();
    for (uint32_t i = tid; i < rows * (DP / 4); i += NW * 64) {
        const uint32_t r = i / (DP / 4), at = i % (DP / 4) * 4;
        if (at >= c.head_dim) continue;
        v4f sum = *(v4f *)&parts[r * DP + at];
        float mm = lds_ml[0][0][r], ll = 0.0f;
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            sum += *(v4f *)&parts[(w * 16 + r) * DP + at];
            mm = fmaxf(mm, lds_ml[w][0][r]);
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) ll += lds_ml[w][1][r] * exp2_fast(lds_ml[w][0][r] - mm);
        const uint64_t out_row = (uint64_t)(s.q_begin + (int32_t)(r / c.group));
        const uint32_t h = kv_head * c.group + r % c.group;
        if (a.splits == 1) {
            const RowEnd e = finish_row(mm, ll, a.sinks, h);
            uint16_t *p = a.out + out_row * a.out_stride + (uint64_t)h * c.head_dim + at;
            *(w2 *)p = w2{T::pack(sum[0] * e.scale_o, sum[1] * e.scale_o), T::pack(sum[2] * e.scale_o, sum[3] * e.scale_o)};
            if (a.lse && at == 0) a.lse[(uint64_t)h * c.total_q + out_row] = e.lse;
        } else {
            const uint64_t part = (uint64_t)split * c.total_q * c.heads + out_row * c.heads + h;
            *(v4f *)(a.part_o + part * c.head_dim + at) = sum;
            if (at == 0) *(v2f *)(a.part_ml + 2 * part) = v2f{mm, ll};
        }
    }
}

// ---- up to 32 or 64 rows, the waves split the keys

// The rest-th part of the keys of a batch of up to 64 sequences: those that hold keys first, sequence by sequence, then the
// empty ones.  Workgroups begin in this order on one place of the chip after the other, whether they have work or not: with the
// empty ones between the others some CUs have two that work and some none (trees of 8 x 16 over up to 8K: 61 us, 50 in order).
struct Part {
    uint32_t seq, split;
    Seq s;
};
__device__ __forceinline__ Part part_of(const AttentionArgs &a, uint32_t rest, bool tree)
{
    const uint32_t lane = threadIdx.x & 63;
    Seq s = load_seq(a.c, min(lane, a.c.n_seq - 1));
    if (lane >= a.c.n_seq) s.n_q = 0;
    uint32_t span = 0;
    if (s.n_q) span = (uint32_t)max(s.kv - keys_of(a, s, tree ? -1 : 0, s.n_q - 1, 0, a.split_keys).begin, 0);
    const uint32_t parts = min((span + a.split_keys - 1) / a.split_keys, a.splits);   // of this lane's sequence that hold keys
    const uint32_t upto = sum_upto(parts), all = (uint32_t)__builtin_amdgcn_readlane(upto, 63);
    const uint32_t empty = s.n_q ? a.splits - parts : 0, empty_upto = sum_upto(empty);
    const bool held = rest < all;
    const uint32_t at = held ? rest : rest - all;
    const uint64_t found = __ballot((held ? upto : empty_upto) > at);
    if (!found) return {kNoTile, 0, s};
    const int who = __ffsll((unsigned long long)found) - 1;
    auto from = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane(x, who); };
    s = {(int32_t)from(s.q_begin), (int32_t)from(s.n_q), (int32_t)from(s.kv)};
    const uint32_t split = held ? at - (from(upto) - from(parts)) : from(parts) + at - (from(empty_upto) - from(empty));
    return {(uint32_t)who, split, s};
}

// Drafts of a few tokens, whose group's heads make 17 to 64 rows: attention_few with products of 32 rows.  A wave has 32
// rows and 32 keys at a time, which its lanes take from memory as the products want them; values pass through the wave's
// own part of LDS, to be read by columns.  With two groups of rows (RG) neighbouring waves load the same keys.
// Bound by reading the cache up to 32 rows: 8 drafts over 128K (32 heads, 8 KV heads, 128) 93 to 97 us by card, 5.5 to 5.8 TB/s
// with the join, in 8 bits 57 to 60, 4.6 to 4.9; trees of 8 x 16 over up to 8K 45 to 49 us, where workgroups of 64 rows in
// attention_rows took 175.  With 64 rows by the vector unit and each wave's own turn: 16 drafts over 128K in 8 bits 88 to 94 us;
// all 64 rows in one wave, without another wave on the SIMD to fill the gaps, took 153.
template <class T, int DP, int KIND, int RG>
__global__ __launch_bounds__(kFewWaves * RG * 64, DP > 128 ? 1 : 2) void attention_some(const AttentionArgs a)
{
    constexpr bool E8 = KIND == kEight;
    constexpr int XW = E8 ? (DP + 127) / 128 : 1;    // words of exponents to a row of 8-bit pages
    constexpr int NW = kFewWaves, TK = kFewKeys;
    constexpr int EL = E8 ? 16 : 8;                  // elements of a load
    constexpr int CH = DP / EL;
    constexpr int PASS = 64 / CH;                    // rows that a wave loads at once
    constexpr int N = TK / PASS;
    constexpr int KS = DP / 16;                      // products of a step with K, 8 elements to a lane
    constexpr int RS = DP + 4;                       // words of a row in the join: rows begin in different banks
    // each wave's values, and at the end its part of the output: [wave][rows][DP] in 32 bits
    constexpr int VB = NW * RG * TK * DP * 2, OB = NW * RG * 32 * RS * 4;
    __shared__ __align__(16) char lds[VB > OB ? VB : OB];
    __shared__ float lds_ml[NW][2][RG * 32];

    const CacheView &c = a.c;
    const uint32_t kv_head = blockIdx.x % c.kv_heads;
    const uint32_t rest = blockIdx.x / c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63, place = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave = place / RG, row0 = place % RG * 32;   // among the keys and among the rows
    const bool tree = a.tree;
    uint32_t split = rest % a.splits, seq = rest / a.splits;
    Seq s;
    if (a.splits > 1 && c.n_seq > 1 && c.n_seq <= 64) {
        const Part p = part_of(a, rest, tree);
        split = __builtin_amdgcn_readfirstlane(p.split);
        seq = __builtin_amdgcn_readfirstlane(p.seq);
        if (seq == kNoTile) return;
        s = {__builtin_amdgcn_readfirstlane(p.s.q_begin), __builtin_amdgcn_readfirstlane(p.s.n_q),
             __builtin_amdgcn_readfirstlane(p.s.kv)};
    } else {
        s = load_seq(c, seq);
    }
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    const uint32_t rows = (uint32_t)s.n_q * c.group;   // at most 32 RG
    if (!rows) return;
    const Split keys = keys_of(a, s, tree ? -1 : 0, s.n_q - 1, split, a.split_keys);
    if (a.splits > 1 && keys.begin >= keys.end) {      // of no weight: its output is not looked at
        for (uint32_t r = tid; r < rows; r += kFewWaves * RG * 64) {
            const uint32_t t = token_of(c, r), h = kv_head * c.group + r - t * c.group;
            const uint64_t part = (uint64_t)split * c.total_q * c.heads + ((uint64_t)s.q_begin + t) * c.heads + h;
            *(v2f *)(a.part_ml + 2 * part) = v2f{kLowest, 0.0f};
        }
        return;
    }

    const int col = lane & 31, half = lane >> 5;
    // with a tree: what is said here of the keys that a row sees holds for those before the new tokens
    const int32_t shift = s.kv - s.n_q;
    const uint32_t row = min((uint32_t)(row0 + col), rows - 1);
    const int32_t token = (int32_t)token_of(c, row);
    const uint32_t head = kv_head * c.group + row - (uint32_t)token * c.group;
    const int32_t limit = tree ? shift - 1 : min(shift + token, s.kv - 1);
    const int64_t end = tree && a.window ? (int64_t)shift + tree_depth(a, s, token) : (int64_t)limit + 1;
    const int32_t floor_key = a.window ? (int32_t)max(end - (int64_t)a.window, (int64_t)0) : 0;
    // a product's 16 elements, 8 to a lane: neighbours, or for 8-bit pages those that two products' lanes load as 16
    auto element_of = [&](int i) __attribute__((always_inline)) {
        return E8 ? 32u * (i / 2) + 16 * half + 8 * (i & 1) : 16u * i + 8 * half;
    };
    w4 q[KS];
    {
        const uint16_t *p = a.q + (uint64_t)(s.q_begin + token) * a.q_stride + (uint64_t)head * c.head_dim;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const uint32_t at = element_of(i);
            q[i] = load16g(p + (at < c.head_dim ? at : 0));
            if (c.head_dim != DP && at >= c.head_dim) q[i] = w4{0, 0, 0, 0};
        }
    }
    const int32_t all_first = tree ? shift - 1 : shift;   // last key that every row sees
    const int64_t all_full = a.window ? (int64_t)s.kv - (int64_t)a.window : 0;   // first key that every row sees

    v16f o[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = v16f{};
    float m = kLowest, l = 0.0f;

    const int load_piece = lane % CH, load_row = lane / CH;
    const bool piece_live = (uint32_t)load_piece * EL < c.head_dim;
    const uint32_t piece_at = piece_live ? load_piece * EL : 0;
    const int32_t mine = keys.begin + wave * TK;     // this wave's first keys; then every NW * TK
    const int32_t steps = keys.end > mine ? (keys.end - mine + NW * TK - 1) / (NW * TK) : 0;

    bool bounded = true;                             // the values of tiles that not all rows see are finite
    w4 rk[KS * 8 / EL], rv[N];
    uint32_t exponents[XW];                          // lane i: of key i, and lane i + 32 of value i
    uint32_t seen_next = 0;
    auto slot_at = [&](int32_t t) __attribute__((always_inline)) {
        const int32_t key = mine + t * (NW * TK) + col;
        return load4g(table + block_of(c, min(key, keys.end - 1)));
    };
    auto load_tile = [&](int32_t t, int32_t slot) __attribute__((always_inline)) {
        const int32_t key = mine + t * (NW * TK) + col;
        const uint32_t r = row_in<KIND>(c, key < keys.end ? slot : -1, kv_head, key);
        seen_next = (uint32_t)__ballot(r != kNoRow);
        uint64_t at_row;                             // bytes
        if constexpr (E8) {
            at_row = elements_at<uint64_t>(a, slot, r);
            const uint8_t *x = (const uint8_t *)(lane < 32 ? a.k : a.v) + exponents_at<uint64_t>(a, slot, r);
#pragma unroll
            for (int w = 0; w < XW; ++w) exponents[w] = (uint32_t)load4g((const int32_t *)x + w);
        } else {
            at_row = (uint64_t)(r == kNoRow ? 0 : r) * (c.head_dim * 2);
        }
        const uint8_t *p = (const uint8_t *)a.k + at_row;   // the lane's own key
#pragma unroll
        for (int i = 0; i < KS * 8 / EL; ++i) {
            const uint32_t at = E8 ? 32u * i + 16 * half : 16u * i + 8 * half;
            const uint8_t *from = p + (at < c.head_dim ? at : 0) * (E8 ? 1 : 2);   // past the end: q is 0 there
            rk[i] = E8 ? load16g_by8(from) : load16g((const uint16_t *)from);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {                // two waves' keys: the second's come from a cache
            const uint8_t *from = (const uint8_t *)a.v + lane_value(at_row, load_row + i * PASS) + piece_at * (E8 ? 1 : 2);
            if constexpr (E8)
                rv[i] = RG > 1 ? load16g_by8(from) : stream16g_by8(from);
            else
                rv[i] = RG > 1 ? load16g((const uint16_t *)from) : stream16g((const uint16_t *)from);
        }
    };
    char *vs = lds + place * (TK * DP * 2);
    auto v_place = [&](int r) __attribute__((always_inline)) { return DP >= 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2; };
    uint32_t v_read[DP / 32];
    {
        const int ti = lane & 15, r = 4 * half + ti / 4;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
            v_read[i] = r * DP * 2 + ((4 * i + 2 * (lane >> 4 & 1) + (ti % 4) / 2) ^ v_place(r)) * 16 + (ti & 1) * 8;
    }

    int32_t slot_next = -1;
    if (steps) {
        const int32_t slot0 = slot_at(0);
        slot_next = slot_at(1);
        loads_arrived();
        load_tile(0, slot0);
    }
    for (int32_t t = 0; t < steps; ++t) {
        const uint32_t seen = seen_next;
        const int32_t k0 = mine + t * (NW * TK);
        const bool edge = !(k0 + TK - 1 <= all_first && (int64_t)k0 >= all_full);   // not all rows see these keys
        v16f z{};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            w4 k;
            if constexpr (E8) {
                const w4 x = rk[i / 2];
                const uint32_t word = lane_value(exponents[i / 8], col);   // 32 elements: two products
                k = widen<T>(i & 1 ? w2{x[2], x[3]} : w2{x[0], x[1]}, power_of(word, i / 2 % 4 * 8));
            } else {
                k = rk[i];
            }
            if (c.head_dim != DP && element_of(i) >= c.head_dim) k = w4{0, 0, 0, 0};
            z = T::mma32(k, q[i], z);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = load_row + i * PASS;
            w4 v[EL / 8];
            if constexpr (E8) {
                uint32_t word = lane_value(exponents[0], 32 + r);
                if constexpr (XW > 1) {
                    const uint32_t other = lane_value(exponents[XW - 1], 32 + r);
                    word = load_piece >= 8 ? other : word;
                }
                const float power = power_of(word, load_piece / 2 % 4 * 8);
                v[0] = widen<T>(w2{rv[i][0], rv[i][1]}, power);
                v[EL / 8 - 1] = widen<T>(w2{rv[i][2], rv[i][3]}, power);
            } else {
                v[0] = rv[i];
            }
#pragma unroll
            for (int j = 0; j < EL / 8; ++j) {
                const bool there = (uint32_t)(EL * load_piece + 8 * j) < c.head_dim && (seen >> r & 1);
                if (!there) v[j] = w4{0, 0, 0, 0};
                if (__builtin_expect(edge, 0)) bounded &= T::bound(v[j]);
                *(w4 *)(vs + r * DP * 2 + (((EL / 8) * load_piece + j) ^ v_place(r)) * 16) = v[j];
            }
        }
        if (t + 1 < steps) {
            load_tile(t + 1, slot_next);
            slot_next = slot_at(t + 2);
        }
        w4 p[2];
        if (edge || seen != ~0u) {
            const uint32_t here = seen >> (4 * half);
            const uint32_t drafted = tree ? ((uint32_t)tree_bits(a, s, token, k0 - shift) & seen) >> (4 * half) : 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int at = 8 * (r / 4) + r % 4;
                const int32_t key = k0 + at + 4 * half;
                const bool sees = (key <= limit && key >= floor_key && (here >> at & 1)) || (drafted >> at & 1);
                z[r] = sees ? z[r] : -INFINITY;
            }
        }
        float top = z[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, z[r]);
        top = fmaxf(top, other_half(top)) * a.scale_log2;
        if (__any(top > m + (8.0f + T::kLift))) {   // as in attention_rows
            const float to = fmaxf(m, top - T::kLift);
            const float f = exp2_fast(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= f;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 8 * i + 2 * j;
                const float x = exp2_fast(__builtin_fmaf(z[r], a.scale_log2, -m));
                const float y = exp2_fast(__builtin_fmaf(z[r + 1], a.scale_log2, -m));
                l += x;
                l += y;
                p[i][j] = T::pack(x, y);
            }
        // the wave's own values: LDS keeps a wave's accesses in order
        wave_lds_order();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) {
                const char *v = vs + v_read[db] + i * 16 * DP * 2;
                const w2 x = read_down((const uint16_t *)v), y = read_down((const uint16_t *)(v + 8 * DP * 2));
                const w4 value = {x[0], x[1], y[0], y[1]};
                o[db] = T::mma32(value, p[i], o[db]);
            }
        wave_lds_order();
    }

    if (__builtin_expect(__any(!bounded), 0)) {
        for (int32_t t = 0; t < steps; ++t) {
            const int32_t k0 = mine + t * (NW * TK), key = k0 + col;
            if (k0 + TK - 1 <= all_first && (int64_t)k0 >= all_full) continue;
            const uint32_t r = row_of(c, key < keys.end ? slot_at(t) : -1, kv_head, key);
            const bool found = r != kNoRow && unbounded_row<T, KIND>(a, r);
            for (uint32_t left = (uint32_t)__ballot(found); left; left &= left - 1) {
                const int j = __ffs(left) - 1;
                const uint32_t at = (uint32_t)__builtin_amdgcn_readlane(r, j);
                const float weight = weight_of<T, KIND>(a, q, at, m, element_of,
                                                        [](float x) { return x + other_half(x); });
                const bool drafted = tree && (tree_bits(a, s, token, k0 + j - shift) & 1);
                if ((k0 + j > limit || k0 + j < floor_key) && !drafted) continue;
#pragma unroll
                for (int i = 0; i < DP / 8; ++i) {
                    const uint32_t d = 8 * i + 4 * half;
                    if (d >= c.head_dim) continue;
                    const w2 v = four_at<T, KIND>(a, at, d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i / 4][4 * (i % 4) + e] += unbounded_part<T>(v, e, weight);
                }
            }
        }
    }

    // join the waves: scale each part to the common maximum, then add
    l += other_half(l);
    if (half == 0) {
        lds_ml[wave][0][row0 + col] = m;
        lds_ml[wave][1][row0 + col] = l;
    }
    __syncthreads();
    float *parts = (float *)lds;
    float top = lds_ml[0][0][row0 + col];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, lds_ml[w][0][row0 + col]);
    const float f = exp2_fast(m - top);
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *(v4f *)&parts[(wave * RG * 32 + row0 + col) * RS + db * 32 + 8 * j + 4 * half] =
                v4f{o[db][4 * j] * f, o[db][4 * j + 1] * f, o[db][4 * j + 2] * f, o[db][4 * j + 3] * f};
    __syncthreads();
    for (uint32_t i = tid; i < rows * (DP / 4); i += NW * RG * 64) {
        const uint32_t r = i / (DP / 4), at = i % (DP / 4) * 4;
        if (at >= c.head_dim) continue;
        v4f sum = *(v4f *)&parts[r * RS + at];
        float mm = lds_ml[0][0][r], ll = 0.0f;
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            sum += *(v4f *)&parts[(w * RG * 32 + r) * RS + at];
            mm = fmaxf(mm, lds_ml[w][0][r]);
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) ll += lds_ml[w][1][r] * exp2_fast(lds_ml[w][0][r] - mm);
        const uint32_t t = token_of(c, r), h = kv_head * c.group + r - t * c.group;
        const uint64_t out_row = (uint64_t)s.q_begin + t;
        if (a.splits == 1) {
            const RowEnd e = finish_row(mm, ll, a.sinks, h);
            uint16_t *p = a.out + out_row * a.out_stride + (uint64_t)h * c.head_dim + at;
            *(w2 *)p = w2{T::pack(sum[0] * e.scale_o, sum[1] * e.scale_o), T::pack(sum[2] * e.scale_o, sum[3] * e.scale_o)};
            if (a.lse && at == 0) a.lse[(uint64_t)h * c.total_q + out_row] = e.lse;
        } else {
            const uint64_t part = (uint64_t)split * c.total_q * c.heads + out_row * c.heads + h;
            *(v4f *)(a.part_o + part * c.head_dim + at) = sum;
            if (at == 0) *(v2f *)(a.part_ml + 2 * part) = v2f{mm, ll};
        }
    }
}

template <class T, int DP, int KIND>
hipError_t rows_as(const AttentionArgs &a, hipStream_t stream)
{
    const uint32_t grid = a.tiles * a.splits * a.c.kv_heads;
    if ((uint64_t)a.c.num_slots * a.slot_bytes <= 0xFFFFFFFFull)
        attention_rows<T, DP, uint32_t, KIND><<<grid, row_waves(DP) * 64, 0, stream>>>(a);
    else
        attention_rows<T, DP, uint64_t, KIND><<<grid, row_waves(DP) * 64, 0, stream>>>(a);
    return hipGetLastError();
}

// Attention over pages of either kind: by the rows of a sequence and by head_dim.
template <class T, int DP, int KIND>
hipError_t by_rows(const AttentionArgs &a, hipStream_t stream)
{
    if (a.few_rows) {
        const uint32_t grid = a.tiles * a.splits * a.c.kv_heads;
        if (a.few_rows <= 16)
            attention_few<T, DP, KIND><<<grid, kFewWaves * 64, 0, stream>>>(a);
        else if (a.few_rows <= 32)
            attention_some<T, DP, KIND, 1><<<grid, kFewWaves * 64, 0, stream>>>(a);
        else if constexpr (some_rows(DP) > 32)
            attention_some<T, DP, KIND, 2><<<grid, kFewWaves * 128, 0, stream>>>(a);
        return hipGetLastError();
    }
    return rows_as<T, DP, KIND>(a, stream);
}
template <class T, int KIND>
hipError_t by_head_dim(const AttentionArgs &a, hipStream_t stream)
{
    if (a.c.head_dim <= 64) return by_rows<T, 64, KIND>(a, stream);
    if (a.c.head_dim <= 128) return by_rows<T, 128, KIND>(a, stream);
    return by_rows<T, 256, KIND>(a, stream);
}

}  // namespace

}  // namespace kvp

#endif
