// Attention of new tokens over the paged cache, for gfx950 (MI355X).
//
// For a new token i of a sequence at cache index c_i, a query head and its KV head:
//   S_j = scale * q_i . k_j   for the cached tokens j with c_i - window < j <= c_i
//   o_i = sum_j exp(S_j - lse_i) v_j,   lse_i = log(sum_j exp S_j + exp sink)
// in one pass over the keys, with a running maximum m and sum l per row (all in 32 bits; weights are
// exp2(S log2e - m log2e), so the exponential is one instruction).
//
// The rows of a KV head are its (new token, query head of the group) pairs, token-major: every key and
// value that is fetched serves the whole group.  Both kernels compute S transposed, S^T = K Q^T: a lane
// then owns one row (column of the MFMA result), so maximum and sum are per-lane values, and the lane's
// results, rounded to 16 bits, already are the B operand of O^T = V^T P^T, with no exchange between lanes:
// the order of the keys inside a product is free, and V's transposed LDS reads follow the order that the
// first product left.
//
// attention_rows: 32 rows to a wave, 256 to a workgroup, kTileKeys keys at a time through LDS.
// attention_few: up to 16 rows (single tokens and very short chunks), where reading the cache is all that
// counts: the waves of a workgroup split the keys, and a join in LDS ends the workgroup.
// Where there are few row tiles both split the keys over workgroups as well; attention_join adds the parts.

#include <type_traits>

#include "wave.hpp"

namespace kvp {

namespace {

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
// Keys of one workgroup: what its rows can see, cut into the launch's parts.
__device__ __forceinline__ Split keys_of(const AttentionArgs &a, const Seq &s, int32_t first_token, int32_t last_token,
                                         uint32_t split)
{
    const int32_t shift = s.kv - s.n_q;
    int32_t lo = 0;
    if (a.window) lo = (int32_t)max((int64_t)0, (int64_t)(shift + first_token) + 1 - (int64_t)a.window);
    lo &= ~(int32_t)(kTileKeys - 1);
    const int32_t hi = min(shift + last_token + 1, s.kv);
    const int64_t begin = (int64_t)lo + (int64_t)split * a.split_keys;
    const int64_t end = split + 1 == a.splits ? (int64_t)hi : min((int64_t)hi, begin + (int64_t)a.split_keys);
    return {(int32_t)min(begin, (int64_t)max(hi, 0)), (int32_t)max(end, (int64_t)0)};
}

// A row must not meet the infinities and NaN of values that it does not see, but a weight of 0 times them is NaN, and in a
// product every row meets every value of a tile.  So both kernels look at the values of the tiles that not all of their
// rows see, and hand the product 0 in the place of those that are not finite.  Where there was one, these tiles are gone
// over once more before a row ends, key by key: what each row that sees such a key lacks of its output is added here.
// 256 new tokens over 64K (32 heads, 8 KV heads, 128) take 0.34 ms with an infinity among the newest values or without;
// going over all keys of the rows once more took 140 ms.

// The weight of key k in this lane's row: q[i] are the row's elements from + i * QSTEP to + 7, and add sums a value over the
// lanes that have the others.
template <class T, int Q, int QSTEP, class Add>
__device__ __forceinline__ float weight_of(const w4 (&q)[Q], uint32_t from, const uint16_t *k, uint32_t head_dim,
                                           float scale_log2, float m, Add add)
{
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        if (from + i * QSTEP >= head_dim) continue;
        const w4 y = load16g(k + from + i * QSTEP);
#pragma unroll
        for (int e = 0; e < 8; ++e) x = __builtin_fmaf(T::unpack(q[i][e / 2], e & 1), T::unpack(y[e / 2], e & 1), x);
    }
    return exp2_fast(__builtin_fmaf(add(x), scale_log2, -m));
}
// What a row lacks of element e of four: the products left out.
template <class T>
__device__ __forceinline__ float unbounded_part(w2 v, int e, float weight)
{
    const float x = T::unpack(v[e / 2], e & 1);
    return __builtin_isfinite(x) ? 0.0f : weight * x;
}
// Whether a value's row has an element that is not finite.
template <class T>
__device__ __forceinline__ bool unbounded_row(const uint16_t *v, uint32_t head_dim)
{
    bool all = true;
    for (uint32_t d = 0; d < head_dim; d += 8) all &= T::finite(load16g(v + d));
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
template <class T, int DP, class Offset>
__global__ __launch_bounds__(row_waves(DP) * 64, row_waves(DP) / 4) void attention_rows(const AttentionArgs a)
{
    constexpr int TK = kTileKeys, NW = row_waves(DP), TR = NW * 32;
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
    const uint32_t split = rest / a.tiles, rank = rest % a.tiles;
    uint32_t seq, row0;
    Seq s;
    if (c.n_seq > 1 && c.n_seq <= 64) {
        const Tile t = tile_by_length(c, rank, TR, TK);
        if (t.tile == kNoTile) return;
        seq = t.seq;
        s = t.s;
        row0 = t.tile * TR;
    } else {
        const uint32_t tile = a.tiles - 1 - rank;
        seq = seq_of_tile(c, tile, TR);
        s = load_seq(c, seq);
        row0 = (tile - first_tile(c, seq, TR)) * TR;
    }
    // the same for all lanes, whichever way they came
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
    const int32_t limit = min(shift + token, s.kv - 1);               // last key that this row sees
    const int32_t floor_key = a.window ? (int32_t)max((int64_t)limit + 1 - (int64_t)a.window, (int64_t)0) : 0;

    const Split keys = keys_of(a, s, (int32_t)token_of(c, row0), (int32_t)token_of(c, row0 + rows_here - 1), split);
    const int32_t tiles_n = keys.end > keys.begin ? (keys.end - keys.begin + TK - 1) / TK : 0;
    // all of the wave's rows see the keys of [wave_full, wave_first]
    const int32_t wave_first = shift + (int32_t)token_of(c, row0 + min(wave_row, rows_here - 1));
    const int32_t wave_last = wave_live ? shift + (int32_t)token_of(c, row0 + min(wave_row + 31, rows_here - 1)) : -1;
    const int32_t wave_full = a.window ? (int32_t)max((int64_t)wave_last + 1 - (int64_t)a.window, (int64_t)0) : 0;

    // and all of the workgroup's rows those of [all_full, all_first]
    const int32_t all_first = shift + (int32_t)token_of(c, row0);
    const int32_t all_last = shift + (int32_t)token_of(c, row0 + rows_here - 1);
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
    const Offset piece_at = piece_live ? load_piece * 16 : 0;
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    w4 rk[N], rv[N];

    auto slot_at = [&](int32_t t) __attribute__((always_inline)) {   // table entry of this lane's key of tile t
        return load4g(table + block_of(c, min(keys.begin + t * TK + lane, keys.end - 1)));
    };
    auto row_at = [&](int32_t t, int32_t slot) __attribute__((always_inline)) {
        const int32_t key = keys.begin + t * TK + lane;
        return row_of(c, key < keys.end ? slot : -1, kv_head, key);
    };
    auto offset_of = [&](uint32_t r) __attribute__((always_inline)) {
        return (Offset)(r == kNoRow ? 0 : r) * (c.head_dim * 2);     // not there: a row that is
    };
    auto load = [&](const uint16_t *cache, Offset at, w4 (&to)[N]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            to[i] = load16g((const uint16_t *)((const char *)cache + (lane_value(at, load_row + i * PASS) + piece_at)));
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
        if (__builtin_expect(c.head_dim != DP, 0) && !piece_live) {
#pragma unroll
            for (int i = 0; i < N; ++i) rk[i] = w4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < N; ++i) *(w4 *)(lds + (k_store + buffer) + i * PASS * DP * 2) = rk[i];
    };
    auto store_v = [&](int32_t t, uint32_t buffer, uint64_t seen) __attribute__((always_inline)) {
        if (__builtin_expect(c.head_dim != DP || seen != ~0ull, 0)) {
#pragma unroll
            for (int i = 0; i < N; ++i)              // what is not there must be finite: its weight is 0
                if (!piece_live || !(seen >> (load_row + i * PASS) & 1)) rv[i] = w4{0, 0, 0, 0};
        }
        const int32_t k0 = keys.begin + t * TK;
        if (__builtin_expect(k0 + TK - 1 > all_first || k0 < all_full, 0)) {
#pragma unroll
            for (int i = 0; i < N; ++i) bounded &= T::bound(rv[i]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) *(w4 *)(lds + (v_store + buffer) + i * PASS * DP * 2) = rv[i];
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
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = kb * 32 + 8 * (r / 4) + r % 4;
                    const int32_t key = k0 + at + 4 * half;
                    const bool sees = key <= limit && key >= floor_key && (mine >> at & 1);
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
        uint32_t r0 = row_at(0, slot_at(0)), r1 = row_at(1, slot_at(1));
        int32_t slot = slot_at(2);
        seen0 = __ballot(r0 != kNoRow);
        seen1 = __ballot(r1 != kNoRow);
        Offset at_v = offset_of(r0), at_k = offset_of(r1);
        load(a.k, at_v, rk);
        load(a.v, at_v, rv);
        store_k(0);
#pragma unroll
        for (int i = 0; i < N; ++i) *(w4 *)(lds + (v_store + 3 * BUF) + i * PASS * DP * 2) = w4{0, 0, 0, 0};   // "V(-1)"
        load(a.k, at_k, rk);
        int32_t next = 2;                            // tile of the next K to load; slot is its table entry
        // stores the pair that was loaded to the buffers of parity odd and starts the next one's loads
        auto pass_on = [&](int32_t t, bool odd, uint64_t seen) __attribute__((always_inline)) {   // t: V's tile
            const uint32_t r = row_at(next, slot);   // before the loads: so that it does not wait for them
            at_v = at_k;
            at_k = offset_of(r);
            store_v(t, odd ? 3 * BUF : 2 * BUF, seen);
            store_k(odd ? 0 : BUF);
            load(a.v, at_v, rv);                     // past the last tile: some row
            load(a.k, at_k, rk);
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
                const uint32_t r = row_at(t, slot_at(t));
                const bool found = r != kNoRow && unbounded_row<T>(a.v + (uint64_t)r * c.head_dim, c.head_dim);
                for (uint64_t left = __ballot(found); left; left &= left - 1) {
                    const int j = __ffsll((unsigned long long)left) - 1;
                    const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(r, j) * c.head_dim;
                    const float weight = weight_of<T, DP / 16, 16>(q, 8 * half, a.k + at, c.head_dim, a.scale_log2, m,
                                                                   [](float x) { return x + other_half(x); });
                    if (k0 + j > limit || k0 + j < floor_key) continue;
#pragma unroll
                    for (int i = 0; i < DP / 8; ++i) {
                        const uint32_t d = 8 * i + 4 * half;
                        if (d >= c.head_dim) continue;
                        const w2 v = load8g(a.v + at + d);
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
template <class T, int DP>
__global__ __launch_bounds__(kFewWaves * 64, 2) void attention_few(const AttentionArgs a)
{
    constexpr int NW = kFewWaves, TK = kFewKeys;
    constexpr int CH = DP / 8;
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
    const int32_t limit = min(s.kv - s.n_q + token, s.kv - 1);
    const int32_t floor_key = a.window ? (int32_t)max((int64_t)limit + 1 - (int64_t)a.window, (int64_t)0) : 0;
    const Split keys = keys_of(a, s, 0, s.n_q - 1, split);
    const int32_t all_first = s.kv - s.n_q;          // last key that every row sees
    const int64_t all_full = a.window ? (int64_t)s.kv - (int64_t)a.window : 0;   // first key that every row sees

    w4 q[KS];
    {
        const uint16_t *p = a.q + (uint64_t)(s.q_begin + token) * a.q_stride + (uint64_t)head * c.head_dim;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const uint32_t at = 32 * i + 8 * quad;
            q[i] = load16g(p + (at < c.head_dim ? at : 0));
            if (c.head_dim != DP && at >= c.head_dim) q[i] = w4{0, 0, 0, 0};
        }
    }
    v4f o[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i] = v4f{};
    float m = kLowest, l = 0.0f;

    const int load_piece = lane % CH, load_row = lane / CH;
    const bool piece_live = (uint32_t)load_piece * 8 < c.head_dim;
    const uint32_t piece_at = piece_live ? load_piece * 8 : 0;
    const int32_t mine = keys.begin + wave * TK;     // this wave's first keys; then every NW * TK
    const int32_t steps = keys.end > mine ? (keys.end - mine + NW * TK - 1) / (NW * TK) : 0;

    bool bounded = true;                             // the values of tiles that not all rows see are finite
    w4 rk[2][KS], rv[N];
    uint32_t seen_next = 0;
    auto slot_at = [&](int32_t t) {
        const int32_t key = mine + t * (NW * TK) + (lane & 31);
        return load4g(table + block_of(c, min(key, keys.end - 1)));
    };
    auto load_tile = [&](int32_t t, int32_t slot) {
        const int32_t key = mine + t * (NW * TK) + (lane & 31);
        const uint32_t r = row_of(c, key < keys.end ? slot : -1, kv_head, key);
        const uint32_t ok = (uint32_t)__ballot(r != kNoRow);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t from = __shfl(r, b * 16 + col);
            from = from == kNoRow ? 0 : from;
            const uint16_t *p = a.k + (uint64_t)from * c.head_dim;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint32_t at = 32 * i + 8 * quad;
                rk[b][i] = load16g(p + (at < c.head_dim ? at : 0));   // past the end: q is 0 there
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
        v4f z[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            z[b] = v4f{};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                w4 k = rk[b][i];
                if (c.head_dim != DP && 32u * i + 8 * quad >= c.head_dim) k = w4{0, 0, 0, 0};
                z[b] = T::mma16(k, q[i], z[b]);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
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
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int32_t key = k0 + b * 16 + 4 * quad + r;
                    const bool sees = key <= limit && key >= floor_key && (here >> (b * 16 + r) & 1);
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
            const bool found = r != kNoRow && unbounded_row<T>(a.v + (uint64_t)r * c.head_dim, c.head_dim);
            for (uint32_t left = (uint32_t)__ballot(found); left; left &= left - 1) {
                const int j = __ffs(left) - 1;
                const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(r, j) * c.head_dim;
                const float weight = weight_of<T, KS, 32>(q, 8 * quad, a.k + at, c.head_dim, a.scale_log2, m, [](float x) {
                    x += __shfl_xor(x, 16);
                    return x + other_half(x);
                });
                if (k0 + j > limit || k0 + j < floor_key) continue;
#pragma unroll
                for (int db = 0; db < DP / 16; ++db) {
                    const uint32_t d = 16 * db + 4 * quad;
                    if (d >= c.head_dim) continue;
                    const w2 v = load8g(a.v + at + d);
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

// Adds the parts of the rows.  A row is the work of `slices` times LANES neighbouring threads: a thread has 4
// elements of head_dim and every slices-th part, U of them in flight; the slices are added through LDS, always in
// the same order.
template <class T, int LANES, int U>
__global__ __launch_bounds__(256) void attention_join(const AttentionArgs a, const uint32_t slices)
{
    constexpr int GROUPS = 256 / LANES;
    __shared__ v4f lds_sum[256];
    __shared__ float lds_l[GROUPS], lds_m[GROUPS];
    const CacheView &c = a.c;
    const uint32_t rows = c.total_q * c.heads;
    const uint32_t group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const uint32_t slice = group % slices, at = lane * 4;
    const uint32_t row = min(blockIdx.x * (GROUPS / slices) + group / slices, rows - 1);
    const bool live = at < c.head_dim;
    // a part of a group's own threads at a time: its maximum and sum first, to rescale by
    float m = kLowest, l = 0.0f;
    v4f sum{};
    for (uint32_t i0 = slice; i0 < a.splits; i0 += U * slices) {
        v2f ml[U];
        v4f o[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t part = (uint64_t)min(i0 + u * slices, a.splits - 1) * rows + row;
            ml[u] = *(const v2f *)(a.part_ml + 2 * part);
            o[u] = *(const v4f *)(a.part_o + part * c.head_dim + (live ? at : 0));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = i0 + u * slices < a.splits && ml[u][1] != 0.0f;   // an empty part wrote no output
            const float to = there ? fmaxf(m, ml[u][0]) : m;
            const float f = exp2_fast(m - to), g = there ? exp2_fast(ml[u][0] - to) : 0.0f;
            m = to;
            l = l * f + (there ? ml[u][1] : 0.0f) * g;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = sum[j] * f + (there ? o[u][j] : 0.0f) * g;
        }
    }
    lds_sum[threadIdx.x] = sum;
    if (lane == 0) lds_m[group] = m, lds_l[group] = l;
    __syncthreads();
    if (slice) return;
    for (uint32_t i = 1; i < slices; ++i) {
        const float to = fmaxf(m, lds_m[group + i]);
        const float f = exp2_fast(m - to), g = exp2_fast(lds_m[group + i] - to);
        const v4f o = lds_sum[threadIdx.x + i * LANES];
        m = to;
        l = l * f + lds_l[group + i] * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = sum[j] * f + o[j] * g;
    }
    const uint32_t head = row % c.heads, token = row / c.heads;
    const RowEnd e = finish_row(m, l, a.sinks, head);
    if (blockIdx.x * (GROUPS / slices) + group / slices >= rows) return;
    if (live)
        *(w2 *)(a.out + (uint64_t)token * a.out_stride + (uint64_t)head * c.head_dim + at) =
            w2{T::pack(sum[0] * e.scale_o, sum[1] * e.scale_o), T::pack(sum[2] * e.scale_o, sum[3] * e.scale_o)};
    if (a.lse && lane == 0) a.lse[(uint64_t)head * c.total_q + token] = e.lse;
}

// ---- attention weight of the cached tokens

constexpr int kMassWaves = 4;
constexpr int kMassKeys = 64;                        // to a wave
constexpr int kMassRows = 64;                        // through LDS at a time

// One step of adding 2 D registers over the lanes: lanes with bit D set keep the upper half.
template <int D>
__device__ __forceinline__ void halve(float (&acc)[32], int lane)
{
    const bool up = lane & D;
#pragma unroll
    for (int r = 0; r < D; ++r) {
        const float low = acc[r], high = acc[r + D];
        acc[r] = (up ? high : low) + __shfl_xor(up ? low : high, D);
    }
}

// A wave holds 64 keys as the A operand and goes over the rows, which come through LDS for all waves: S^T again,
// so every lane adds up the weights of its own 32 keys, for one row of each 32, in a fixed order; the lanes are
// added at the end.  Bound by the vector unit: a difference, an exponential and a sum to a weight.  256 tokens over 128K
// (32 heads, 4 KV heads, 128): 321 us, 854 TFLOP/s.
template <class T, int DP>
__global__ __launch_bounds__(kMassWaves * 64, DP > 128 ? 1 : 2) void attention_mass(const MassArgs a)
{
    constexpr int CH = DP / 8, TK = kMassKeys, TR = kMassRows, NT = kMassWaves * 64;
    constexpr int PASS = NT / CH, N = TR / PASS;     // rows that the workgroup loads at once
    __shared__ __align__(16) uint16_t lds[kMassWaves * TK * DP];    // the keys at first, then two tiles of rows
    __shared__ float lds_lse[2][TR];
    static_assert(2 * TR <= kMassWaves * TK, "two tiles of rows fit the keys' space");

    const CacheView &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const uint32_t kv_head = blockIdx.x % c.kv_heads;
    const uint32_t tile = blockIdx.x / c.kv_heads;
    const uint32_t tiles = (c.max_kv + kMassWaves * TK - 1) / (kMassWaves * TK);
    const uint32_t seq = tile / tiles;
    const Seq s = load_seq(c, seq);
    const int32_t group_k0 = (int32_t)(tile % tiles * (kMassWaves * TK));
    if (group_k0 >= s.kv) return;
    const int32_t k0 = group_k0 + wave * TK;

    // rows that see some key of the workgroup
    const int32_t shift = s.kv - s.n_q;
    int32_t first = a.last ? max(0, s.n_q - (int32_t)min(a.last, 0x7FFFFFFFu)) : 0;
    first = max(first, group_k0 - shift);
    int32_t last = s.n_q - 1;
    if (a.window)
        last = (int32_t)min((int64_t)last, (int64_t)group_k0 + kMassWaves * TK - 1 + (int64_t)a.window - 1 - shift);
    const uint32_t row_begin = (uint32_t)max(first, 0) * c.group;
    const uint32_t row_end = last < first ? row_begin : (uint32_t)(last + 1) * c.group;
    if (row_begin == row_end) {                      // none: under a window, most of a long context
        const int32_t key = k0 + lane;
        const uint64_t to = ((uint64_t)seq * c.kv_heads + kv_head) * a.score_stride + key;
        if (key < s.kv) a.score_out[to] = a.score_in ? a.score_in[to] : 0.0f;
        return;
    }

    const int load_piece = tid % CH, load_row = tid / CH;
    const bool piece_live = (uint32_t)load_piece * 8 < c.head_dim;
    const uint32_t piece_at = piece_live ? load_piece * 8 : 0;
    // Where the heads of a group divide a tile, a thread's rows keep their heads from tile to tile and their places
    // move by a constant; else, and for the last rows, they are worked out.
    w4 rq[N];
    float r_lse = 0.0f;
    const uint16_t *q_at[N];
    const float *lse_at = a.lse;
    const bool steady = TR % c.group == 0;
    const uint64_t q_step = TR / c.group * a.q_stride;
    auto place_rows = [&](uint32_t r0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t row = min(r0 + load_row + i * PASS, row_end - 1), token = token_of(c, row);
            const uint32_t head = kv_head * c.group + row - token * c.group;
            q_at[i] = a.q + (uint64_t)(s.q_begin + token) * a.q_stride + (uint64_t)head * c.head_dim + piece_at;
        }
        const uint32_t row = min(r0 + (tid & (TR - 1)), row_end - 1), token = token_of(c, row);
        lse_at = a.lse + (uint64_t)(kv_head * c.group + row - token * c.group) * c.total_q + s.q_begin + token;
    };
    auto load_rows = [&](uint32_t r0) __attribute__((always_inline)) {
        if (r0 == row_begin || !steady || r0 + TR > row_end) {
            place_rows(r0);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) q_at[i] += q_step;
            lse_at += TR / c.group;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) rq[i] = load16g(q_at[i]);
        r_lse = *lse_at;
    };
    auto store_rows = [&](int buf, uint32_t r0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = load_row + i * PASS;
            const int qp = load_piece ^ (DP >= 128 ? r & 15 : (r >> 1) & 7);
            if (c.head_dim != DP && !piece_live) rq[i] = w4{0, 0, 0, 0};
            *(w4 *)&lds[(buf * TR + r) * DP + qp * 8] = rq[i];
        }
        // a row past the end, or without keys, gives no weight: exp2(-inf)
        if (tid < TR) lds_lse[buf][tid] = r0 + tid < row_end && r_lse != -INFINITY ? r_lse * kLog2e : INFINITY;
    };

    uint64_t seen = 0;
    w4 k[2][DP / 16];
    {
        constexpr int KPASS = 64 / CH;               // rows that a wave loads at once
        const int piece = lane % CH, load_key = lane / CH;
        const bool live = (uint32_t)piece * 8 < c.head_dim;
        const int32_t key = k0 + lane;
        const int32_t slot = load4g(c.table + (uint64_t)seq * c.table_stride + block_of(c, min(key, s.kv - 1)));
        const uint32_t r = row_of(c, key < s.kv ? slot : -1, kv_head, key);
        seen = __ballot(r != kNoRow);
        uint16_t *ks = lds + wave * TK * DP;
        w4 rk[TK / KPASS];
#pragma unroll
        for (int i = 0; i < TK / KPASS; ++i) {
            uint32_t from = __shfl(r, load_key + i * KPASS);
            from = from == kNoRow ? 0 : from;
            rk[i] = load16g(a.k + (uint64_t)from * c.head_dim + (live ? piece * 8 : 0));
        }
        load_rows(row_begin);
#pragma unroll
        for (int i = 0; i < TK / KPASS; ++i) {
            const int at = load_key + i * KPASS;
            const int kp = piece ^ (DP >= 128 ? at & 15 : (at >> 1) & 7);
            *(w4 *)&ks[at * DP + kp * 8] = live ? rk[i] : w4{0, 0, 0, 0};
        }
        __syncthreads();
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const int at = kb * 32 + col;
                const int kp = (2 * i + half) ^ (DP >= 128 ? at & 15 : (at >> 1) & 7);
                k[kb][i] = *(const w4 *)&ks[at * DP + kp * 8];
            }
        __syncthreads();
    }

    float acc[32];
#pragma unroll
    for (int r = 0; r < 32; ++r) acc[r] = 0.0f;
    store_rows(0, row_begin);
    loads_arrived();
    int buf = 0;
    for (uint32_t r0 = row_begin; r0 < row_end; r0 += TR, buf ^= 1) {
        if (r0 + TR < row_end) load_rows(r0 + TR);
        __syncthreads();                             // the rows are in LDS; everyone has left the tile before
        const int32_t t_first = (int32_t)token_of(c, r0), t_last = (int32_t)token_of(c, min(r0 + TR, row_end) - 1);
        const bool some = k0 < s.kv && k0 <= shift + t_last &&
                          (!a.window || (int64_t)k0 + TK - 1 > (int64_t)shift + t_first - a.window);
        const bool full = some && k0 + TK - 1 <= shift + t_first &&
                          (!a.window || (int64_t)k0 > (int64_t)shift + t_last - a.window);
        auto logits = [&](int rb, v16f (&z)[2]) __attribute__((always_inline)) {
            const int at = rb * 32 + col;
            z[0] = z[1] = v16f{};
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const int qp = (2 * i + half) ^ (DP >= 128 ? at & 15 : (at >> 1) & 7);
                const w4 q = *(const w4 *)&lds[(buf * TR + at) * DP + qp * 8];
                z[0] = T::mma32(k[0][i], q, z[0]);
                z[1] = T::mma32(k[1][i], q, z[1]);
            }
        };
        if (full) {
#pragma unroll
            for (int rb = 0; rb < TR / 32; ++rb) {
                v16f z[2];
                logits(rb, z);
                const float lse = lds_lse[buf][rb * 32 + col];
#pragma unroll
                for (int r = 0; r < 32; r += 8) {
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        w[i] = exp2_fast(__builtin_fmaf(z[(r + i) / 16][(r + i) % 16], a.scale_log2, -lse));
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[r + i] += w[i];
                }
                __builtin_amdgcn_sched_barrier(0);   // mixed, the blocks' logits do not fit the registers
            }
        } else if (some) {
            for (int rb = 0; rb < TR / 32; ++rb) {
                v16f z[2];
                logits(rb, z);
                const float lse = lds_lse[buf][rb * 32 + col];
                const int32_t limit = shift + (int32_t)token_of(c, r0 + rb * 32 + col);
                const int32_t floor_key = a.window ? (int32_t)max((int64_t)limit + 1 - (int64_t)a.window, (int64_t)0) : 0;
#pragma unroll
                for (int r = 0; r < 32; ++r) {
                    const int32_t key = k0 + 32 * (r / 16) + 8 * (r % 16 / 4) + r % 4 + 4 * half;
                    const bool sees = key <= limit && key >= floor_key;
                    const float z1 = sees ? __builtin_fmaf(z[r / 16][r % 16], a.scale_log2, -lse) : -INFINITY;
                    acc[r] += exp2_fast(z1);
                }
            }
        }
        if (r0 + TR < row_end) store_rows(buf ^ 1, r0 + TR);
    }

    // over the 32 lanes of each half: at every step a lane keeps half of its keys and gives the others away, so
    // that lane i ends with the sum of register i
    halve<16>(acc, lane);
    halve<8>(acc, lane);
    halve<4>(acc, lane);
    halve<2>(acc, lane);
    halve<1>(acc, lane);
    const int at = 32 * (col / 16) + 8 * (col % 16 / 4) + col % 4 + 4 * half;
    const int32_t key = k0 + at;
    if (key < s.kv) {
        const uint64_t to = ((uint64_t)seq * c.kv_heads + kv_head) * a.score_stride + key;
        const float sum = seen >> at & 1 ? acc[0] : 0.0f;            // an absent key may have been anything
        a.score_out[to] = (a.score_in ? a.score_in[to] : 0.0f) + sum;
    }
}

// Up to 16 rows: bound by reading the keys, which go from memory to the registers that the product takes them from.
// 8 tokens over 16K (32 heads, 8 KV heads, 128): 31 us, 4.2 TB/s where inputs change from call to call; 27 us on the
// same ones again, by way of LDS 31 to 34.
constexpr int kMassSteps = 4;                        // of 32 keys a wave

template <class T, int DP>
__global__ __launch_bounds__(kMassWaves * 64, 2) void attention_mass_few(const MassArgs a)
{
    constexpr int KS = DP / 32, NW = kMassWaves, S = kMassSteps;
    const CacheView &c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, quad = lane >> 4;
    const uint32_t kv_head = blockIdx.x % c.kv_heads;
    const uint32_t tile = blockIdx.x / c.kv_heads;
    const uint32_t tiles = (c.max_kv + NW * 32 * S - 1) / (NW * 32 * S);
    const uint32_t seq = tile / tiles;
    const uint32_t first_key = tile % tiles * (NW * 32 * S) + wave * 32;   // then every NW * 32
    int32_t slot[S];                                 // asked for before the sequence's length is known
#pragma unroll
    for (int t = 0; t < S; ++t)
        slot[t] = load4g(c.table + (uint64_t)seq * c.table_stride +
                         block_of(c, min(first_key + t * NW * 32 + (lane & 31), c.max_kv - 1)));
    const Seq s = load_seq(c, seq);
    if (first_key >= (uint32_t)s.kv) return;
    const uint32_t rows = (uint32_t)s.n_q * c.group;                       // at most 16
    const uint32_t row = rows ? min((uint32_t)col, rows - 1) : 0, token = token_of(c, row);
    const uint32_t head = kv_head * c.group + row - token * c.group;
    int32_t limit = -1;                              // a row past the end, not asked for or without keys: no weight,
    float lse = 0.0f;                                // whatever its query holds
    w4 q[KS];
    if (rows) {
        const uint16_t *p = a.q + (uint64_t)(s.q_begin + token) * a.q_stride + (uint64_t)head * c.head_dim;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const uint32_t at = 32 * i + 8 * quad;
            q[i] = load16g(p + (at < c.head_dim ? at : 0));
            if (c.head_dim != DP && at >= c.head_dim) q[i] = w4{0, 0, 0, 0};
        }
        const float x = a.lse[(uint64_t)head * c.total_q + s.q_begin + token];
        const bool asked = a.last == 0 || (uint32_t)s.n_q - token <= a.last;
        if ((uint32_t)col < rows && asked && x != -INFINITY) {
            limit = s.kv - s.n_q + (int32_t)token;
            lse = x * kLog2e;
        }
    } else {
#pragma unroll
        for (int i = 0; i < KS; ++i) q[i] = w4{0, 0, 0, 0};
    }
    const int64_t floor_key = a.window ? (int64_t)limit + 1 - (int64_t)a.window : 0;
    // the first key that any of the asked rows sees: in place of keys before it one row is read, again and again (a
    // branch around the loads would have every step wait for the next one's)
    const int64_t lowest = !rows ? s.kv
                           : a.window ? (int64_t)s.kv - (int64_t)min((uint32_t)s.n_q, a.last ? a.last : ~0u) + 1 - (int64_t)a.window
                                      : 0;
    uint32_t seen[S];
    w4 k[2][2][KS];
    auto load = [&](int t, w4 (&to)[2][KS]) __attribute__((always_inline)) {
        const uint32_t key = first_key + t * NW * 32 + (lane & 31);
        const bool asked = key < (uint32_t)s.kv && (int64_t)first_key + t * NW * 32 + 31 >= lowest;
        const uint32_t r = row_of(c, asked ? slot[t] : -1, kv_head, key);
        seen[t] = (uint32_t)__ballot(r != kNoRow);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t from = __shfl(r, b * 16 + col);
            from = from == kNoRow ? 0 : from;
            const uint16_t *p = a.k + (uint64_t)from * c.head_dim;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint32_t at = 32 * i + 8 * quad;
                to[b][i] = load16g(p + (at < c.head_dim ? at : 0));
            }
        }
    };
    load(0, k[0]);
#pragma unroll
    for (int t = 0; t < S; ++t) {
        if (t + 1 < S) load(t + 1, k[(t + 1) & 1]);
        const uint32_t k0 = first_key + t * NW * 32;
        float w[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            v4f z{};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                w4 x = k[t & 1][b][i];
                if (c.head_dim != DP && 32u * i + 8 * quad >= c.head_dim) x = w4{0, 0, 0, 0};
                z = T::mma16(x, q[i], z);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int32_t key = (int32_t)k0 + 16 * b + 4 * quad + r;
                const float x = key <= limit && key >= floor_key ? __builtin_fmaf(z[r], a.scale_log2, -lse) : -INFINITY;
                w[4 * b + r] = exp2_fast(x);
            }
        }
        // over the 16 rows: lanes with bit d keep the upper half of their keys; at the end both of a pair have the sum
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (col & 8 ? w[i + 4] : w[i]) + __shfl_xor(col & 8 ? w[i] : w[i + 4], 8);
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = (col & 4 ? w[i + 2] : w[i]) + __shfl_xor(col & 4 ? w[i] : w[i + 2], 4);
        w[0] = (col & 2 ? w[1] : w[0]) + __shfl_xor(col & 2 ? w[0] : w[1], 2);
        w[0] += __shfl_xor(w[0], 1);
        const int e = col >> 1, at = 16 * (e >> 2) + 4 * quad + (e & 3);
        if (!(col & 1) && k0 + at < (uint32_t)s.kv) {
            const uint64_t to = ((uint64_t)seq * c.kv_heads + kv_head) * a.score_stride + k0 + at;
            a.score_out[to] = (a.score_in ? a.score_in[to] : 0.0f) + (seen[t] >> at & 1 ? w[0] : 0.0f);
        }
    }
}

template <template <class, int> class Launch, class Args>
hipError_t by_type(uint32_t dtype, uint32_t head_dim, const Args &a, hipStream_t stream)
{
    if (dtype == KVP_BF16) {
        if (head_dim <= 64) return Launch<BF16, 64>::go(a, stream);
        if (head_dim <= 128) return Launch<BF16, 128>::go(a, stream);
        return Launch<BF16, 256>::go(a, stream);
    }
    if (head_dim <= 64) return Launch<F16, 64>::go(a, stream);
    if (head_dim <= 128) return Launch<F16, 128>::go(a, stream);
    return Launch<F16, 256>::go(a, stream);
}

template <class T, int DP>
struct Rows {
    static hipError_t go(const AttentionArgs &a, hipStream_t stream)
    {
        const uint32_t grid = a.tiles * a.splits * a.c.kv_heads;
        const uint64_t bytes = (uint64_t)a.c.num_slots * a.c.kv_heads * a.c.block * a.c.head_dim * 2;
        if (bytes <= 0xFFFFFFFFull)
            attention_rows<T, DP, uint32_t><<<grid, row_waves(DP) * 64, 0, stream>>>(a);
        else
            attention_rows<T, DP, uint64_t><<<grid, row_waves(DP) * 64, 0, stream>>>(a);
        return hipGetLastError();
    }
};
template <class T, int DP>
struct Few {
    static hipError_t go(const AttentionArgs &a, hipStream_t stream)
    {
        const uint32_t grid = a.tiles * a.splits * a.c.kv_heads;
        attention_few<T, DP><<<grid, kFewWaves * 64, 0, stream>>>(a);
        return hipGetLastError();
    }
};
template <class T, int DP>
struct Join {
    static hipError_t go(const AttentionArgs &a, hipStream_t stream)
    {
        constexpr uint32_t groups = 256 / (DP / 4);
        uint32_t slices = 1;
        while (slices < groups && slices * 4 < a.splits) slices *= 2;
        const uint32_t per = groups / slices, rows = a.c.total_q * a.c.heads;
        if (a.splits <= 2)
            attention_join<T, DP / 4, 2><<<(rows + per - 1) / per, 256, 0, stream>>>(a, slices);
        else
            attention_join<T, DP / 4, 4><<<(rows + per - 1) / per, 256, 0, stream>>>(a, slices);
        return hipGetLastError();
    }
};
template <class T, int DP>
struct Mass {
    static hipError_t go(const MassArgs &a, hipStream_t stream)
    {
        if ((uint64_t)a.c.max_q * a.c.group <= kFewRows) {
            const uint32_t tiles = (a.c.max_kv + kMassWaves * 32 * kMassSteps - 1) / (kMassWaves * 32 * kMassSteps);
            attention_mass_few<T, DP><<<tiles * a.c.n_seq * a.c.kv_heads, kMassWaves * 64, 0, stream>>>(a);
            return hipGetLastError();
        }
        const uint32_t tiles = (a.c.max_kv + kMassWaves * kMassKeys - 1) / (kMassWaves * kMassKeys);
        attention_mass<T, DP><<<tiles * a.c.n_seq * a.c.kv_heads, kMassWaves * 64, 0, stream>>>(a);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_attention(const AttentionArgs &a, uint32_t dtype, hipStream_t stream)
{
    return a.few_rows ? by_type<Few>(dtype, a.c.head_dim, a, stream) : by_type<Rows>(dtype, a.c.head_dim, a, stream);
}

hipError_t launch_attention_join(const AttentionArgs &a, uint32_t dtype, hipStream_t stream)
{
    return by_type<Join>(dtype, a.c.head_dim, a, stream);
}

hipError_t launch_mass(const MassArgs &a, uint32_t dtype, hipStream_t stream)
{
    return by_type<Mass>(dtype, a.c.head_dim, a, stream);
}

}  // namespace kvp
