// Attention of new tokens over the paged cache, for gfx950 (MI355X).
//
// For a new token i of a sequence at cache index c_i, a query head and its KV head:
//   S_j = scale * q_i . k_j   for the cached tokens j with c_i - window < j <= c_i
//   o_i = sum_j exp(S_j - lse_i) v_j,   lse_i = log(sum_j exp S_j + exp sink)
// in one pass over the keys, with a running maximum m and sum l per row (all in 32 bits; weights are
// exp2(S log2e - m log2e), so the exponential is one instruction).
//
// The rows of a KV head are its (new token, query head of the group) pairs, token-major: every key and
// value that is fetched serves the whole group.  The kernels compute S transposed, S^T = K Q^T: a lane
// then owns one row (column of the MFMA result), so maximum and sum are per-lane values, and the lane's
// results, rounded to 16 bits, already are the B operand of O^T = V^T P^T, with no exchange between lanes:
// the order of the keys inside a product is free, and V's transposed LDS reads follow the order that the
// first product left.
//
// attention_rows: 32 rows to a wave, 256 to a workgroup, kTileKeys keys at a time through LDS.
// attention_few: up to 16 rows (single tokens and very short chunks), where reading the cache is all that
// counts: the waves of a workgroup split the keys, and a join in LDS ends the workgroup.
// attention_some: the same for 17 to 64 rows, of drafts or over 8-bit pages.
// Where there are few row tiles all split the keys over workgroups as well; attention_join adds the parts.

#include "attention_kernels.hpp"

namespace kvp {

namespace {

// Adds the parts of the rows.  A row is the work of `slices` times LANES neighbouring threads: a thread has 4
// elements of head_dim and every slices-th part, U of them in flight; the slices are added through LDS, always in
// the same order.  SPARSE: parts without weight have no output to be asked for, which a look at their sums tells first.
template <class T, int LANES, int U, bool SPARSE>
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
    const int32_t end = load4g(c.cu_q + c.n_seq);
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
            if (!SPARSE) o[u] = *(const v4f *)(a.part_o + part * c.head_dim + (live ? at : 0));
        }
        if (SPARSE) {                                // many parts of short sequences are empty
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint64_t part = (uint64_t)min(i0 + u * slices, a.splits - 1) * rows + row;
                o[u] = v4f{};
                if (ml[u][1] != 0.0f) o[u] = *(const v4f *)(a.part_o + part * c.head_dim + (live ? at : 0));
            }
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
    if (blockIdx.x * (GROUPS / slices) + group / slices >= rows || (int32_t)token >= end) return;
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
        const uint32_t grid = (rows + per - 1) / per;
        if (a.uneven)
            attention_join<T, DP / 4, 4, true><<<grid, 256, 0, stream>>>(a, slices);
        else if (a.splits <= 2)
            attention_join<T, DP / 4, 2, false><<<grid, 256, 0, stream>>>(a, slices);
        else
            attention_join<T, DP / 4, 4, false><<<grid, 256, 0, stream>>>(a, slices);
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
