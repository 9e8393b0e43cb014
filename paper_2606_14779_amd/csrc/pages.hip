// New tokens into pages of either kind, pages from one kind to the other, accepted drafts moved together, for gfx950
// (MI355X).
//
// append: a head x of the queries or keys becomes
//   y = x / sqrt(mean(x^2) + eps) * w           (where there is a norm)
//   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin) for the pairs of its first `rot` elements, by the angle that the
//   table has for the pair and the token's position on the pair's axis
// in 32 bits, and is rounded once: to 16 bits, or to e4m3 with the least power of two that holds 32 elements.
// A head is the work of 2^lanes_log2 neighbouring lanes with 8 elements each, so that sums of squares and largest
// elements are exchanges within a wave.  Queries, keys and values are read once and written once.
//
// Bound by memory and by what a token has to wait for: packed prompts of 12.7K tokens (64 heads, 8 KV heads, 64; norms, three
// axes, pairs interleaved, 16-bit pages) 55.5 to 59.5 us by card, 263 MB at 4.7 TB/s, vector unit busy for 57 % of the cycles.  With every
// head's weights and angles worked out anew 73; with the token's positions, sequence and slot asked for one after the other
// 65.  A decoding step of 32 tokens takes 6.5 us on the GPU.  Tokens of few heads (8 heads, 1 KV head, 128) take 27 us for
// 66 MB, as a workgroup's chain of loads is paid for 4 KB; pairs that lie anyhow (24 heads, 8 KV heads, 80, half of them
// turned) 110 for 159 MB, by their partners' loads of two bytes.

#include <algorithm>
#include <type_traits>

#include "e4m3.hpp"

namespace kvp {

namespace {

__device__ __forceinline__ float largest_of(const float (&x)[8])
{
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_isfinite(x[i]) ? __builtin_fabsf(x[i]) : 0.0f);
    return top;
}

// Another lane's value within the vector unit: the neighbour's, that of the other pair of four, of the mirrored four of
// eight, of the mirrored eight of sixteen.
constexpr int kNeighbour = 0xB1, kOtherPair = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
template <int WHICH>
__device__ __forceinline__ float lane_of(float x)
{
    const int v = __builtin_bit_cast(int, x);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, WHICH, 0xF, 0xF, true));
}

// Over the lanes of a row, or the four lanes of 32 elements.  Once four lanes agree, a mirror is as good as an exchange.
template <class F>
__device__ __forceinline__ float over(float x, uint32_t lanes, F f)
{
    if (lanes > 1) x = f(x, lane_of<kNeighbour>(x));
    if (lanes > 2) x = f(x, lane_of<kOtherPair>(x));
    if (lanes > 4) x = f(x, lane_of<kHalfMirror>(x));
    if (lanes > 8) x = f(x, lane_of<kMirror>(x));
    if (lanes > 16) x = f(x, __shfl_xor(x, 16));
    return x;
}
__device__ __forceinline__ float sum_over(float x, uint32_t lanes)
{
    return over(x, lanes, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float largest_over(float x, uint32_t lanes)
{
    return over(x, lanes, [](float a, float b) { return fmaxf(a, b); });
}

// The word of a row's first four exponents (or of each 16 lanes' four) in its first lane, where every fourth lane has one.
__device__ __forceinline__ uint32_t gather_bytes(uint32_t byte, uint32_t lanes_log2)
{
    uint32_t word = byte;
    if (lanes_log2 > 2) word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x104, 0xF, 0xF, true) << 8;   // 4 lanes on
    if (lanes_log2 > 3) {
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x108, 0xF, 0xF, true) << 16;
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x10C, 0xF, 0xF, true) << 24;
    }
    return word;
}

template <class T>
__device__ __forceinline__ void unpack8(w4 w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = T::unpack(w[i / 2], i & 1);
}
template <class T>
__device__ __forceinline__ w4 pack8(const float (&x)[8])
{
    return w4{T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7])};
}

// Where a token of a KV head lies in a slot of 8-bit pages; `row` counts the slot's rows.
__device__ __forceinline__ uint32_t row_in_slot(const CacheView &c, uint32_t kv_head, uint32_t token)
{
    return kv_head * c.block + token - block_of(c, token) * c.block;
}

// 8 elements of a row of 8-bit pages, from all lanes of a row together; those with `asked` write, to the slot `to`.
template <class T>
__device__ __forceinline__ void put8(const PageView &p, uint32_t head_dim, uint8_t *to, bool asked, uint32_t row, uint32_t piece,
                                     uint32_t lanes_log2, const float (&x)[8])
{
    // the largest |x| as an integer, which has the order of the floats: from 0x7F800000 on there is one that is not finite
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu);
    const bool live = piece * 8 < head_dim;
    if (!live) top = 0;
    const uint32_t group = min(1u << lanes_log2, 4u);
    float largest = __builtin_bit_cast(float, top);
    bool plain = top < 0x7F800000u;
    if (!plain) largest = largest_of(x);             // of the finite ones
    largest = largest_over(largest, group);
    const int32_t e = exponent_for<T>(largest);
    plain &= e < E4M3<T>::kMost;
    uint32_t word = live ? (uint32_t)(e + 127) : 0;
    word = gather_bytes(word, lanes_log2);
    const w2 out = __builtin_expect(__all(plain), 1) ? narrow_plain(x, e) : narrow<T>(x, e);
    if (!asked) return;
    *(w2 *)(to + (uint64_t)row * head_dim + piece * 8) = out;
    if (piece % 16 == 0) *(uint32_t *)(to + p.exponents + (uint64_t)row * p.row_exponents + piece / 16 * 4) = word;
}

// How the pairs lie: both in the 8 elements of a lane, in two lanes, or anyhow.
enum Pairs { kInside, kApart, kAnyhow };

// The norm's factor of a head whose lanes hold x.  Where the squares leave the range of 32 bits (as bf16's may) and eps does
// not make up for it, x and its partners y are scaled by a power of two first: what `up` says.
template <class T>
__device__ __forceinline__ float norm_factor(const AppendArgs &a, float (&x)[8], float (&y)[8], uint32_t lanes, float &up)
{
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
    sum = sum_over(sum, lanes);
    up = 1.0f;
    const bool fits = sum < 1e36f && (sum > 1e-30f || a.eps > 1e-20f);
    float mean = __builtin_fmaf(sum, a.per_dim, a.eps);
    if (__builtin_expect(__any(!fits), 0)) {
        const float top = largest_over(largest_of(x), lanes);
        if (!fits && top > 0.0f) up = top > 1.0f ? 0x1p-96f : 0x1p96f;   // squares from 2^-74 to 2^92
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= up;
            y[i] *= up;
            s = __builtin_fmaf(x[i], x[i], s);
        }
        s = sum_over(s, lanes);
        if (up != 1.0f) mean = __builtin_fmaf(s, a.per_dim, a.eps * up * up);
    }
    return __builtin_amdgcn_rsqf(mean);
}

// A token to a workgroup.  A wave takes whole heads of one kind (queries, keys or values) at a time, so that its lanes go
// one way, and a lane the same eight elements of every head: what an element and its partner are multiplied by, weight and
// angle in one, is worked out once for all heads.
template <class T, bool E8, int PAIRS>
__global__ __launch_bounds__(256) void append(const AppendArgs a)
{
    enum Kind { kQueries, kKeys, kValues };
    __shared__ v2f angles[kMostRotary / 2];          // of this token
    const CacheView &c = a.c;
    const uint32_t token = blockIdx.x, lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t lanes = 1u << a.lanes_log2, per_wave = 64 >> a.lanes_log2;
    const uint32_t piece = lane & (lanes - 1), at = piece * 8, mine = lane >> a.lanes_log2;
    const bool live = at < c.head_dim;
    const uint32_t jobs_log2 = 6 - a.lanes_log2;
    const uint32_t q_jobs = a.q ? (c.heads + per_wave - 1) >> jobs_log2 : 0;
    const uint32_t k_jobs = (c.kv_heads + per_wave - 1) >> jobs_log2;
    const uint16_t *q = a.q + token * a.q_stride, *k = a.k + token * a.k_stride, *v = a.v + token * a.v_stride;

    auto load = [&](auto kind, uint32_t job) __attribute__((always_inline)) {
        constexpr int what = decltype(kind)::value;
        const uint32_t head = job * per_wave + mine;
        const uint16_t *from = what == kQueries ? q : what == kKeys ? k : v;
        return live && head < (what == kQueries ? c.heads : c.kv_heads) ? load16g(from + (uint64_t)(head * c.head_dim + at))
                                                                        : w4{0, 0, 0, 0};
    };
    // jobs go round the waves, queries, then keys, then values; the first of each kind are asked for before all else
    typedef std::integral_constant<int, kQueries> Queries;
    typedef std::integral_constant<int, kKeys> Keys;
    typedef std::integral_constant<int, kValues> Values;
    const uint32_t first_k = (wave - q_jobs) & (waves - 1), first_v = (first_k - k_jobs) & (waves - 1);   // 1, 2 or 4 waves
    w4 ahead_q{}, ahead_k{}, ahead_v{};
    if (wave < q_jobs) ahead_q = load(Queries(), wave);
    if (first_k < k_jobs) ahead_k = load(Keys(), first_k);
    if (first_v < k_jobs) ahead_v = load(Values(), first_v);
    // and what they are multiplied by, with their partners' in the other half of the pairs
    const uint32_t half = a.rot / 2;
    const bool turns = at < a.rot, upper = at >= half;
    const uint32_t partner = upper ? at - half : at + half;
    w4 weight[2]{}, weight_of_partner[2]{};
    auto load_weights = [&](int kind, const uint16_t *from) __attribute__((always_inline)) {
        if (!from || !live) return;
        weight[kind] = load16g(from + at);
        if (PAIRS == kApart && turns) weight_of_partner[kind] = load16g(from + partner);
    };
    if (wave < q_jobs) load_weights(0, a.q_weight);
    if (first_k < k_jobs) load_weights(1, a.k_weight);

    // Then what has to be known of the token: few loads one after the other, as they are most of a token's time.
    int32_t position[kMostAxes];
#pragma unroll
    for (uint32_t i = 0; i < kMostAxes; ++i) position[i] = load4g(a.positions + (uint64_t)min(i, a.axes - 1) * c.total_q + token);
    const uint32_t my_axis = a.axes > 1 && threadIdx.x < half ? a.axis_of[threadIdx.x] : 0;
    // its sequence: the last one that begins at or before it, 64 at a time
    Seq s;
    uint32_t seq = 0;
    if (c.n_seq <= 64) {
        const Seq its = load_seq(c, min(lane, c.n_seq - 1));
        const uint64_t begun = __ballot(lane < c.n_seq && its.q_begin <= (int32_t)token);
        seq = begun ? 63 - __builtin_clzll(begun) : 0;
        s = {__builtin_amdgcn_readlane(its.q_begin, seq), __builtin_amdgcn_readlane(its.n_q, seq),
             __builtin_amdgcn_readlane(its.kv, seq)};
    } else {
        for (uint32_t n = c.n_seq; n > 1;) {
            const uint32_t step = (n + 63) / 64, first = seq + lane * step;
            const uint32_t count = __popcll(__ballot(lane * step < n && load4g(c.cu_q + min(first, c.n_seq)) <= (int32_t)token));
            const uint32_t last = count ? count - 1 : 0;
            seq += last * step;
            n = min(step, n - last * step);
        }
        s = load_seq(c, seq);
    }
    const int32_t i = (int32_t)token - s.q_begin, index = s.kv - s.n_q + i;
    if (i < 0 || i >= s.n_q) return;                 // behind the last sequence
    const bool placed = index >= 0;
    const int32_t slot = placed ? load4g(c.table + (uint64_t)seq * c.table_stride + block_of(c, index)) : -1;
    // a position that the table does not have: NaN, so that it shows
    bool known = true;
#pragma unroll
    for (uint32_t i = 0; i < kMostAxes; ++i) known &= position[i] >= 0 && (uint32_t)position[i] < a.n_positions;
    for (uint32_t j = threadIdx.x; j < half; j += blockDim.x) {
        const uint32_t axis = j == threadIdx.x ? my_axis : a.axis_of[j];
        const int32_t p = axis < 2 ? axis ? position[1] : position[0] : axis == 2 ? position[2] : position[3];
        angles[j] = *(const v2f *)(a.angles + (uint64_t)(uint32_t)(known ? p : 0) * a.rot + 2 * j);
    }
    const bool there = (uint32_t)slot < c.num_slots;
    const uint64_t slot_at = there ? (uint64_t)(uint32_t)slot * a.pages.slot_bytes : 0;
    __syncthreads();

    // factors of the lane's elements and of their partners
    float p[8], r[8];
    auto factors = [&](int kind, bool weighted) __attribute__((always_inline)) {
        float w[8], o[8];
        unpack8<T>(weight[kind], w);
        unpack8<T>(weight_of_partner[kind], o);
        if (!weighted) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = o[e] = 1.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = known ? w[e] : __builtin_nanf("");
            r[e] = 0.0f;
            if (PAIRS == kAnyhow || !turns) continue;
            const v2f f = angles[PAIRS == kInside ? (at + e) / 2 : at + e - (upper ? half : 0)];
            const float other = PAIRS == kInside ? w[e ^ 1] : o[e];
            const bool second = PAIRS == kInside ? e & 1 : upper;
            p[e] *= f[0];
            r[e] = second ? other * f[1] : -(other * f[1]);
        }
    };
    auto process = [&](auto kind, uint32_t job, w4 raw) __attribute__((always_inline)) {
        constexpr bool query = decltype(kind)::value == kQueries, value = decltype(kind)::value == kValues;
        const uint32_t head = job * per_wave + mine;
        const bool asked = live && head < (query ? c.heads : c.kv_heads);
        float x[8];
        if (E8 || !value) unpack8<T>(raw, x);
        if (!value) {
            float y[8] = {}, up = 1.0f, factor = 1.0f;
            if constexpr (PAIRS == kApart) {
                const int other = (int)(lane + (upper ? -half / 8 : half / 8)) & 63;
                w4 far;
#pragma unroll
                for (int w = 0; w < 4; ++w) far[w] = __shfl(raw[w], other);
                unpack8<T>(far, y);
            }
            if (a.norm) {                            // before the weight, as their product stays within 32 bits then
                factor = norm_factor<T>(a, x, y, lanes, up);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] *= factor;
                    if constexpr (PAIRS == kApart) y[e] *= factor;
                }
            }
            if constexpr (PAIRS == kInside) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
            }
            if constexpr (PAIRS == kAnyhow) {
                const uint16_t *from = (query ? q : k) + (uint64_t)(head * c.head_dim), *weight = query ? a.q_weight : a.k_weight;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] *= p[e];
                    if (!asked || at + e >= a.rot) continue;
                    const bool upper = a.interleaved ? e & 1 : at + e >= half;
                    const uint32_t other = a.interleaved ? (at + e) ^ 1 : upper ? at + e - half : at + e + half;
                    const float y = T::unpack(from[other], 0) * up * factor * (weight ? T::unpack(weight[other], 0) : 1.0f);
                    const v2f f = angles[a.interleaved ? (at + e) / 2 : upper ? other : at + e];
                    x[e] = __builtin_fmaf(x[e], f[0], upper ? y * f[1] : -(y * f[1]));
                }
            } else if (turns) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(x[e], p[e], y[e] * r[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= p[e];
            }
        }
        if constexpr (query) {
            if (asked) *(w4 *)(a.q_out + token * a.q_out_stride + (uint64_t)(head * c.head_dim + at)) = pack8<T>(x);
            return;
        }
        if (!value && asked && piece == 0 && a.pos && placed)
            a.pos[((uint64_t)seq * c.kv_heads + head) * a.pos_stride + index] = position[0];
        if (!there) return;
        const uint32_t row = row_in_slot(c, head, index);
        uint8_t *to = (value ? a.pages.v : a.pages.k) + slot_at;
        if constexpr (E8)
            put8<T>(a.pages, c.head_dim, to, asked, row, piece, a.lanes_log2, x);
        else if (asked)
            *(w4 *)(to + ((uint64_t)row * c.head_dim + at) * 2) = value ? raw : pack8<T>(x);
    };
    auto all_of = [&](auto kind, uint32_t first, uint32_t jobs, w4 ahead) __attribute__((always_inline)) {
        for (uint32_t job = first; job < jobs; job += waves) {
            const w4 raw = ahead;
            if (job + waves < jobs) ahead = load(kind, job + waves);
            process(kind, job, raw);
        }
    };
    if (wave < q_jobs) {
        factors(0, a.q_weight);
        all_of(Queries(), wave, q_jobs, ahead_q);
    }
    if (first_k < k_jobs) {
        factors(1, a.k_weight);
        all_of(Keys(), first_k, k_jobs, ahead_k);
    }
    all_of(Values(), first_v, k_jobs, ahead_v);
}

// A workgroup has kConvertTokens tokens of a sequence and KV head: all of its loads are asked for before the first store.
// Bound by memory: 49.7K cached tokens (8 KV heads, 128) from 8 bits to 16 in 60.7 us, 308 MB at 5.1 TB/s, the rate of a copy
// of this size by torch; 66.7 where the stores stay in the caches, 64.4 where the loads go past them too.  128K from 16 bits to
// 8 in 165 us, 814 MB at 4.9 TB/s, and back in 162.  5001 tokens (5 KV heads, 80) from 16 bits to 8 take 7.8 us, four dependent
// loads and the exchanges of an exponent.
template <class T, bool BACK, int ROWS>
__global__ __launch_bounds__(256) void convert(const ConvertArgs a)
{
    const CacheView &c = a.c;
    const uint32_t kv_head = blockIdx.x % c.kv_heads, rest = blockIdx.x / c.kv_heads;
    const uint32_t parts = (c.max_kv + kConvertTokens - 1) / kConvertTokens;
    const uint32_t seq = rest / parts, token0 = rest % parts * kConvertTokens;
    const int32_t kv = min(max(load4g(c.kv_len + seq), 0), (int32_t)c.max_kv);
    const int32_t begin = a.first ? max(load4g(a.first + seq), 0) : 0;
    if ((int32_t)token0 >= kv || (int32_t)(token0 + kConvertTokens) <= begin) return;
    const uint32_t lane = threadIdx.x & 63, lanes = 1u << a.lanes_log2, step = 256 >> a.lanes_log2;
    const uint32_t piece = lane & (lanes - 1);
    const bool live = piece * 8 < c.head_dim;
    const uint8_t *from_cache[2] = {a.from.k, a.from.v};
    uint8_t *to_cache[2] = {a.to.k, a.to.v};
    for (uint32_t t0 = 0; t0 < kConvertTokens; t0 += ROWS * step) {
        uint32_t row[ROWS];
        uint64_t from[ROWS], to[ROWS];
        bool there[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const uint32_t t = t0 + r * step + (threadIdx.x >> a.lanes_log2), token = token0 + t;
            const bool asked = t < kConvertTokens && (int32_t)token >= begin && (int32_t)token < kv;
            const uint32_t b = block_of(c, asked ? token : token0);
            const int32_t s0 = load4g(c.table + (uint64_t)seq * c.table_stride + b);
            const int32_t s1 = load4g(a.to_table + (uint64_t)seq * a.to_stride + b);
            there[r] = asked && (uint32_t)s0 < a.from.num_slots && (uint32_t)s1 < a.to.num_slots;
            row[r] = there[r] ? row_in_slot(c, kv_head, token) : 0;
            from[r] = there[r] ? (uint64_t)(uint32_t)s0 * a.from.slot_bytes : 0;
            to[r] = (uint64_t)(uint32_t)s1 * a.to.slot_bytes;
        }
        w4 wide[2][ROWS];
        w2 thin[2][ROWS];
        uint32_t word[2][ROWS];
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const uint8_t *p = from_cache[v] + from[r];
                const uint64_t at = (uint64_t)row[r] * c.head_dim + (live ? piece * 8 : 0);
                if constexpr (BACK) {
                    thin[v][r] = load8g((const uint16_t *)(p + at));
                    word[v][r] = (uint32_t)load4g((const int32_t *)(p + a.from.exponents + (uint64_t)row[r] * a.from.row_exponents) +
                                                  (live ? piece / 16 : 0));
                } else {
                    wide[v][r] = load16g((const uint16_t *)(p + at * 2));
                }
            }
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                uint8_t *p = to_cache[v] + (there[r] ? to[r] : 0);
                if constexpr (BACK) {
                    if (there[r] && live)
                        __builtin_nontemporal_store(widen<T>(thin[v][r], power_of(word[v][r], piece / 4 % 4 * 8)),
                                                    (w4 *)(p + ((uint64_t)row[r] * c.head_dim + piece * 8) * 2));
                } else {
                    float x[8];
                    unpack8<T>(wide[v][r], x);
                    put8<T>(a.to, c.head_dim, p, there[r] && live, row[r], piece, a.lanes_log2, x);
                }
            }
    }
}

// A workgroup has a sequence and KV head.  As the path ascends, a row moves down or stays, so rows are taken in order:
// what a pass stores lies where it or an earlier one has read.
// Bound by dependent loads: the path, the block table, the rows.  1024 lanes with four rows each in flight: 256 drafts x 48 (4
// KV heads, 128, 8 bits) 6.7 us, 11.0 with 256 lanes and one row; 8 x 32 3.2 us.
template <bool E8, int ROWS>
__global__ __launch_bounds__(ROWS > 1 ? 1024 : 256) void commit(const CommitArgs a)
{
    const CacheView &c = a.c;
    const uint32_t kv_head = blockIdx.x % c.kv_heads, seq = blockIdx.x / c.kv_heads;
    const Seq s = load_seq(c, seq);
    const int32_t count = min(max(load4g(a.accepted + seq), 0), s.n_q), shift = s.kv - s.n_q;
    if (a.len_out && kv_head == 0 && threadIdx.x == 0) a.len_out[seq] = max(shift, 0) + count;
    const uint32_t lanes = 1u << a.lanes_log2, step = blockDim.x >> a.lanes_log2, piece = threadIdx.x & (lanes - 1);
    const bool live = piece * 8 < c.head_dim;
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    int32_t *pos = a.pos ? a.pos + ((uint64_t)seq * c.kv_heads + kv_head) * a.pos_stride : nullptr;
    uint8_t *cache[2] = {a.pages.k, a.pages.v};
    for (int32_t i0 = 0; i0 < count; i0 += ROWS * step) {
        w4 wide[ROWS][2];
        w2 thin[ROWS][2];
        uint32_t word[ROWS][2];
        int32_t slot_to[ROWS], position[ROWS];
        bool moves[ROWS], listed[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int32_t i = i0 + u * step + (int32_t)(threadIdx.x >> a.lanes_log2);
            const int32_t j = i < count ? min(max(load4g(a.path + s.q_begin + i), 0), s.n_q - 1) : i;
            const int32_t to = shift + i, from = shift + j;
            listed[u] = i < count && j != i && to >= 0 && from >= 0;
            const int32_t slot = listed[u] ? load4g(table + block_of(c, from)) : -1;
            slot_to[u] = listed[u] ? load4g(table + block_of(c, to)) : -1;
            moves[u] = (uint32_t)slot < c.num_slots && (uint32_t)slot_to[u] < c.num_slots;
            const uint64_t at = moves[u] ? (uint64_t)(uint32_t)slot * a.pages.slot_bytes : 0;
            const uint32_t row = moves[u] ? row_in_slot(c, kv_head, from) : 0;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const uint8_t *p = cache[v] + at;
                const uint64_t element = (uint64_t)row * c.head_dim + (live ? piece * 8 : 0);
                if constexpr (E8) {
                    thin[u][v] = load8g((const uint16_t *)(p + element));
                    word[u][v] = (uint32_t)load4g((const int32_t *)(p + a.pages.exponents + (uint64_t)row * a.pages.row_exponents) +
                                                  (live ? piece / 16 : 0));
                } else {
                    wide[u][v] = load16g((const uint16_t *)(p + element * 2));
                }
            }
            position[u] = pos && listed[u] && piece == 0 ? pos[from] : 0;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int32_t to = shift + i0 + u * (int32_t)step + (int32_t)(threadIdx.x >> a.lanes_log2);
            if (pos && listed[u] && piece == 0) pos[to] = position[u];
            if (!moves[u] || !live) continue;
            const uint32_t row = row_in_slot(c, kv_head, to);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                uint8_t *p = cache[v] + (uint64_t)(uint32_t)slot_to[u] * a.pages.slot_bytes;
                const uint64_t element = (uint64_t)row * c.head_dim + piece * 8;
                if constexpr (E8) {
                    *(w2 *)(p + element) = thin[u][v];
                    if (piece % 16 == 0)
                        *(uint32_t *)(p + a.pages.exponents + (uint64_t)row * a.pages.row_exponents + piece / 16 * 4) = word[u][v];
                } else {
                    *(w4 *)(p + element * 2) = wide[u][v];
                }
            }
        }
    }
}

// The new lengths where they take the place of the old ones, which the move still reads.
__global__ __launch_bounds__(256) void commit_lengths(const CommitArgs a, int32_t *len_out)
{
    const uint32_t seq = blockIdx.x * 256 + threadIdx.x;
    if (seq >= a.c.n_seq) return;
    const Seq s = load_seq(a.c, seq);
    len_out[seq] = max(s.kv - s.n_q, 0) + min(max(load4g(a.accepted + seq), 0), s.n_q);
}

template <class T, bool E8>
hipError_t launch_append_as(const AppendArgs &a, hipStream_t stream)
{
    // as many waves as a token's heads fill, up to four
    const uint32_t per_wave = 64 >> a.lanes_log2;
    const uint32_t jobs = ((a.q ? a.c.heads : 0) + per_wave - 1) / per_wave + 2 * ((a.c.kv_heads + per_wave - 1) / per_wave);
    const uint32_t threads = jobs >= 4 ? 256 : jobs >= 2 ? 128 : 64;
    if (a.rot == 0 || (a.interleaved && a.rot % 8 == 0))
        append<T, E8, kInside><<<a.c.total_q, threads, 0, stream>>>(a);
    else if (!a.interleaved && a.rot % 16 == 0)
        append<T, E8, kApart><<<a.c.total_q, threads, 0, stream>>>(a);
    else
        append<T, E8, kAnyhow><<<a.c.total_q, threads, 0, stream>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_convert_as(const ConvertArgs &a, hipStream_t stream)
{
    const uint32_t grid = (a.c.max_kv + kConvertTokens - 1) / kConvertTokens * a.c.n_seq * a.c.kv_heads;
    // as many rows to a thread as a workgroup's tokens need
    if (a.from.exponents) {
        if (a.lanes_log2 >= 4)
            convert<T, true, 4><<<grid, 256, 0, stream>>>(a);
        else
            convert<T, true, 2><<<grid, 256, 0, stream>>>(a);
    } else {
        if (a.lanes_log2 >= 4)
            convert<T, false, 4><<<grid, 256, 0, stream>>>(a);
        else
            convert<T, false, 2><<<grid, 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, uint32_t dtype, hipStream_t stream)
{
    const bool e8 = a.pages.exponents;
    if (dtype == KVP_BF16) return e8 ? launch_append_as<BF16, true>(a, stream) : launch_append_as<BF16, false>(a, stream);
    return e8 ? launch_append_as<F16, true>(a, stream) : launch_append_as<F16, false>(a, stream);
}

hipError_t launch_convert(const ConvertArgs &a, uint32_t dtype, hipStream_t stream)
{
    return dtype == KVP_BF16 ? launch_convert_as<BF16>(a, stream) : launch_convert_as<F16>(a, stream);
}

hipError_t launch_commit(const CommitArgs &a, hipStream_t stream)
{
    const uint32_t grid = a.c.n_seq * a.c.kv_heads;
    const bool more = a.c.max_q > 256u >> a.lanes_log2;   // than a workgroup moves at once
    if (a.pages.exponents)
        more ? commit<true, 4><<<grid, 1024, 0, stream>>>(a) : commit<true, 1><<<grid, 256, 0, stream>>>(a);
    else
        more ? commit<false, 4><<<grid, 1024, 0, stream>>>(a) : commit<false, 1><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_commit_lengths(const CommitArgs &a, int32_t *len_out, hipStream_t stream)
{
    commit_lengths<<<(a.c.n_seq + 255) / 256, 256, 0, stream>>>(a, len_out);
    return hipGetLastError();
}

}  // namespace kvp
