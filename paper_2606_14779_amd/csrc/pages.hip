// New tokens into pages of either kind, pages from one kind to the other, accepted drafts moved together, for gfx950
// (MI355X).
//
// append: a head x of the queries or keys becomes
//   y = x / sqrt(mean(x^2) + eps) * w           (where there is a norm)
//   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin) for the pairs of its first `rot` elements, by the angle that the
//   table has for the pair and the token's position on the pair's axis
// in 32 bits, and is rounded once: to 16 bits, or to e4m3 with the least power of two that holds 32 elements.
// A head is the work of 2^lanes_log2 neighbouring lanes with 8 elements each, so that sums of squares and largest
// elements are exchanges within a wave.

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

// Over the lanes of a row, or the four lanes of 32 elements.
__device__ __forceinline__ float sum_over(float x, uint32_t lanes)
{
    for (uint32_t d = 1; d < lanes; d *= 2) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float largest_over(float x, uint32_t lanes)
{
    for (uint32_t d = 1; d < lanes; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
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

// 8 elements of a row of 8-bit pages, from all lanes of a row together (the exponents' word comes from all of them);
// to: the slot, null: not written.
template <class T>
__device__ __forceinline__ void put8(const PageView &p, uint32_t head_dim, uint8_t *to, uint32_t row, uint32_t piece,
                                     uint32_t lanes_log2, const float (&x)[8])
{
    const uint32_t lanes = 1u << lanes_log2;
    const bool live = piece * 8 < head_dim;
    const int32_t e = exponent_for<T>(largest_over(live ? largest_of(x) : 0.0f, min(lanes, 4u)));
    const uint32_t word = exponent_word(live ? e + 127 : 0, threadIdx.x & 63, lanes_log2);
    if (!to || !live) return;
    *(w2 *)(to + (uint64_t)row * head_dim + piece * 8) = narrow<T>(x, e);
    if (piece % 16 == 0) *(uint32_t *)(to + p.exponents + (uint64_t)row * p.row_exponents + piece / 16 * 4) = word;
}

// How the pairs lie: both in the 8 elements of a lane, in two lanes, or anyhow.
enum Pairs { kInside, kApart, kAnyhow };

// The norm's factor of a head whose lanes hold x.  Squares that leave the range of 32 bits are taken of x * 2^k instead.
template <class T>
__device__ __forceinline__ float norm_factor(const AppendArgs &a, const float (&x)[8], uint32_t lanes)
{
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
    sum = sum_over(sum, lanes);
    float factor = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, a.per_dim, a.eps));
    if (__builtin_expect(__any(!(sum < 1e36f && sum > 1e-30f)), 0)) {
        const float top = largest_over(largest_of(x), lanes);
        if (top > 0.0f && !(sum < 1e36f && sum > 1e-30f)) {
            const int k = top > 1.0f ? -64 : 64;     // bf16 ends at 2^128, and f16 does not come here but with eps below it
            const float up = __builtin_ldexpf(1.0f, k);
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[i] * up, x[i] * up, s);
            for (uint32_t d = 1; d < lanes; d *= 2) s += __shfl_xor(s, d);
            const float mean = s * a.per_dim + __builtin_ldexpf(a.eps, 2 * k);
            factor = __builtin_ldexpf(__builtin_amdgcn_rsqf(mean), k);
        }
    }
    return factor;
}

template <class T, bool E8, int PAIRS>
__global__ __launch_bounds__(256) void append(const AppendArgs a)
{
    __shared__ v2f angles[kMostRotary / 2];          // of this token
    const CacheView &c = a.c;
    const uint32_t token = blockIdx.x, lane = threadIdx.x & 63;
    const uint32_t lanes = 1u << a.lanes_log2;
    const uint32_t q_heads = a.q ? c.heads : 0, keys_end = q_heads + c.kv_heads;
    const uint32_t units = (keys_end + c.kv_heads) << a.lanes_log2;

    // a position that the table does not have: NaN, so that it shows
    bool known = true;
    for (uint32_t i = 0; i < a.axes; ++i) {
        const int32_t p = load4g(a.positions + (uint64_t)i * c.total_q + token);
        known &= p >= 0 && (uint32_t)p < a.n_positions;
    }
    for (uint32_t j = threadIdx.x; j < a.rot / 2; j += blockDim.x) {
        const int32_t p = known ? load4g(a.positions + (uint64_t)a.axis_of[j] * c.total_q + token) : 0;
        angles[j] = *(const v2f *)(a.angles + (uint64_t)(uint32_t)p * a.rot + 2 * j);
    }
    // the token's sequence: the last one that begins at or before it, 64 at a time
    uint32_t seq = 0;
    for (uint32_t n = c.n_seq; n > 1;) {
        const uint32_t step = (n + 63) / 64, at = seq + lane * step;
        const uint32_t count = __popcll(__ballot(lane * step < n && load4g(c.cu_q + min(at, c.n_seq)) <= (int32_t)token));
        const uint32_t last = count ? count - 1 : 0;
        seq += last * step;
        n = min(step, n - last * step);
    }
    const Seq s = load_seq(c, seq);
    const int32_t i = (int32_t)token - s.q_begin, index = s.kv - s.n_q + i;
    const bool placed = i >= 0 && i < s.n_q && index >= 0;
    const int32_t slot = placed ? load4g(c.table + (uint64_t)seq * c.table_stride + block_of(c, index)) : -1;
    const bool there = (uint32_t)slot < c.num_slots;
    __syncthreads();

    for (uint32_t first = threadIdx.x & ~63u; first < units; first += blockDim.x) {
        const uint32_t unit = first + lane, piece = unit & (lanes - 1), at = piece * 8;
        const uint32_t all = unit >> a.lanes_log2;   // head among queries, keys and values
        const bool query = all < q_heads, value = all >= keys_end;
        const uint32_t head = query ? all : value ? all - keys_end : all - q_heads;
        const bool live = unit < units && at < c.head_dim;
        const uint16_t *from = (query ? a.q + token * a.q_stride : value ? a.v + token * a.v_stride : a.k + token * a.k_stride) +
                               (uint64_t)head * c.head_dim;
        const w4 raw = live ? load16g(from + at) : w4{0, 0, 0, 0};
        float x[8];
        unpack8<T>(raw, x);
        const uint16_t *weight = query ? a.q_weight : a.k_weight;
        float factor = 1.0f;
        if (a.norm) {
            factor = norm_factor<T>(a, x, lanes);
            if (!value) {
                float w[8];
                unpack8<T>(weight && live ? load16g(weight + at) : w4{0, 0, 0, 0}, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * factor * (weight ? w[e] : 1.0f);
            }
        }
        if constexpr (PAIRS == kInside) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                if (value || at + e >= a.rot) continue;
                const v2f f = angles[(at + e) / 2];
                const float p = x[e], q = x[e + 1];
                x[e] = __builtin_fmaf(p, f[0], -(q * f[1]));
                x[e + 1] = __builtin_fmaf(q, f[0], p * f[1]);
            }
        } else if constexpr (PAIRS == kApart) {
            const uint32_t half = a.rot / 16;        // lanes
            const bool upper = piece >= half;
            const int other = (int)lane + (upper ? -(int)half : (int)half);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], other & 63);
            if (!value && at < a.rot) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const v2f f = angles[at + e - (upper ? a.rot / 2 : 0)];
                    x[e] = __builtin_fmaf(x[e], f[0], upper ? y[e] * f[1] : -(y[e] * f[1]));
                }
            }
        } else {
            if (live && !value) {
                const uint32_t half = a.rot / 2;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (at + e >= a.rot) continue;
                    const bool upper = at + e >= half;
                    const uint32_t other = upper ? at + e - half : at + e + half;
                    float y = T::unpack(from[other], 0);
                    if (a.norm) y = y * factor * (weight ? T::unpack(weight[other], 0) : 1.0f);
                    const v2f f = angles[upper ? other : at + e];
                    x[e] = __builtin_fmaf(x[e], f[0], upper ? y * f[1] : -(y * f[1]));
                }
            }
        }
        if (!known && !value) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __builtin_nanf("");
        }
        if (live && query) *(w4 *)(a.q_out + token * a.q_out_stride + (uint64_t)head * c.head_dim + at) = pack8<T>(x);
        const bool cached = unit < units && !query;
        if (cached && !value && piece == 0 && a.pos && placed)
            a.pos[((uint64_t)seq * c.kv_heads + head) * a.pos_stride + index] = load4g(a.positions + token);
        const uint32_t row = cached && there ? row_in_slot(c, head, index) : 0;
        uint8_t *to = (value ? a.pages.v : a.pages.k) + (uint64_t)(there ? slot : 0) * a.pages.slot_bytes;
        if constexpr (E8) {
            if (__any(cached)) put8<T>(a.pages, c.head_dim, cached && there ? to : nullptr, row, piece, a.lanes_log2, x);
        } else {
            if (live && cached && there)
                *(w4 *)(to + ((uint64_t)row * c.head_dim + at) * 2) = value ? raw : pack8<T>(x);
        }
    }
}

// A workgroup has kConvertTokens tokens of a sequence and KV head: all of its loads are asked for before the first store.
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
                        *(w4 *)(p + ((uint64_t)row[r] * c.head_dim + piece * 8) * 2) =
                            widen<T>(thin[v][r], power_of(word[v][r], piece / 4 % 4 * 8));
                } else {
                    float x[8];
                    unpack8<T>(wide[v][r], x);
                    put8<T>(a.to, c.head_dim, there[r] ? p : nullptr, row[r], piece, a.lanes_log2, x);
                }
            }
    }
}

// A workgroup has a sequence and KV head.  As the path ascends, a row moves down or stays, so rows are taken in order:
// what a pass stores lies where it or an earlier one has read.
template <bool E8>
__global__ __launch_bounds__(256) void commit(const CommitArgs a)
{
    const CacheView &c = a.c;
    const uint32_t kv_head = blockIdx.x % c.kv_heads, seq = blockIdx.x / c.kv_heads;
    const Seq s = load_seq(c, seq);
    const int32_t count = min(max(load4g(a.accepted + seq), 0), s.n_q), shift = s.kv - s.n_q;
    if (a.len_out && kv_head == 0 && threadIdx.x == 0) a.len_out[seq] = max(shift, 0) + count;
    const uint32_t lanes = 1u << a.lanes_log2, step = 256 >> a.lanes_log2, piece = threadIdx.x & (lanes - 1);
    const bool live = piece * 8 < c.head_dim;
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    int32_t *pos = a.pos ? a.pos + ((uint64_t)seq * c.kv_heads + kv_head) * a.pos_stride : nullptr;
    for (int32_t i0 = 0; i0 < count; i0 += step) {
        const int32_t i = i0 + (int32_t)(threadIdx.x >> a.lanes_log2);
        const int32_t j = i < count ? min(max(load4g(a.path + s.q_begin + i), 0), s.n_q - 1) : i;
        const int32_t to = shift + i, from = shift + j;
        bool moves = i < count && j != i && to >= 0 && from >= 0;
        const int32_t slot_from = moves ? load4g(table + block_of(c, from)) : -1;
        const int32_t slot_to = moves ? load4g(table + block_of(c, to)) : -1;
        const bool listed = moves;
        moves = (uint32_t)slot_from < c.num_slots && (uint32_t)slot_to < c.num_slots;
        w4 wide[2];
        w2 thin[2];
        uint32_t word[2];
        int32_t position = 0;
        uint8_t *cache[2] = {a.pages.k, a.pages.v};
        const uint64_t at = moves ? (uint64_t)(uint32_t)slot_from * a.pages.slot_bytes : 0;
        const uint32_t row = moves ? row_in_slot(c, kv_head, from) : 0;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const uint8_t *p = cache[v] + at;
            const uint64_t element = (uint64_t)row * c.head_dim + (live ? piece * 8 : 0);
            if constexpr (E8) {
                thin[v] = load8g((const uint16_t *)(p + element));
                word[v] = (uint32_t)load4g((const int32_t *)(p + a.pages.exponents + (uint64_t)row * a.pages.row_exponents) +
                                           (live ? piece / 16 : 0));
            } else {
                wide[v] = load16g((const uint16_t *)(p + element * 2));
            }
        }
        if (pos && listed && piece == 0) position = pos[from];
        __syncthreads();
        if (pos && listed && piece == 0) pos[to] = position;
        if (moves && live) {
            const uint32_t row_to = row_in_slot(c, kv_head, to);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                uint8_t *p = cache[v] + (uint64_t)(uint32_t)slot_to * a.pages.slot_bytes;
                const uint64_t element = (uint64_t)row_to * c.head_dim + piece * 8;
                if constexpr (E8) {
                    *(w2 *)(p + element) = thin[v];
                    if (piece % 16 == 0)
                        *(uint32_t *)(p + a.pages.exponents + (uint64_t)row_to * a.pages.row_exponents + piece / 16 * 4) = word[v];
                } else {
                    *(w4 *)(p + element * 2) = wide[v];
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
    // whole wavefronts, as many as a token's units fill, up to four
    const uint32_t units = ((a.q ? a.c.heads : 0) + 2 * a.c.kv_heads) << a.lanes_log2;
    const uint32_t threads = units >= 256 ? 256 : (units + 63) / 64 * 64;
    if (a.interleaved || a.rot == 0)
        append<T, E8, kInside><<<a.c.total_q, threads, 0, stream>>>(a);
    else if (a.rot % 16 == 0)
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
    if (dtype == KVP_BF16) return a.pages.exponents ? launch_append_as<BF16, true>(a, stream) : launch_append_as<BF16, false>(a, stream);
    return a.pages.exponents ? launch_append_as<F16, true>(a, stream) : launch_append_as<F16, false>(a, stream);
}

hipError_t launch_convert(const ConvertArgs &a, uint32_t dtype, hipStream_t stream)
{
    return dtype == KVP_BF16 ? launch_convert_as<BF16>(a, stream) : launch_convert_as<F16>(a, stream);
}

hipError_t launch_commit(const CommitArgs &a, hipStream_t stream)
{
    const uint32_t grid = a.c.n_seq * a.c.kv_heads;
    if (a.pages.exponents)
        commit<true><<<grid, 256, 0, stream>>>(a);
    else
        commit<false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_commit_lengths(const CommitArgs &a, int32_t *len_out, hipStream_t stream)
{
    commit_lengths<<<(a.c.n_seq + 255) / 256, 256, 0, stream>>>(a, len_out);
    return hipGetLastError();
}

}  // namespace kvp
