// Eviction from the paged cache by score, for gfx950 (MI355X).
//
// A sequence of n tokens keeps, for every KV head by itself, the `keep` tokens of largest key: protected
// tokens first, by lower index, then the others by score and lower index; a NaN score counts below every number.  Kept tokens at
// index >= keep move into the places below keep that fell free, both in ascending order.  No source is a
// destination, so the moves need no order among themselves and the cache is compacted in place; and since
// attention without a window does not depend on the order of the keys before the new ones, nothing else has to move.
// (A window counts cache indexes, and these no longer follow the positions.)
//
// Bound by what has to wait for what: digits counted, picked, counted again, then the moves listed and made.  64 of
// 2112 tokens of 16 sequences and 8 KV heads: 11 us to select in one workgroup a list, 5 to move.  128K tokens to 8K, 8
// heads: 7 us to count, 10 to mark, 19 to finish, 10 to move; with a single workgroup a list to select, 96 + 10.

#include <algorithm>

#include "wave.hpp"

namespace kvp {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kShortKeys = kEvictShort / kSelectThreads;   // keys of a thread
constexpr int kPartThreads = 256;
constexpr int kPartWaves = kPartThreads / 64;
constexpr int kStretches = kEvictParts * kPartWaves;
constexpr int kBins = 2048;                                // of the first digit; the others: 11 and 10 bits
static_assert(kBins == 1 << 11, "digits of 11, 11 and 10 bits");

// Order-preserving key of a score; 0 is NaN's, the largest value the protected tokens'.
__device__ __forceinline__ uint32_t key_of(float score, bool guarded)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, score);
    uint32_t k = u << 1 == 0 ? 0x80000000u : u & 0x80000000u ? ~u : u | 0x80000000u;
    k = score != score ? 0 : k;
    return guarded ? 0xFFFFFFFFu : k;
}

// What a list's kernels leave each other: (to, from) pairs and a bit per kept token, and for long lists the counts
// of the first digit per part, the candidates (key, token) of every wave's stretch and how many there are.  The
// candidates share the pairs' space: they are done before a pair is written.
struct Lists {
    uint32_t *head;                                  // pairs, tokens, the first digit, keys wanted of it
    uint32_t *pairs;
    w2 *candidates;
    uint64_t *kept;
    uint32_t *hist, *found;
};
__device__ __forceinline__ Lists lists_of(const EvictArgs &a, uint32_t list)
{
    uint32_t *p = a.moves + (uint64_t)list * a.list_words;
    const uint64_t n = a.c.max_kv, words = 2 * ((n + 63) / 64);
    uint32_t *h = p + 4 + 2 * n + words;
    return {p, p + 4, (w2 *)(p + 4), (uint64_t *)(p + 4 + 2 * n), h, h + kEvictParts * kBins};
}

struct List {
    uint32_t index, n, keep;
    const float *score;
    const int32_t *pos;
    bool guards;
    int32_t guard;
    __device__ __forceinline__ uint32_t key(uint32_t at, float x, int32_t p) const
    {
        return key_of(x, guards && (pos ? p : (int32_t)at) >= guard);
    }
};
__device__ __forceinline__ List list_of(const EvictArgs &a, uint32_t index)
{
    const CacheView &c = a.c;
    const uint32_t seq = index / c.kv_heads;
    return {index,
            (uint32_t)min(max(load4g(c.kv_len + seq), 0), (int32_t)c.max_kv),
            (uint32_t)max(load4g(a.keep + seq), 0),
            a.score_in + (uint64_t)index * a.score_stride,
            a.pos_in ? a.pos_in + (uint64_t)index * a.pos_stride : nullptr,
            a.protect != nullptr,
            a.protect ? load4g(a.protect + seq) : 0};
}

// Exclusive sum over the workgroup's threads; *all: the sum of all of them.
template <int WAVES>
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t *lds, int wave, int lane, uint32_t *all)
{
    uint32_t upto = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
    }
    __syncthreads();                                 // lds may still be read from the last time
    if (lane == 63) lds[wave] = upto;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    *all = total;
    return before + upto - x;
}

// Counts a digit per lane.  Equal scores are common (tokens that no query looked at): the lanes that agree with
// the first one are counted by one addition instead of one after the other.
__device__ __forceinline__ void count_digit(uint32_t *hist, uint32_t digit, bool mine, int lane)
{
    const uint64_t active = __ballot(mine);
    if (!active) return;
    const int leader = __ffsll((unsigned long long)active) - 1;
    const uint32_t first = __builtin_amdgcn_readlane(digit, leader);
    const uint64_t same = __ballot(mine && digit == first);
    if (lane == leader) atomicAdd(&hist[first], (uint32_t)__popcll(same));
    if (mine && digit != first) atomicAdd(&hist[digit], 1u);
}

// From the largest digit down, the one in which the left-th key lies; *above: the keys of larger digits.  A thread
// has the counts of PER digits, mine[i] of digit bins - 1 - (tid * PER + i).
template <int PER, int WAVES>
__device__ __forceinline__ uint32_t pick_digit(const uint32_t (&mine)[PER], uint32_t *lds, uint32_t *pick, uint32_t left,
                                               int tid, uint32_t *above)
{
    uint32_t sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += mine[i];
    uint32_t before = sum_before<WAVES>(sum, lds, tid >> 6, tid & 63, &all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (before < left && left <= before + mine[i]) {
            pick[0] = PER * WAVES * 64 - 1 - (tid * PER + i);
            pick[1] = before;
        }
        before += mine[i];
    }
    __syncthreads();
    *above = pick[1];
    return pick[0];
}

// A sequence of up to kEvictShort tokens, one workgroup to a KV head: the keys stay in registers, the smallest kept
// one is found digit by digit (the counts are integers, so the atomics' order does not matter), and the moves are
// listed in order, every wave over a stretch of its own.
__global__ __launch_bounds__(kSelectThreads) void evict_short(const EvictArgs a)
{
    __shared__ uint32_t hist[kBins], lds_sum[kSelectWaves], lds_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const List t = list_of(a, blockIdx.x);
    const Lists lists = lists_of(a, blockIdx.x);
    if (t.n <= t.keep) {
        if (tid == 0) lists.head[0] = 0, lists.head[1] = t.n;
        return;
    }
    const uint32_t n = t.n, keep = t.keep;
    const uint32_t stretch = (n + kSelectThreads - 1) / kSelectThreads * 64;
    const uint32_t from = min(wave * stretch, n), to = min(from + stretch, n);
    float x[kShortKeys];
    int32_t p[kShortKeys];
    uint32_t key[kShortKeys];
#pragma unroll
    for (int j = 0; j < kShortKeys; ++j) {
        const uint32_t at = min(from + 64 * j + lane, n - 1);
        x[j] = from + 64 * j < to ? t.score[at] : 0.0f;
        p[j] = from + 64 * j < to && t.guards && t.pos ? t.pos[at] : 0;
    }
#pragma unroll
    for (int j = 0; j < kShortKeys; ++j) key[j] = t.key(from + 64 * j + lane, x[j], p[j]);
    auto there = [&](int j) { return from + 64 * j + lane < to; };

    uint32_t prefix = 0xFFFFFFFFu, left = 0, above = 0;
    if (keep) {
        left = keep;
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
            hist[tid] = 0;
            hist[tid + kSelectThreads] = 0;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kShortKeys; ++j)
                if (from + 64 * j < to)
                    count_digit(hist, key[j] >> shift & ((1u << bits) - 1),
                                there(j) && (round == 0 || key[j] >> (shift + bits) == prefix), lane);
            __syncthreads();
            const uint32_t mine[2] = {hist[kBins - 1 - 2 * tid], hist[kBins - 2 - 2 * tid]};
            const uint32_t digit = pick_digit<2, kSelectWaves>(mine, lds_sum, lds_pick, left, tid, &above);
            prefix = round ? prefix << bits | digit : digit;
            left -= above;
            __syncthreads();
        }
    }
    // kept: keys above the smallest one, and the first `left` of those equal to it
    uint32_t equal = 0, all;
#pragma unroll
    for (int j = 0; j < kShortKeys; ++j)
        if (from + 64 * j < to) equal += __popcll(__ballot(keep && there(j) && key[j] == prefix));
    uint32_t rank = __shfl(sum_before<kSelectWaves>(lane ? 0 : equal, lds_sum, wave, lane, &all), 0);
    const uint64_t below = (1ull << lane) - 1;
    uint64_t kept[kShortKeys], low[kShortKeys];
    uint32_t holes = 0, movers = 0;
#pragma unroll
    for (int j = 0; j < kShortKeys; ++j) {
        const uint32_t first = from + 64 * j;
        kept[j] = 0;
        if (first >= to) continue;
        const uint64_t same = __ballot(keep && there(j) && key[j] == prefix);
        kept[j] = __ballot(keep && there(j) && (key[j] > prefix || (key[j] == prefix && rank + __popcll(same & below) < left)));
        rank += __popcll(same);
        if (lane == 0) lists.kept[first >> 6] = kept[j];
        low[j] = keep <= first ? 0 : keep - first >= 64 ? ~0ull : (1ull << (keep - first)) - 1;   // below keep, and keep < n
        holes += __popcll(~kept[j] & low[j]);
        movers += __popcll(kept[j] & ~low[j]);
    }
    // both counts in one sum: there are at most kEvictShort of each
    static_assert(kEvictShort < 1 << 16, "two counts to a word");
    const uint32_t both = __shfl(sum_before<kSelectWaves>(lane ? 0 : holes | movers << 16, lds_sum, wave, lane, &all), 0);
    uint32_t h = both & 0xFFFF, v = both >> 16;
#pragma unroll
    for (int j = 0; j < kShortKeys; ++j) {
        const uint32_t at = from + 64 * j + lane;
        if (from + 64 * j >= to) continue;
        const uint64_t hole = ~kept[j] & low[j], mover = kept[j] & ~low[j];
        if (hole >> lane & 1) lists.pairs[2 * (h + __popcll(hole & below))] = at;
        if (mover >> lane & 1) lists.pairs[2 * (v + __popcll(mover & below)) + 1] = at;
        h += __popcll(hole);
        v += __popcll(mover);
    }
    const uint32_t count = all & 0xFFFF;             // as many movers as holes
    if (tid == 0) lists.head[0] = count, lists.head[1] = n;
}

// ---- longer sequences: the two passes over the scores are spread over kEvictParts workgroups a list

constexpr int kAhead = 8;        // loads in flight per lane

// The tokens of a part's wave, the stretches of all parts' waves one after the other.
struct Stretch {
    uint32_t from, to;
};
__device__ __forceinline__ Stretch stretch_of(uint32_t n, uint32_t index)
{
    const uint32_t size = (n + kStretches * 64 - 1) / (kStretches * 64) * 64;
    const uint32_t from = (uint32_t)min((uint64_t)index * size, (uint64_t)n);
    return {from, (uint32_t)min((uint64_t)from + size, (uint64_t)n)};
}

// f(token of this lane, its key, whether there is one) over a stretch, 64 tokens at a time
template <class F>
__device__ __forceinline__ void over_keys(const List &t, Stretch s, int lane, F f)
{
    for (uint32_t i = s.from; i < s.to; i += 64 * kAhead) {
        float x[kAhead];
        int32_t p[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[j] = t.score[min(i + 64 * j + lane, s.to - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) p[j] = t.guards && t.pos ? t.pos[min(i + 64 * j + lane, s.to - 1)] : 0;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t at = i + 64 * j + lane;
            if (i + 64 * j < s.to) f(at, t.key(at, x[j], p[j]), at < s.to);
        }
    }
}

// Counts the first digits of a part.
__global__ __launch_bounds__(kPartThreads) void evict_count(const EvictArgs a)
{
    __shared__ uint32_t hist[kBins];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t part = blockIdx.x % kEvictParts;
    const List t = list_of(a, blockIdx.x / kEvictParts);
    if (t.n <= t.keep || t.keep == 0) return;
    for (int i = tid; i < kBins; i += kPartThreads) hist[i] = 0;
    __syncthreads();
    over_keys(t, stretch_of(t.n, part * kPartWaves + wave), lane,
              [&](uint32_t, uint32_t key, bool there) { count_digit(hist, key >> 21, there, lane); });
    __syncthreads();
    uint32_t *out = lists_of(a, t.index).hist + part * kBins;
    for (int i = tid; i < kBins; i += kPartThreads) out[i] = hist[i];
}

// Marks a part's tokens above the digit that the last kept key has, and collects those in it.
__global__ __launch_bounds__(kPartThreads) void evict_mark(const EvictArgs a)
{
    __shared__ uint32_t lds_sum[kPartWaves], lds_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t part = blockIdx.x % kEvictParts, stretch = part * kPartWaves + wave;
    const List t = list_of(a, blockIdx.x / kEvictParts);
    const Lists lists = lists_of(a, t.index);
    if (t.n <= t.keep) return;
    uint32_t prefix = 0xFFFFFFFFu, above = 0;
    if (t.keep) {
        constexpr int PER = kBins / kPartThreads;
        uint32_t mine[PER] = {};
#pragma unroll 4
        for (int q = 0; q < kEvictParts; ++q) {
            const uint32_t *h = lists.hist + q * kBins + (kBins - PER - tid * PER);   // bins in order: the last is mine[0]
#pragma unroll
            for (int i = 0; i < PER; ++i) mine[i] += h[PER - 1 - i];
        }
        prefix = pick_digit<PER, kPartWaves>(mine, lds_sum, lds_pick, t.keep, tid, &above);
    }
    const Stretch s = stretch_of(t.n, stretch);
    uint32_t found = 0;
    over_keys(t, s, lane, [&](uint32_t at, uint32_t key, bool there) {
        const uint64_t more = __ballot(there && t.keep && key >> 21 > prefix);
        const bool in = there && t.keep && key >> 21 == prefix;
        const uint64_t ins = __ballot(in);
        if (lane == 0) lists.kept[at >> 6] = more;
        if (in) lists.candidates[s.from + found + __popcll(ins & ((1ull << lane) - 1))] = w2{key, at};
        found += __popcll(ins);
    });
    if (lane == 0) lists.found[stretch] = found;
    if (part == 0 && tid == 0) lists.head[2] = prefix, lists.head[3] = t.keep - above;
}

// Finds the smallest kept key among the candidates, marks those that are kept, and lists the moves.
__global__ __launch_bounds__(kSelectThreads) void evict_finish(const EvictArgs a)
{
    __shared__ uint32_t hist[kBins], lds_sum[kSelectWaves], lds_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const List t = list_of(a, blockIdx.x);
    const Lists lists = lists_of(a, blockIdx.x);
    const uint32_t n = t.n, keep = t.keep;
    if (n <= keep) {
        if (tid == 0) lists.head[0] = 0, lists.head[1] = n;
        return;
    }
    constexpr int PER = kStretches / kSelectWaves;   // stretches of a wave
    const uint32_t size = stretch_of(n, 1).from;     // of a stretch, or n
    // the wave's stretches one after the other: ends[q] candidates up to stretch q's end
    uint32_t ends[PER], total = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) ends[q] = total += lists.found[wave * PER + q];
    constexpr int U = 8;
    auto load = [&](uint32_t i0, w2 (&k)[U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = min(i0 + 64 * u + lane, total - 1);
            uint32_t q = 0, begin = 0;
#pragma unroll
            for (int e = 0; e + 1 < PER; ++e)
                if (i >= ends[e]) q = e + 1, begin = ends[e];
            k[u] = lists.candidates[(uint64_t)(wave * PER + q) * size + (i - begin)];
        }
    };
    // f(candidate, whether there is one) in order; the first ones stay in registers, as a rule all of them
    w2 first[U];
    if (total) load(0, first);
    auto over_candidates = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (64u * u < total) f(first[u], 64 * u + lane < total);
        for (uint32_t i0 = 64 * U; i0 < total; i0 += 64 * U) {
            w2 k[U];
            load(i0, k);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + 64 * u < total) f(k[u], i0 + 64 * u + lane < total);
        }
    };
    uint32_t prefix = lists.head[2], left = lists.head[3], above = 0, all;
    for (int round = 1; keep && round < 3; ++round) {
        const int shift = round == 1 ? 10 : 0, bits = round == 1 ? 11 : 10;
        hist[tid] = 0;
        hist[tid + kSelectThreads] = 0;
        __syncthreads();
        over_candidates([&](w2 k, bool there) {
            count_digit(hist, k[0] >> shift & ((1u << bits) - 1), there && k[0] >> (shift + bits) == prefix, lane);
        });
        __syncthreads();
        const uint32_t mine[2] = {hist[kBins - 1 - 2 * tid], hist[kBins - 2 - 2 * tid]};
        prefix = prefix << bits | pick_digit<2, kSelectWaves>(mine, lds_sum, lds_pick, left, tid, &above);
        left -= above;
        __syncthreads();
    }
    if (keep) {
        uint32_t equal = 0;
        over_candidates([&](w2 k, bool there) { equal += __popcll(__ballot(there && k[0] == prefix)); });
        uint32_t rank = __shfl(sum_before<kSelectWaves>(lane ? 0 : equal, lds_sum, wave, lane, &all), 0);
        over_candidates([&](w2 k, bool there) {
            const uint64_t same = __ballot(there && k[0] == prefix);
            const bool kept = there && (k[0] > prefix ||
                                        (k[0] == prefix && rank + __popcll(same & ((1ull << lane) - 1)) < left));
            rank += __popcll(same);
            if (kept)
                __hip_atomic_fetch_or(lists.kept + (k[1] >> 6), 1ull << (k[1] & 63), __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
        });
        __builtin_amdgcn_s_waitcnt(0);               // the bits are set before another wave reads them
    }
    __syncthreads();
    // holes and movers in order, a word of 64 tokens to a thread
    const uint32_t words = (n + 63) / 64;
    uint32_t holes = 0, movers = 0;
    for (uint32_t w0 = 0; w0 < words; w0 += kSelectThreads) {
        const uint32_t w = w0 + tid;
        uint64_t hole = 0, mover = 0;
        if (w < words) {
            const uint64_t kept = __hip_atomic_load(lists.kept + w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const uint64_t low = keep <= 64 * w ? 0 : keep - 64 * w >= 64 ? ~0ull : (1ull << (keep - 64 * w)) - 1;   // below keep
            hole = ~kept & low;                      // keep < n: every token below keep is there
            mover = kept & ~low;
        }
        if (64 * (uint64_t)w0 < keep) {              // the same for all
            uint32_t h = sum_before<kSelectWaves>(__popcll(hole), lds_sum, wave, lane, &all) + holes;
            holes += all;
            for (; hole; hole &= hole - 1) lists.pairs[2 * (uint64_t)h++] = 64 * w + __ffsll((unsigned long long)hole) - 1;
        }
        if (64 * (uint64_t)(w0 + kSelectThreads) > keep) {
            uint32_t m = sum_before<kSelectWaves>(__popcll(mover), lds_sum, wave, lane, &all) + movers;
            movers += all;
            for (; mover; mover &= mover - 1) lists.pairs[2 * (uint64_t)m++ + 1] = 64 * w + __ffsll((unsigned long long)mover) - 1;
        }
    }
    if (tid == 0) lists.head[0] = holes, lists.head[1] = n;   // as many as movers
}

// The rows of the listed moves, 16 bytes to a lane; scores and positions of the moves, and of the kept tokens that
// stay where the outputs are other arrays; zeros past the new length.  Score arrays may be the same: a move's score
// is read and replaced by 0 by one thread, and no other one writes a mover's place.
__global__ __launch_bounds__(256) void evict_move(const EvictArgs a, const uint32_t groups)
{
    const CacheView &c = a.c;
    const uint32_t list = blockIdx.x / groups, group = blockIdx.x % groups;
    const uint32_t head = list % c.kv_heads, seq = list / c.kv_heads;
    const Lists lists = lists_of(a, list);
    // not from kv_len, which may be written here
    const uint32_t n = min(lists.head[1], c.max_kv), keep = (uint32_t)max(load4g(a.keep + seq), 0), left = min(n, keep);
    const uint32_t count = min(lists.head[0], c.max_kv / 2), pieces = c.head_dim / 8;
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    if (group == 0 && head == 0 && threadIdx.x == 0) a.len_out[seq] = (int32_t)left;
    const uint64_t sl = (uint64_t)list * a.score_stride, pl = (uint64_t)list * a.pos_stride;
    // move i, piece of it: their product may pass 32 bits
    const uint32_t begin = group * 256 + threadIdx.x, step = groups * 256;
    const uint32_t step_i = step / pieces, step_piece = step % pieces;
    uint32_t i = begin / pieces, piece = begin % pieces;
    for (; i < count; i += step_i, piece += step_piece) {
        if (piece >= pieces) {
            piece -= pieces;
            if (++i >= count) break;
        }
        const uint32_t hole = lists.pairs[2 * (uint64_t)i], mover = lists.pairs[2 * (uint64_t)i + 1];
        if (piece == 0) {
            const float x = a.score_in[sl + mover];
            const int32_t p = a.pos_in ? a.pos_in[pl + mover] : (int32_t)mover;
            a.score_out[sl + hole] = x;
            a.score_out[sl + mover] = 0.0f;
            if (a.pos_out) a.pos_out[pl + hole] = p;
        }
        const uint32_t to = row_of(c, load4g(table + block_of(c, hole)), head, hole);
        const uint32_t from = row_of(c, load4g(table + block_of(c, mover)), head, mover);
        if (to == kNoRow || from == kNoRow) continue;
        const uint64_t d = (uint64_t)to * c.head_dim + piece * 8, s = (uint64_t)from * c.head_dim + piece * 8;
        const w4 k = load16g(a.k_cache + s), v = load16g(a.v_cache + s);
        *(w4 *)(a.k_cache + d) = k;
        *(w4 *)(a.v_cache + d) = v;
    }
    const bool copies = a.score_out != a.score_in || (a.pos_out && a.pos_out != a.pos_in);
    for (i = begin; i < n; i += step) {
        if (i < left && !copies) continue;
        const bool kept = n <= keep || (lists.kept[i >> 6] >> (i & 63) & 1);
        if (i >= left && !kept) a.score_out[sl + i] = 0.0f;
        if (i < left && kept) {
            a.score_out[sl + i] = a.score_in[sl + i];
            if (a.pos_out) a.pos_out[pl + i] = a.pos_in ? a.pos_in[pl + i] : (int32_t)i;
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, hipStream_t stream)
{
    const uint32_t lists = a.c.n_seq * a.c.kv_heads;
    if (a.c.max_kv <= kEvictShort) {
        evict_short<<<lists, kSelectThreads, 0, stream>>>(a);
    } else {
        evict_count<<<lists * kEvictParts, kPartThreads, 0, stream>>>(a);
        evict_mark<<<lists * kEvictParts, kPartThreads, 0, stream>>>(a);
        evict_finish<<<lists, kSelectThreads, 0, stream>>>(a);
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    // 8 workgroups to a CU, and to a list no more than it has tokens for
    const uint64_t groups = std::max<uint64_t>(1, std::min<uint64_t>((a.c.max_kv + 255) / 256, 2048 / lists));
    evict_move<<<(uint32_t)(lists * groups), 256, 0, stream>>>(a, (uint32_t)groups);
    return hipGetLastError();
}

}  // namespace kvp
