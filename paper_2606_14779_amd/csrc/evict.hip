// Eviction from the paged cache by score, for gfx950 (MI355X).
//
// A sequence of n tokens keeps, for every KV head by itself, the `keep` tokens of largest key: protected
// tokens first, then by score, then by lower index; a NaN score counts below every number.  Kept tokens at
// index >= keep move into the places below keep that fell free, both in ascending order.  No source is a
// destination, so the moves need no order among themselves and the cache is compacted in place; and since
// attention does not depend on the order of the keys before the new ones, nothing else has to move.

#include <algorithm>

#include "wave.hpp"

namespace kvp {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;

// Order-preserving key of a score; 0 is NaN's, the largest value the protected tokens'.
__device__ __forceinline__ uint32_t key_of(float score, bool guarded)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, score);
    uint32_t k = u << 1 == 0 ? 0x80000000u : u & 0x80000000u ? ~u : u | 0x80000000u;
    k = score != score ? 0 : k;
    return guarded ? 0xFFFFFFFFu : k;
}

// What the first kernel leaves of a list for the second: (to, from) pairs and a bit per kept token.  The
// candidates (key, token) of the search share the pairs' space: they are done before a pair is written.
struct Lists {
    uint32_t *head;                                  // pairs, tokens
    uint32_t *pairs;
    w2 *candidates;
    uint64_t *kept;
};
__device__ __forceinline__ Lists lists_of(const EvictArgs &a, uint32_t list)
{
    uint32_t *p = a.moves + (uint64_t)list * a.list_words;
    return {p, p + 2, (w2 *)(p + 2), (uint64_t *)(p + 2 + 2 * (uint64_t)a.c.max_kv)};
}

// Exclusive sum over the workgroup's threads; *all: the sum of all of them.
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
    for (int w = 0; w < kSelectWaves; ++w) {
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
    const uint32_t first = __shfl(digit, leader);
    const uint64_t same = __ballot(mine && digit == first);
    if (lane == leader) atomicAdd(&hist[first], (uint32_t)__popcll(same));
    if (mine && digit != first) atomicAdd(&hist[digit], 1u);
}

// From the largest digit down, the one in which the left-th key lies; *above: the keys of larger digits.
template <int PER>
__device__ __forceinline__ uint32_t pick_digit(const uint32_t *hist, uint32_t *lds, uint32_t *pick, uint32_t left, int tid,
                                               uint32_t *above)
{
    constexpr int bins = PER * kSelectThreads;
    uint32_t mine[PER], sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += mine[i] = hist[bins - 1 - (tid * PER + i)];
    uint32_t before = sum_before(sum, lds, tid >> 6, tid & 63, &all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (before < left && left <= before + mine[i]) {
            pick[0] = bins - 1 - (tid * PER + i);
            pick[1] = before;
        }
        before += mine[i];
    }
    __syncthreads();
    *above = pick[1];
    return pick[0];
}

constexpr int kAhead = 8;        // loads in flight per lane

// One workgroup to a sequence and KV head.  The smallest kept key is found digit by digit (12, 10 and 10 bits;
// the counts are integers, so the atomics' order does not matter): the scores are read once to count their first
// digits and once to mark the tokens above the digit and collect those in it, which the rest goes over.  Each wave
// has a stretch of the tokens, so what it collects is in their order, and ties go to the lower index.
__global__ __launch_bounds__(kSelectThreads) void evict_select(const EvictArgs a)
{
    __shared__ uint32_t hist[4096], lds_sum[kSelectWaves], lds_pick[2];
    const CacheView &c = a.c;
    const uint32_t seq = blockIdx.x / c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t n = (uint32_t)min(max(load4g(c.kv_len + seq), 0), (int32_t)c.max_kv);
    const uint32_t keep = (uint32_t)max(load4g(a.keep + seq), 0);
    const Lists lists = lists_of(a, blockIdx.x);
    if (n <= keep) {
        if (tid == 0) lists.head[0] = 0, lists.head[1] = n;
        return;
    }
    const uint64_t list = (uint64_t)blockIdx.x * a.score_stride, pos_list = (uint64_t)blockIdx.x * a.pos_stride;
    const float *score = a.score_in + list;
    const int32_t *pos = a.pos_in ? a.pos_in + pos_list : nullptr;
    const bool guards = a.protect != nullptr;
    const int32_t guard = guards ? load4g(a.protect + seq) : 0;

    const uint32_t stretch = (n + kSelectThreads - 1) / kSelectThreads * 64;
    const uint32_t from = min(wave * stretch, n), to = min(from + stretch, n);
    // f(token of this lane, its key, whether there is one) for the wave's stretch, 64 tokens at a time
    auto over_keys = [&](auto f) {
        for (uint32_t i = from; i < to; i += 64 * kAhead) {
            float x[kAhead];
            int32_t p[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) x[j] = score[min(i + 64 * j + lane, to - 1)];
            if (guards && pos) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j) p[j] = pos[min(i + 64 * j + lane, to - 1)];
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const uint32_t at = i + 64 * j + lane;
                if (i + 64 * j < to) f(at, key_of(x[j], guards && (pos ? p[j] : (int32_t)at) >= guard), at < to);
            }
        }
    };

    for (int i = tid; i < 4096; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    uint32_t prefix = 0xFFFFFFFFu, left = 0, above = 0, found = 0;
    if (keep) {
        over_keys([&](uint32_t, uint32_t key, bool there) { count_digit(hist, key >> 20, there, lane); });
        __syncthreads();
        prefix = pick_digit<4>(hist, lds_sum, lds_pick, keep, tid, &above);
        left = keep - above;
    }
    // mark what is above, collect what is in the digit; with nothing to keep, no digit is looked at
    over_keys([&](uint32_t at, uint32_t key, bool there) {
        const uint64_t more = __ballot(there && keep && key >> 20 > prefix);
        const bool in = there && keep && key >> 20 == prefix;
        const uint64_t ins = __ballot(in);
        if (lane == 0) lists.kept[at >> 6] = more;
        if (in) {
            const uint32_t k = from + found + __popcll(ins & ((1ull << lane) - 1));
            lists.candidates[k] = w2{key, at};
        }
        found += __popcll(ins);
    });
    // the candidates' other digits
    for (int shift = 10; keep && shift >= 0; shift -= 10) {
        __syncthreads();
        hist[tid] = 0;
        __syncthreads();
        for (uint32_t i = 0; i < found; i += 64) {
            const uint32_t k = i + lane < found ? lists.candidates[from + i + lane][0] : 0;
            count_digit(hist, k >> shift & 1023, i + lane < found && k >> (shift + 10) == prefix, lane);
        }
        __syncthreads();
        prefix = prefix << 10 | pick_digit<1>(hist, lds_sum, lds_pick, left, tid, &above);
        left -= above;
    }
    // kept among the candidates: keys above the smallest one, and the first `left` equal to it
    uint32_t equal = 0, all;
    for (uint32_t i = 0; i < found; i += 64)
        equal += __popcll(__ballot(i + lane < found && lists.candidates[from + i + lane][0] == prefix));
    uint32_t rank = sum_before(lane ? 0 : equal, lds_sum, wave, lane, &all);
    rank = __shfl(rank, 0);
    for (uint32_t i = 0; i < found; i += 64) {
        const bool there = i + lane < found;
        const w2 one = there ? lists.candidates[from + i + lane] : w2{0, 0};
        const uint32_t key = one[0], at = one[1];
        const uint64_t same = __ballot(there && key == prefix);
        const bool kept = there && (key > prefix || (key == prefix && rank + __popcll(same & ((1ull << lane) - 1)) < left));
        rank += __popcll(same);
        if (kept) __hip_atomic_fetch_or(lists.kept + (at >> 6), 1ull << (at & 63), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __builtin_amdgcn_s_waitcnt(0);                   // the bits are set before another wave reads them
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
            uint32_t h = sum_before(__popcll(hole), lds_sum, wave, lane, &all) + holes;
            holes += all;
            for (; hole; hole &= hole - 1) lists.pairs[2 * (uint64_t)h++] = 64 * w + __ffsll((unsigned long long)hole) - 1;
        }
        if (64 * (uint64_t)(w0 + kSelectThreads) > keep) {
            uint32_t m = sum_before(__popcll(mover), lds_sum, wave, lane, &all) + movers;
            movers += all;
            for (; mover; mover &= mover - 1) lists.pairs[2 * (uint64_t)m++ + 1] = 64 * w + __ffsll((unsigned long long)mover) - 1;
        }
    }
    if (tid == 0) lists.head[0] = holes, lists.head[1] = n;   // as many as movers
    __syncthreads();
    // scores and positions of the moves; a hole's own are read by no one any more
    for (uint32_t i = tid; i < holes; i += kSelectThreads) {
        const uint32_t hole = lists.pairs[2 * (uint64_t)i], mover = lists.pairs[2 * (uint64_t)i + 1];
        const float x = score[mover];
        const int32_t p = pos ? pos[mover] : (int32_t)mover;
        a.score_out[list + hole] = x;
        if (a.pos_out) a.pos_out[pos_list + hole] = p;
    }
}

// The rows of the listed moves, 16 bytes to a lane, and what is left of scores and positions: those of the kept
// tokens that stay, where the outputs are other arrays, and the zeros past the new length.
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
    for (uint32_t u = group * 256 + threadIdx.x; u < count * pieces; u += groups * 256) {
        const uint32_t i = u / pieces, at = (u - i * pieces) * 8;
        const uint32_t hole = lists.pairs[2 * (uint64_t)i], mover = lists.pairs[2 * (uint64_t)i + 1];
        const uint32_t to = row_of(c, load4g(table + block_of(c, hole)), head, hole);
        const uint32_t from = row_of(c, load4g(table + block_of(c, mover)), head, mover);
        if (to == kNoRow || from == kNoRow) continue;
        const uint64_t d = (uint64_t)to * c.head_dim + at, s = (uint64_t)from * c.head_dim + at;
        const w4 k = load16g(a.k_cache + s), v = load16g(a.v_cache + s);
        *(w4 *)(a.k_cache + d) = k;
        *(w4 *)(a.v_cache + d) = v;
    }
    const uint64_t sl = (uint64_t)list * a.score_stride, pl = (uint64_t)list * a.pos_stride;
    const bool copies = a.score_out != a.score_in || (a.pos_out && a.pos_out != a.pos_in);
    for (uint32_t i = group * 256 + threadIdx.x; i < n; i += groups * 256) {
        if (i >= left)
            a.score_out[sl + i] = 0.0f;
        else if (copies && (n <= keep || (lists.kept[i >> 6] >> (i & 63) & 1))) {
            a.score_out[sl + i] = a.score_in[sl + i];
            if (a.pos_out) a.pos_out[pl + i] = a.pos_in ? a.pos_in[pl + i] : (int32_t)i;
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, hipStream_t stream)
{
    const uint32_t lists = a.c.n_seq * a.c.kv_heads;
    evict_select<<<lists, kSelectThreads, 0, stream>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    // about 8 workgroups to a CU, and no more than there can be rows to move
    const uint64_t most = ((uint64_t)a.c.max_kv / 2 * (a.c.head_dim / 8) + 255) / 256;
    const uint64_t groups = std::max<uint64_t>(1, std::min<uint64_t>(most, 2048 / lists));
    evict_move<<<(uint32_t)(lists * groups), 256, 0, stream>>>(a, (uint32_t)groups);
    return hipGetLastError();
}

}  // namespace kvp
