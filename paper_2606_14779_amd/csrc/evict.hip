// Eviction from the paged cache by score, for gfx950 (MI355X).
//
// A sequence of n tokens keeps, for every KV head by itself, the `keep` tokens of largest key: protected
// tokens first, then by score, then by lower index; a NaN score counts below every number.  Kept tokens at
// index >= keep move into the places below keep that fell free, both in ascending order.  No source is a
// destination, so the moves need no order among themselves and the cache is compacted in place; and since
// attention does not depend on the order of the keys before the new ones, nothing else has to move.

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

__device__ __forceinline__ uint32_t sum_of_waves(uint32_t *lds, uint32_t mine, int wave, int lane, uint32_t *before)
{
    if (lane == 0) lds[wave] = mine;
    __syncthreads();
    uint32_t all = 0, b = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        b = w == wave ? all : b;
        all += lds[w];
    }
    __syncthreads();
    *before = b;
    return all;
}

// One workgroup to a sequence and KV head: finds the smallest kept key digit by digit (the counts are
// integers, so the atomics' order does not matter), then lists the moves in order, each wave over a
// stretch of its own.
__global__ __launch_bounds__(kSelectThreads) void evict_select(const EvictArgs a)
{
    __shared__ uint32_t hist[kSelectWaves][256], lds_sum[kSelectWaves], lds_pick[2];
    const CacheView &c = a.c;
    const uint32_t head = blockIdx.x % c.kv_heads, seq = blockIdx.x / c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t n = (uint32_t)min(max(load4g(c.kv_len + seq), 0), (int32_t)c.max_kv);
    const uint32_t keep = (uint32_t)max(load4g(a.keep + seq), 0);
    const uint64_t list = (uint64_t)blockIdx.x * a.score_stride, pos_list = (uint64_t)blockIdx.x * a.pos_stride;
    const float *score = a.score_in + list;
    float *score_out = a.score_out + list;
    const int32_t *pos = a.pos_in ? a.pos_in + pos_list : nullptr;
    int32_t *pos_out = a.pos_out ? a.pos_out + pos_list : nullptr;
    uint32_t *moves = a.moves + (uint64_t)blockIdx.x * (2 + 2 * a.room);
    const int32_t guard = a.protect ? load4g(a.protect + seq) : 0x7FFFFFFF;
    const bool guards = a.protect != nullptr;

    auto pos_at = [&](uint32_t i) { return pos ? pos[i] : (int32_t)i; };
    auto key_at = [&](uint32_t i) { return key_of(score[i], guards && pos_at(i) >= guard); };

    if (n <= keep) {
        if (tid == 0) moves[0] = 0;
        for (uint32_t i = tid; i < n; i += kSelectThreads) {
            const float x = score[i];
            const int32_t p = pos_at(i);
            score_out[i] = x;
            if (pos_out) pos_out[i] = p;
        }
        return;
    }
    uint32_t prefix = 0, mask = 0, left = keep;      // the kept keys that are still to be found, from the largest
    for (int shift = 24; keep && shift >= 0; shift -= 8) {
        for (int i = tid; i < kSelectWaves * 256; i += kSelectThreads) (&hist[0][0])[i] = 0;
        __syncthreads();
        for (uint32_t i = tid; i < n; i += kSelectThreads) {
            const uint32_t k = key_at(i);
            if ((k & mask) == prefix) atomicAdd(&hist[wave][k >> shift & 255], 1u);
        }
        __syncthreads();
        if (tid < 256) {
            uint32_t sum = 0;
#pragma unroll
            for (int w = 0; w < kSelectWaves; ++w) sum += hist[w][tid];
            hist[0][tid] = sum;
        }
        __syncthreads();
        if (tid == 0) {
            uint32_t d = 255, above = 0;
            while (d > 0 && above + hist[0][d] < left) above += hist[0][d--];
            lds_pick[0] = d;
            lds_pick[1] = above;
        }
        __syncthreads();
        prefix |= lds_pick[0] << shift;
        mask |= 255u << shift;
        left -= lds_pick[1];
        __syncthreads();
    }
    // kept: key > prefix, and the first `left` of those equal to it (none where keep is 0)
    const uint32_t stretch = ((n + kSelectThreads - 1) / kSelectThreads) * 64;
    const uint32_t from = min(wave * stretch, n), to = min(from + stretch, n);
    uint32_t equal = 0;
    for (uint32_t i = from; i < to; i += 64) {
        const uint32_t at = i + lane;
        equal += __popcll(__ballot(keep && at < to && key_at(at) == prefix));
    }
    uint32_t equal_before;
    sum_of_waves(lds_sum, equal, wave, lane, &equal_before);
    const uint64_t below = (1ull << lane) - 1;

    uint32_t holes = 0, movers = 0, holes_before = 0, movers_before = 0, count = 0;
    for (int write = 0; write < 2; ++write) {
        uint32_t e = equal_before;
        uint32_t h = holes_before, v = movers_before;
        for (uint32_t i = from; i < to; i += 64) {
            const uint32_t at = i + lane;
            const uint32_t k = at < to ? key_at(at) : 0;
            const bool same = keep && at < to && k == prefix;
            const uint64_t sames = __ballot(same);
            const bool kept = at < to && keep && (k > prefix || (same && e + __popcll(sames & below) < left));
            e += __popcll(sames);
            const uint64_t hb = __ballot(at < to && at < keep && !kept), vb = __ballot(kept && at >= keep);
            if (write) {
                if (hb >> lane & 1) moves[2 + 2 * (h + __popcll(hb & below))] = at;
                if (vb >> lane & 1) moves[3 + 2 * (v + __popcll(vb & below))] = at;
            }
            h += __popcll(hb);
            v += __popcll(vb);
        }
        if (!write) {
            holes = h;
            movers = v;
            count = sum_of_waves(lds_sum, holes, wave, lane, &holes_before);
            sum_of_waves(lds_sum, movers, wave, lane, &movers_before);
        }
    }
    if (tid == 0) moves[0] = count;
    __syncthreads();                                 // the list is whole, and every score has been read as a key
    for (uint32_t i = tid; i < count; i += kSelectThreads) {
        const uint32_t hole = moves[2 + 2 * i], mover = moves[3 + 2 * i];
        const float x = score[mover];
        const int32_t p = pos_at(mover);
        // a hole's own score and position are read by no one any more
        score_out[hole] = x;
        if (pos_out) pos_out[hole] = p;
    }
    __syncthreads();
    if (score_out != score || (pos_out && pos_out != pos)) {
        // the kept ones that stay: everything below keep that is no hole.  Holes are in ascending order: look one up
        for (uint32_t i = tid; i < min(keep, n); i += kSelectThreads) {
            uint32_t lo = 0, hi = count;
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (moves[2 + 2 * mid] < i)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            if (lo < count && moves[2 + 2 * lo] == i) continue;
            score_out[i] = score[i];
            if (pos_out) pos_out[i] = pos_at(i);
        }
    }
    for (uint32_t i = keep + tid; i < n; i += kSelectThreads) score_out[i] = 0.0f;
}

// The rows of the listed moves, 16 bytes to a lane.
__global__ __launch_bounds__(256) void evict_move(const EvictArgs a, const uint32_t groups)
{
    const CacheView &c = a.c;
    const uint32_t list = blockIdx.x / groups, head = list % c.kv_heads, seq = list / c.kv_heads;
    const uint32_t *moves = a.moves + (uint64_t)list * (2 + 2 * a.room);
    const uint32_t pieces = c.head_dim / 8, count = min(moves[0], a.room);
    const int32_t *table = c.table + (uint64_t)seq * c.table_stride;
    if (blockIdx.x % groups == 0 && head == 0 && threadIdx.x == 0) {
        // written here, where no workgroup reads lengths any more: it may be the same array
        const int32_t n = min(max(load4g(c.kv_len + seq), 0), (int32_t)c.max_kv);
        a.len_out[seq] = min(n, max(load4g(a.keep + seq), 0));
    }
    for (uint32_t u = (blockIdx.x % groups) * 256 + threadIdx.x; u < count * pieces; u += groups * 256) {
        const uint32_t i = u / pieces, at = (u - i * pieces) * 8;
        const uint32_t hole = moves[2 + 2 * i], mover = moves[3 + 2 * i];
        const uint32_t to = row_of(c, load4g(table + block_of(c, hole)), head, hole);
        const uint32_t from = row_of(c, load4g(table + block_of(c, mover)), head, mover);
        if (to == kNoRow || from == kNoRow) continue;
        const uint64_t d = (uint64_t)to * c.head_dim + at, s = (uint64_t)from * c.head_dim + at;
        const w4 k = load16g(a.k_cache + s), v = load16g(a.v_cache + s);
        *(w4 *)(a.k_cache + d) = k;
        *(w4 *)(a.v_cache + d) = v;
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, hipStream_t stream)
{
    const uint32_t lists = a.c.n_seq * a.c.kv_heads;
    evict_select<<<lists, kSelectThreads, 0, stream>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const uint64_t most = (uint64_t)a.room * (a.c.head_dim / 8);
    uint64_t groups = (2048 + lists - 1) / lists;
    if (groups > (most + 255) / 256) groups = (most + 255) / 256;
    if (!groups) groups = 1;
    evict_move<<<(uint32_t)(lists * groups), 256, 0, stream>>>(a, (uint32_t)groups);
    return hipGetLastError();
}

}  // namespace kvp
