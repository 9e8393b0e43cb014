// Rotary positions for new tokens, written to the paged cache, for gfx950 (MI355X).
//
// A pair (x, y) of a head's first `rot` elements turns by the angle of its position and frequency:
//   x' = x cos a - y sin a,   y' = y cos a + x sin a
// Pairs are (j, j + rot/2), or (2j, 2j + 1) when interleaved; the elements past `rot` stay.  One pass:
// queries go to q_out, keys and values to their pages, positions to the per-head list that eviction keeps.
// Cosines and sines come from a table made once in 64 bits (rope_table): an angle of a long context has to
// be reduced with more than 32 bits, and a table row of 4 * rot bytes serves all heads of a token.
// Products are in 32 bits, rounded once to the cache's type.
//
// Bound by memory: packed prompts of 12.7K tokens (64 heads, 8 KV heads, 64; pairs interleaved) take 51 us, 263 MB at 5.1
// TB/s, where inputs change from call to call (44 us on the same ones again); of 12.3K (32, 8, 128; pairs in halves) 53 us
// on the same ones, 302 MB at 5.7 TB/s, where a copy moves 6.1.  A table of 128K positions of 64 pairs takes 32 us, for 64-bit
// sines and cosines of 67 MB that a copy would write in 11.  A decoding step of 32 tokens takes 3.7 us on the GPU, a chain of four dependent loads.

#include "wave.hpp"

namespace kvp {

namespace {

// How the pairs lie: 8 of them in the same 16 bytes, in two pieces of 16 bytes, or anyhow.
enum Pairs { kInside, kApart, kAnyhow };

// Rotates the 8 elements at `at` of a head row x, wherever their partners are; c_s: the token's (cos, sin) pairs.
template <class T>
__device__ __forceinline__ w4 turn_anyhow(const uint16_t *x, uint32_t at, uint32_t rot, bool interleaved, const float *c_s)
{
    const w4 mine = load16g(x + at);
    w4 out;
    const uint32_t half = rot / 2;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float r[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t e = at + 2 * w + i;
            const float v = T::unpack(mine[w], i);
            r[i] = v;
            if (e < rot) {                          // rot is even: a pair is inside or outside
                const bool upper = interleaved ? e & 1 : e >= half;
                const uint32_t j = interleaved ? e / 2 : upper ? e - half : e;
                const float other = T::unpack(x[interleaved ? e ^ 1 : upper ? j : j + half], 0);
                const float c = c_s[2 * j], s = c_s[2 * j + 1];
                r[i] = upper ? __builtin_fmaf(v, c, other * s) : __builtin_fmaf(v, c, -(other * s));
            }
        }
        out[w] = T::pack(r[0], r[1]);
    }
    return out;
}

// Four floats of a table, which is 8-byte aligned.
typedef float v4f_at8 __attribute__((ext_vector_type(4), aligned(8)));
__device__ __forceinline__ v4f load4f(const float *p) { return *(__attribute__((address_space(1))) const v4f_at8 *)p; }

// A token to a workgroup.  What it loads and stores of its heads does not wait for its place in the cache: that
// takes a search among the sequences, their lengths and the block table, one after the other.
template <class T, int PAIRS>
__global__ __launch_bounds__(256) void rope_append(const RopeArgs a)
{
    const CacheView &c = a.c;
    const uint32_t token = blockIdx.x;
    const int lane = threadIdx.x & 63;
    const uint32_t q_heads = a.q ? c.heads : 0, pieces = c.head_dim / 8;
    // units of a rotated head: pairs of pieces where they lie apart, else pieces
    const uint32_t pairs = PAIRS == kApart ? a.rot / 16 : 0;
    const uint32_t turned = (q_heads + c.kv_heads) * a.per_head, units = turned + c.kv_heads * pieces;

    const int32_t position = load4g(a.positions + token);
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
    // a position that the table does not have: NaN, so that it shows
    const bool known = position >= 0 && (uint32_t)position < a.n_positions;
    const float *c_s = a.angles + (uint64_t)(known ? position : 0) * a.rot;
    const w4 nan = {0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};

    for (uint32_t unit = threadIdx.x; unit < units; unit += blockDim.x) {
        if (unit >= turned) {                        // values
            const uint32_t head = (unit - turned) / pieces, at = (unit - turned - head * pieces) * 8;
            const w4 x = load16g(a.v + token * a.v_stride + (uint64_t)head * c.head_dim + at);
            const uint32_t row = row_of(c, slot, head, max(index, 0));
            if (row != kNoRow) *(w4 *)(a.v_cache + (uint64_t)row * c.head_dim + at) = x;
            continue;
        }
        uint32_t head = __umulhi(2 * unit, a.per_magic) >> a.per_shift;
        const uint32_t u = unit - head * a.per_head;
        const bool query = head < q_heads;
        head -= query ? 0 : q_heads;
        const uint16_t *x = (query ? a.q + token * a.q_stride : a.k + token * a.k_stride) + (uint64_t)head * c.head_dim;
        const uint32_t at = (u < pairs ? u : u + pairs) * 8, partner = at + a.rot / 2;
        w4 low, high{};
        if constexpr (PAIRS == kAnyhow) {
            low = at < a.rot ? turn_anyhow<T>(x, at, a.rot, a.interleaved, c_s) : load16g(x + at);
        } else if constexpr (PAIRS == kInside) {
            low = load16g(x + at);
            if (at < a.rot) {
                const v4f f0 = load4f(c_s + at), f1 = load4f(c_s + at + 4);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float cos = w < 2 ? f0[2 * w] : f1[2 * w - 4], sin = w < 2 ? f0[2 * w + 1] : f1[2 * w - 3];
                    const float p = T::unpack(low[w], 0), q = T::unpack(low[w], 1);
                    low[w] = T::pack(__builtin_fmaf(p, cos, -(q * sin)), __builtin_fmaf(q, cos, p * sin));
                }
            }
        } else {
            low = load16g(x + at);
            if (u < pairs) {
                high = load16g(x + partner);
                v4f f[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) f[w] = load4f(c_s + 2 * at + 4 * w);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float p0 = T::unpack(low[w], 0), p1 = T::unpack(low[w], 1);
                    const float q0 = T::unpack(high[w], 0), q1 = T::unpack(high[w], 1);
                    low[w] = T::pack(__builtin_fmaf(p0, f[w][0], -(q0 * f[w][1])), __builtin_fmaf(p1, f[w][2], -(q1 * f[w][3])));
                    high[w] = T::pack(__builtin_fmaf(q0, f[w][0], p0 * f[w][1]), __builtin_fmaf(q1, f[w][2], p1 * f[w][3]));
                }
            }
        }
        if (!known) low = high = nan;
        uint16_t *to;
        if (query) {
            to = a.q_out + token * a.q_out_stride + (uint64_t)head * c.head_dim;
        } else {
            if (u == 0 && a.pos && placed) a.pos[((uint64_t)seq * c.kv_heads + head) * a.pos_stride + index] = position;
            const uint32_t row = row_of(c, slot, head, max(index, 0));
            if (row == kNoRow) continue;
            to = a.k_cache + (uint64_t)row * c.head_dim;
        }
        *(w4 *)(to + at) = low;
        if (u < pairs) *(w4 *)(to + partner) = high;
    }
}

// cos and sin of position * frequency: revolutions in 64 bits, reduced before the functions are taken.
__global__ __launch_bounds__(256) void rope_table(const RopeTableArgs a)
{
    const uint64_t pairs = (uint64_t)a.n_positions * a.half;
    for (uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x; idx < pairs; idx += (uint64_t)gridDim.x * 256) {
        const uint64_t position = idx / a.half;
        const uint32_t j = (uint32_t)(idx - position * a.half);
        double t = (double)position * a.turns[j];
        t -= rint(t);
        double s, c;
        sincospi(2.0 * t, &s, &c);
        *(v2f *)(a.angles + 2 * idx) = v2f{(float)(c * a.magnitude), (float)(s * a.magnitude)};
    }
}

}  // namespace

template <class T>
static hipError_t launch_rope_as(const RopeArgs &a, hipStream_t stream)
{
    // whole wavefronts, as many as a token's units fill, up to four
    const uint32_t units = ((a.q ? a.c.heads : 0) + a.c.kv_heads) * a.per_head + a.c.kv_heads * (a.c.head_dim / 8);
    const uint32_t threads = units >= 256 ? 256 : (units + 63) / 64 * 64;
    if (a.interleaved ? a.rot % 8 == 0 : a.rot == 0)
        rope_append<T, kInside><<<a.c.total_q, threads, 0, stream>>>(a);
    else if (!a.interleaved && a.rot % 16 == 0)
        rope_append<T, kApart><<<a.c.total_q, threads, 0, stream>>>(a);
    else
        rope_append<T, kAnyhow><<<a.c.total_q, threads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_rope(const RopeArgs &a, uint32_t dtype, hipStream_t stream)
{
    return dtype == KVP_BF16 ? launch_rope_as<BF16>(a, stream) : launch_rope_as<F16>(a, stream);
}

hipError_t launch_rope_table(const RopeTableArgs &a, hipStream_t stream)
{
    // a pair to a thread; a launch has less than 2^32 threads, larger tables are gone over in steps
    const uint64_t groups = ((uint64_t)a.n_positions * a.half + 255) / 256;
    rope_table<<<(uint32_t)(groups < 1u << 22 ? groups : 1u << 22), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace kvp
