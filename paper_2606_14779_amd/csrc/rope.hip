// Rotary positions for new tokens, written to the paged cache, for gfx950 (MI355X).
//
// A pair (x, y) of a head's first `rot` elements turns by the angle of its position and frequency:
//   x' = x cos a - y sin a,   y' = y cos a + x sin a
// Pairs are (j, j + rot/2), or (2j, 2j + 1) when interleaved; the elements past `rot` stay.  One pass:
// queries go to q_out, keys and values to their pages, positions to the per-head list that eviction keeps.
// Cosines and sines come from a table made once in 64 bits (rope_table): an angle of a long context has to
// be reduced with more than 32 bits, and a table row of 4 * rot bytes serves all heads of a token.
// Products are in 32 bits, rounded once to the cache's type.

#include "wave.hpp"

namespace kvp {

namespace {

// Rotates the 8 elements at `at` of a head row x; c_s: the token's (cos, sin) pairs.
template <class T>
__device__ __forceinline__ w4 turn_piece(const uint16_t *x, uint32_t at, uint32_t rot, bool interleaved, const float *c_s)
{
    const w4 mine = load16g(x + at);
    if (at >= rot) return mine;
    w4 out;
    const uint32_t half = rot / 2;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float r[2];
        if (interleaved) {
            const uint32_t e = at + 2 * w;
            const float a = T::unpack(mine[w], 0), b = T::unpack(mine[w], 1);
            r[0] = a, r[1] = b;
            if (e < rot) {                          // rot is even: a pair is inside or outside
                const float c = c_s[e], s = c_s[e + 1];
                r[0] = __builtin_fmaf(a, c, -(b * s));
                r[1] = __builtin_fmaf(b, c, a * s);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t e = at + 2 * w + i;
                const float v = T::unpack(mine[w], i);
                r[i] = v;
                if (e < rot) {
                    const bool upper = e >= half;
                    const uint32_t j = upper ? e - half : e;
                    const float other = T::unpack(x[upper ? j : j + half], 0);
                    const float c = c_s[2 * j], s = c_s[2 * j + 1];
                    r[i] = upper ? __builtin_fmaf(v, c, other * s) : __builtin_fmaf(v, c, -(other * s));
                }
            }
        }
        out[w] = T::pack(r[0], r[1]);
    }
    return out;
}

template <class T>
__global__ __launch_bounds__(256) void rope_append(const RopeArgs a)
{
    const CacheView &c = a.c;
    const uint32_t pieces = c.head_dim / 8;
    const uint32_t q_heads = a.q ? c.heads : 0;
    const uint32_t units = (q_heads + 2 * c.kv_heads) * pieces;
    const uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint64_t token = idx / units;
    if (token >= c.total_q) return;
    const uint32_t unit = (uint32_t)(idx - token * units);
    const uint32_t at = unit % pieces * 8;
    uint32_t head = unit / pieces;
    const int32_t position = a.positions[token];
    // a position that the table does not have: NaN, so that it shows
    const bool known = position >= 0 && (uint32_t)position < a.n_positions;
    const float *c_s = a.angles + (uint64_t)(known ? position : 0) * a.rot;
    const w4 nan = {0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};
    if (head < q_heads) {
        const w4 r = turn_piece<T>(a.q + token * a.q_stride + (uint64_t)head * c.head_dim, at, a.rot, a.interleaved, c_s);
        *(w4 *)(a.q_out + token * a.q_out_stride + (uint64_t)head * c.head_dim + at) = known ? r : nan;
        return;
    }
    head -= q_heads;
    const bool value = head >= c.kv_heads;
    if (value) head -= c.kv_heads;
    // the token's sequence: the last one that begins at or before it
    uint32_t lo = 0, hi = c.n_seq;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (load4g(c.cu_q + mid) <= (int32_t)token)
            lo = mid;
        else
            hi = mid;
    }
    const Seq s = load_seq(c, lo);
    const int32_t i = (int32_t)token - s.q_begin;
    const int32_t index = s.kv - s.n_q + i;
    if (i < 0 || i >= s.n_q || index < 0) return;
    const uint32_t row =
        row_of(c, load4g(c.table + (uint64_t)lo * c.table_stride + block_of(c, index)), head, index);
    if (!value && at == 0 && a.pos) a.pos[((uint64_t)lo * c.kv_heads + head) * a.pos_stride + index] = position;
    if (row == kNoRow) return;
    if (value)
        *(w4 *)(a.v_cache + (uint64_t)row * c.head_dim + at) =
            load16g(a.v + token * a.v_stride + (uint64_t)head * c.head_dim + at);
    else {
        const w4 r = turn_piece<T>(a.k + token * a.k_stride + (uint64_t)head * c.head_dim, at, a.rot, a.interleaved, c_s);
        *(w4 *)(a.k_cache + (uint64_t)row * c.head_dim + at) = known ? r : nan;
    }
}

// cos and sin of position * frequency: revolutions in 64 bits, reduced before the functions are taken.
__global__ __launch_bounds__(256) void rope_table(const RopeTableArgs a)
{
    const uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint64_t position = idx / a.half;
    if (position >= a.n_positions) return;
    const uint32_t j = (uint32_t)(idx - position * a.half);
    double t = (double)position * a.turns[j];
    t -= rint(t);
    double s, c;
    sincospi(2.0 * t, &s, &c);
    *(v2f *)(a.angles + 2 * idx) = v2f{(float)(c * a.magnitude), (float)(s * a.magnitude)};
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, uint32_t dtype, hipStream_t stream)
{
    const uint32_t units = ((a.q ? a.c.heads : 0) + 2 * a.c.kv_heads) * (a.c.head_dim / 8);
    const uint32_t grid = (uint32_t)(((uint64_t)a.c.total_q * units + 255) / 256);
    if (dtype == KVP_BF16)
        rope_append<BF16><<<grid, 256, 0, stream>>>(a);
    else
        rope_append<F16><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_rope_table(const RopeTableArgs &a, hipStream_t stream)
{
    const uint32_t grid = (uint32_t)(((uint64_t)a.n_positions * a.half + 255) / 256);
    rope_table<<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace kvp
