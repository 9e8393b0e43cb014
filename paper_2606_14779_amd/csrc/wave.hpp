// Device helpers of the matrix kernels: element types, MFMA operands, transposed
// LDS reads and the two-halves exchanges of a 64-lane wavefront (gfx950).
//
// Operand layouts, lane l:
//   32x32x16  A: row l%32, k = 8*(l/32)..+7   B: column l%32, same k
//             C: column l%32, register r holds row 8*(r/4) + 4*(l/32) + r%4
//   16x16x32  A: row l%16, k = 8*(l/16)..+7   B: column l%16, same k
//             C: column l%16, register r holds row 4*(l/16) + r
#ifndef KVP_WAVE_HPP
#define KVP_WAVE_HPP

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_ops.hpp"

namespace kvp {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t w4 __attribute__((ext_vector_type(4)));
typedef uint32_t w2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) const w4 gw4;
typedef __attribute__((address_space(1))) const int32_t gi32;

// Whether eight 16-bit floats of this exponent are all finite.
__device__ __forceinline__ bool finite_to(w4 x, uint32_t exponent)
{
    bool all = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) all &= (x[i] & exponent) != exponent && (x[i] >> 16 & exponent) != exponent;
    return all;
}

// Puts 0 in the place of those that are not; whether there were none.
__device__ __forceinline__ bool bound_to(w4 &x, uint32_t exponent)
{
    const bool all = finite_to(x, exponent);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((x[i] & exponent) == exponent) x[i] &= 0xFFFF0000u;
        if ((x[i] >> 16 & exponent) == exponent) x[i] &= 0xFFFFu;
    }
    return all;
}

// kLift: what the reference point of a row's weights lies below their maximum, in powers of two (see the softmax).
struct BF16 {
    static constexpr float kLift = 0.0f;
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ v16f mma32(w4 a, w4 b, v16f c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ v4f mma16(w4 a, w4 b, v4f c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)   // to nearest even
    {
        const v2f f = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, x2));
    }
    static __device__ __forceinline__ float unpack(uint32_t w, int i)
    {
        return __builtin_bit_cast(float, i ? (w & 0xFFFF0000u) : (w << 16));
    }
    static __device__ __forceinline__ bool finite(w4 x) { return finite_to(x, 0x7F80u); }
    static __device__ __forceinline__ bool bound(w4 &x) { return bound_to(x, 0x7F80u); }
};

struct F16 {
    static constexpr float kLift = 7.0f;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ v16f mma32(w4 a, w4 b, v16f c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ v4f mma16(w4 a, w4 b, v4f c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)   // to nearest even
    {
        const v2f f = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, x2));
    }
    static __device__ __forceinline__ float unpack(uint32_t w, int i)
    {
        return (float)__builtin_bit_cast(x2, w)[i];
    }
    static __device__ __forceinline__ bool finite(w4 x) { return finite_to(x, 0x7C00u); }
    static __device__ __forceinline__ bool bound(w4 &x) { return bound_to(x, 0x7C00u); }
};

__device__ __forceinline__ w4 load16g(const uint16_t *p) { return *(gw4 *)p; }
__device__ __forceinline__ w2 load8g(const uint16_t *p) { return *(__attribute__((address_space(1))) const w2 *)p; }
__device__ __forceinline__ int32_t load4g(const int32_t *p) { return *(gi32 *)p; }

// Orders a wave's own accesses of LDS, which the hardware keeps in order, for the compiler.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four 16-bit elements down a column: within 16 lanes, lane i names 4 elements of row i/4
// (columns 4*(i%4)..+3 of a 4x16 tile) and receives column i of the tile's four rows.
__device__ __forceinline__ w2 read_down(const uint16_t *lds)
{
    return __builtin_bit_cast(w2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)lds));
}

// The other 32 lanes' value.
__device__ __forceinline__ float other_half(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);   // p[0]: low halves twice, p[1]: high halves twice
    return __builtin_bit_cast(float, (uint32_t)(threadIdx.x & 32 ? p[0] : p[1]));
}

// Another lane's value.
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return __shfl(x, lane); }
__device__ __forceinline__ uint64_t lane_value(uint64_t x, int lane)
{
    return (uint64_t)(uint32_t)__shfl((uint32_t)(x >> 32), lane) << 32 | (uint32_t)__shfl((uint32_t)x, lane);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kLowest = -3.0e38f;        // start of a running maximum: finite, so that -inf minus it is -inf
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// A sequence of a batch.  Device arrays are not trusted: lengths are clamped to what the host was told.
struct Seq {
    int32_t q_begin, n_q, kv;
};
__device__ __forceinline__ Seq load_seq(const CacheView &c, uint32_t s)
{
    const int32_t total = (int32_t)c.total_q;
    const int32_t b = min(max(load4g(c.cu_q + s), 0), total);
    const int32_t e = min(max(load4g(c.cu_q + s + 1), b), total);
    const int32_t kv = min(max(load4g(c.kv_len + s), 0), (int32_t)c.max_kv);
    return {b, min(e - b, (int32_t)c.max_q), kv};
}

// Row number (of head_dim elements) of a sequence's cached token, or kNoRow where its slot is none of the cache's.
__device__ __forceinline__ uint32_t block_of(const CacheView &c, uint32_t token)
{
    return __umulhi(2 * token, c.block_magic) >> c.block_shift;
}
__device__ __forceinline__ uint32_t row_of(const CacheView &c, int32_t slot, uint32_t kv_head, uint32_t token)
{
    const uint32_t off = token - block_of(c, token) * c.block;
    return (uint32_t)slot < c.num_slots ? ((uint32_t)slot * c.kv_heads + kv_head) * c.block + off : kNoRow;
}

// New token of a KV head's row (its rows are token-major).
__device__ __forceinline__ uint32_t token_of(const CacheView &c, uint32_t row)
{
    return __umulhi(2 * row, c.group_magic) >> c.group_shift;
}

// All loads so far have arrived (vmcnt 0): said before a loop, so that the loop does not wait for its own prefetches
// on behalf of loads that were issued before it.
__device__ __forceinline__ void loads_arrived() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// Sequence of a row tile: sequence s owns the tiles from floor(rows before it / tile) + s on, at least as many
// as its rows need, so no prefix of tile counts has to be made.
__device__ __forceinline__ uint32_t first_tile(const CacheView &c, uint32_t s, uint32_t tile_rows)
{
    const uint32_t before = (uint32_t)min(max(load4g(c.cu_q + s), 0), (int32_t)c.total_q);
    return (uint32_t)((uint64_t)before * c.group / tile_rows) + s;
}
__device__ __forceinline__ uint32_t seq_of_tile(const CacheView &c, uint32_t tile, uint32_t tile_rows)
{
    uint32_t lo = 0, hi = c.n_seq;              // first_tile(lo) <= tile < first_tile(hi)
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (first_tile(c, mid, tile_rows) <= tile)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Inclusive sum over the lanes up to this one, within the vector unit.
__device__ __forceinline__ uint32_t sum_upto(uint32_t x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);   // the lane 1 below in a row of 16, then 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // a row's last lane to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // lane 31 to the upper half
    return x;
}

// The rank-th longest row tile of a batch of up to 64 sequences: tiles of tile_rows rows (of a KV head) by the keys
// that a causal mask leaves them, in units of `keys`; of equal ones the earlier sequence's first.  Workgroups begin
// in this order, so that none with much to do begins last.  Ranks past the last tile give tile == none.
struct Tile {
    uint32_t seq, tile;
    Seq s;
};
constexpr uint32_t kNoTile = 0xFFFFFFFFu;
__device__ __forceinline__ Tile tile_by_length(const CacheView &c, uint32_t rank, uint32_t tile_rows, uint32_t keys)
{
    const uint32_t lane = threadIdx.x & 63;
    Seq s = load_seq(c, min(lane, c.n_seq - 1));
    if (lane >= c.n_seq) s.n_q = 0;
    const uint32_t tiles = (uint32_t)(((uint64_t)s.n_q * c.group + tile_rows - 1) / tile_rows);
    // tiles of this lane's sequence with x or more units of keys: those whose last token sees key (x - 1) * keys
    auto at_least = [&](uint32_t x) {
        const int64_t token = ((int64_t)x - 1) * keys - (s.kv - s.n_q);
        if (x == 0 || token <= 0) return tiles;
        return token >= s.n_q ? 0u : tiles - (uint32_t)((uint64_t)token * c.group / tile_rows);
    };
    auto all = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane(sum_upto(x), 63); };
    if (rank >= all(tiles)) return {0, kNoTile, s};
    uint32_t lo = 0, hi = c.max_kv / keys + 2;       // all(at_least(lo)) > rank >= all(at_least(hi))
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (all(at_least(mid)) > rank)
            lo = mid;
        else
            hi = mid;
    }
    const uint32_t longer = at_least(hi), these = at_least(lo) - longer;
    const uint32_t left = rank - all(longer), upto = sum_upto(these);
    const uint64_t found = __ballot(upto > left);
    const int who = __ffsll((unsigned long long)found) - 1;
    auto from = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane(x, who); };
    s = {(int32_t)from(s.q_begin), (int32_t)from(s.n_q), (int32_t)from(s.kv)};
    return {(uint32_t)who, from(tiles) - from(longer + these) + left - (from(upto) - from(these)), s};
}

}  // namespace kvp

#endif
