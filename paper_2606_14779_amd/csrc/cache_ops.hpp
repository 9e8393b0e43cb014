// Operators on the engine's paged cache: what their host side (cache_ops.cpp)
// and their kernels (attention.hip, rope.hip, evict.hip) share.
#ifndef KVP_CACHE_OPS_HPP
#define KVP_CACHE_OPS_HPP

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "kvpool.h"

namespace kvp {

// One layer's cache and the batch over it, as the kernels see them.
struct CacheView {
    const int32_t *cu_q, *kv_len, *table;
    uint32_t n_seq, total_q, max_q, max_kv, table_stride;
    uint32_t num_slots, heads, kv_heads, group, head_dim, block;
    // x / block = (2 x * magic) >> 32 >> shift for x below 2^31, and the same for group
    uint32_t block_magic, block_shift, group_magic, group_shift;
};
constexpr uint32_t kNoRow = 0xFFFFFFFFu;

struct AttentionArgs {
    CacheView c;
    const uint16_t *q, *k, *v;
    uint64_t q_stride, out_stride;   // elements between tokens
    uint16_t *out;
    float *lse;                      // [heads][total_q] or null
    const float *sinks;              // [heads] or null
    float scale_log2;                // scale * log2(e)
    uint32_t window;                 // 0: none
    uint32_t few_rows;               // attention_few, else attention_rows
    uint32_t tiles, splits, split_keys;
    float *part_o;                   // [splits][total_q * heads][head_dim]
    float *part_ml;                  // [splits][total_q * heads][2]
};

struct MassArgs {
    CacheView c;
    const uint16_t *q, *k;
    uint64_t q_stride;
    const float *lse, *score_in;
    float *score_out;
    float scale_log2;
    uint32_t window, last, score_stride;
};

struct RopeArgs {
    CacheView c;
    const float *angles;             // [n_positions][rot / 2][2]
    const int32_t *positions;
    uint32_t n_positions, rot, interleaved;
    uint32_t per_head, per_magic, per_shift;   // units of a rotated head, and its division
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_cache, *v_cache;
    uint64_t q_stride, q_out_stride, k_stride, v_stride;
    int32_t *pos;
    uint32_t pos_stride;
};

constexpr uint32_t kMostRotary = 256;   // rotated elements of a head
struct RopeTableArgs {
    float *angles;
    uint32_t n_positions, half;
    double magnitude;
    double turns[kMostRotary / 2];   // revolutions per position
};

struct EvictArgs {
    CacheView c;
    const int32_t *keep, *protect;   // protect: null = none
    const float *score_in;
    float *score_out;
    const int32_t *pos_in;           // null: a token's position is its index
    int32_t *pos_out;
    uint32_t score_stride, pos_stride;
    uint16_t *k_cache, *v_cache;
    int32_t *len_out;
    uint32_t *moves;                 // [n_seq * kv_heads][list_words]
    uint64_t list_words;
};

// Each launcher enqueues on `stream` of the current device.
hipError_t launch_attention(const AttentionArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_attention_join(const AttentionArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_mass(const MassArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_rope(const RopeArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_rope_table(const RopeTableArgs &a, hipStream_t stream);
hipError_t launch_evict(const EvictArgs &a, hipStream_t stream);

// Rows (new tokens times the heads of a KV head) and keys of the attention kernels' tiles.
constexpr uint32_t kFewRows = 16;
// 32 rows to a wave, two waves to a SIMD; at a head_dim of more than 128 the registers hold one.
constexpr int row_waves(uint32_t head_dim) { return head_dim > 128 ? 4 : 8; }
constexpr uint32_t kTileKeys = 64;

// Eviction: tokens that one workgroup holds in registers, and the workgroups that a longer list is spread over.
constexpr uint32_t kEvictShort = 8192;
constexpr uint32_t kEvictParts = 32;

}  // namespace kvp

#endif
