// Operators on the engine's paged cache: what their host side (cache_ops.cpp)
// and their kernels (attention.hip, rope.hip, evict.hip, attention_tree.hip, attention_e4m3.hip, pages.hip) share.
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

// Pages of either kind: slots of 16-bit elements, or of bytes with a power of two to 32 of them.
struct PageView {
    uint8_t *k, *v;
    uint64_t slot_bytes;
    uint32_t exponents;              // where a slot's exponents begin; 0: 16-bit elements
    uint32_t row_exponents;          // bytes of exponents to a row
    uint32_t num_slots;
};

struct AttentionArgs {
    CacheView c;
    const uint16_t *q, *k, *v;       // k, v: of 8-bit pages too, by bytes
    uint64_t q_stride, out_stride;   // elements between tokens
    uint16_t *out;
    float *lse;                      // [heads][total_q] or null
    const float *sinks;              // [heads] or null
    float scale_log2;                // scale * log2(e)
    uint32_t window;                 // 0: none
    uint32_t few_rows;               // most rows of a sequence where the waves split the keys; 0: attention_rows
    uint32_t tiles, splits, split_keys;
    uint32_t uneven;                 // sequences of different lengths, whose parts are not all there; for attention_rows
                                     // splits is a bound and split_keys is found by the lengths
    float *part_o;                   // [splits][total_q * heads][head_dim]
    float *part_ml;                  // [splits][total_q * heads][2]
    // of attention over pages alone
    uint32_t exponents, row_exponents;   // of 8-bit pages; 0: 16-bit elements
    uint64_t slot_bytes;
    const uint64_t *tree;            // [total_q][tree_words] or null
    uint32_t tree_words;
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
constexpr uint32_t kMostAxes = 4;
struct AppendArgs {
    CacheView c;
    PageView pages;
    const float *angles;             // [n_positions][rot / 2][2]
    const int32_t *positions;        // [axes][total_q]
    uint32_t n_positions, rot, interleaved, axes;
    uint32_t lanes_log2;             // lanes to a head: 8 elements each
    uint32_t norm;                   // whether queries and keys are normed
    float eps, per_dim;              // 1 / head_dim
    const uint16_t *q_weight, *k_weight;   // null: ones
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    uint64_t q_stride, q_out_stride, k_stride, v_stride;
    int32_t *pos;
    uint32_t pos_stride;
    uint8_t axis_of[kMostRotary / 2];
};

struct ConvertArgs {
    CacheView c;
    PageView from, to;
    const int32_t *to_table, *first; // first: null = 0
    uint32_t to_stride, lanes_log2;
};

struct CommitArgs {
    CacheView c;
    PageView pages;
    const int32_t *path, *accepted;
    int32_t *pos, *len_out;          // len_out: null = by a launch of its own
    uint32_t pos_stride, lanes_log2;
};
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
hipError_t launch_attention_e4m3(const AttentionArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_attention_tree(const AttentionArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_append(const AppendArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_convert(const ConvertArgs &a, uint32_t dtype, hipStream_t stream);
hipError_t launch_commit(const CommitArgs &a, hipStream_t stream);
hipError_t launch_commit_lengths(const CommitArgs &a, int32_t *len_out, hipStream_t stream);

// Rows (new tokens times the heads of a KV head) and keys of the attention kernels' tiles.
constexpr uint32_t kFewRows = 16;
// 32 rows to a wave, two waves to a SIMD; at a head_dim of more than 128 the registers hold one.
constexpr int row_waves(uint32_t head_dim) { return head_dim > 128 ? 4 : 8; }
constexpr uint32_t kTileKeys = 64;
// Rows of a sequence up to which attention over pages has its waves split the keys.
constexpr uint32_t some_rows(uint32_t head_dim) { return head_dim > 128 ? 32 : 64; }

constexpr uint32_t kConvertTokens = 64;    // to a workgroup

// Eviction: tokens that one workgroup holds in registers, and the workgroups that a longer list is spread over.
constexpr uint32_t kEvictShort = 8192;
constexpr uint32_t kEvictParts = 32;

}  // namespace kvp

#endif
