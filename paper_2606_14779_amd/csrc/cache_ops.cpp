// Host side of the operators on the paged cache: argument checks and launch rules.  The C entry points are in abi.cpp.

#include "cache_ops.hpp"

#include <algorithm>
#include <cmath>
#include <string>

#include "internal.hpp"

namespace kvp {

namespace {

void need(bool ok, const char *what)
{
    if (!ok) fail(KVP_ERR_INVALID, what);
}

bool aligned(const void *p, uintptr_t to) { return !(reinterpret_cast<uintptr_t>(p) & (to - 1)); }

void need_pointer(const void *p, uintptr_t align, const char *what)
{
    if (!p) fail(KVP_ERR_INVALID, std::string(what) + " is null");
    if (!aligned(p, align)) fail(KVP_ERR_INVALID, std::string(what) + " is not aligned to " + std::to_string(align) + " bytes");
}

// x / d for x below 2^31 as (2 x * magic) >> 32 >> shift: with 2^(shift - 1) < d <= 2^shift and
// magic = ceil(2^(31 + shift) / d), the product is too large by less than x / 2^31 / d, so by less than 1 / d.
void divide_by(uint32_t d, uint32_t *magic, uint32_t *shift)
{
    *shift = 0;
    while ((1u << *shift) < d) ++*shift;
    *magic = (uint32_t)(((1ull << (31 + *shift)) + d - 1) / d);
}

// What a launch's grid can count, with room: new tokens times query heads, sequences times KV heads, parts of a call.
constexpr uint64_t kMostRows = 1ull << 29, kMostLists = 1ull << 18, kMostParts = 1ull << 22;

// Checks the shape and the batch; queries says whether cu_q is used, arrays whether the batch's arrays are (a workspace
// is asked for by sizes alone).
CacheView view_of(const kvp_cache_shape *s, const kvp_batch *b, bool queries, bool arrays = true)
{
    need(s && b, "null argument");
    need(s->dtype == KVP_BF16 || s->dtype == KVP_F16, "dtype is neither KVP_BF16 nor KVP_F16");
    need(s->num_kv_heads > 0 && s->num_q_heads > 0, "no heads");
    need(s->num_q_heads % s->num_kv_heads == 0, "num_q_heads is no multiple of num_kv_heads");
    need(s->head_dim >= 8 && s->head_dim <= 256 && s->head_dim % 8 == 0, "head_dim is no multiple of 8 up to 256");
    need(s->block_size > 0, "block_size is 0");
    need(s->num_slots > 0, "num_slots is 0");
    need(s->num_q_heads <= 65536 && s->block_size <= 65536, "more than 65536 heads or tokens per block");
    need((uint64_t)s->num_slots * s->num_kv_heads <= 0xFFFFFFFEull / s->block_size, "a cache of 2^32 rows or more");
    need(s->reserved == 0 && b->reserved == 0, "reserved fields are not 0");
    need(b->max_kv <= 1u << 30 && b->max_q <= 1u << 30 && b->total_q <= 1u << 30, "a length of more than 2^30");
    need(!arrays || (uint64_t)b->table_stride * s->block_size >= b->max_kv, "table_stride * block_size is less than max_kv");
    need((uint64_t)b->n_seq * s->num_kv_heads <= kMostLists, "more than 2^18 sequences times KV heads");
    CacheView c{};
    if (b->n_seq) {
        if (arrays) {
            need_pointer(b->kv_len, 4, "kv_len");
            if (b->max_kv) need_pointer(b->block_table, 4, "block_table");
            if (queries) need_pointer(b->cu_q, 4, "cu_q");
        }
        if (queries) {
            need(b->max_q <= b->total_q, "max_q is more than total_q");
            need((uint64_t)b->total_q * s->num_q_heads <= kMostRows, "more than 2^29 new tokens times query heads");
        }
    } else {
        need(!queries || b->total_q == 0, "new tokens without a sequence");
    }
    c.cu_q = b->cu_q;
    c.kv_len = b->kv_len;
    c.table = b->block_table;
    c.n_seq = b->n_seq;
    c.total_q = b->total_q;
    c.max_q = b->max_q;
    c.max_kv = b->max_kv;
    c.table_stride = b->table_stride;
    c.num_slots = s->num_slots;
    c.heads = s->num_q_heads;
    c.kv_heads = s->num_kv_heads;
    c.group = s->num_q_heads / s->num_kv_heads;
    c.head_dim = s->head_dim;
    c.block = s->block_size;
    divide_by(c.block, &c.block_magic, &c.block_shift);
    divide_by(c.group, &c.group_magic, &c.group_shift);
    return c;
}

void need_rows(const void *p, uint64_t stride, uint64_t least, const char *what)
{
    need_pointer(p, 16, what);
    if (stride % 8) fail(KVP_ERR_INVALID, std::string(what) + ": its stride is no multiple of 8 elements");
    if (stride < least) fail(KVP_ERR_INVALID, std::string(what) + ": its stride is less than a token's heads");
    need(stride <= 1ull << 40, "a stride of more than 2^40 elements");
}

// Rows of a sequence up to which the waves split the keys, and the parts that such a call is cut into.
struct CutRule {
    uint32_t few_rows, parts;
};

struct Cut {
    uint32_t few;     // most rows of a sequence, or 0: tiles of rows
    uint32_t tiles, splits, split_keys;
    bool uneven;      // sequences of different lengths, which the kernels go by
    uint64_t bytes;   // of workspace
};

// How an attention call is cut.  A KV head's rows (new tokens x group) go to attention_few if no sequence has more
// than a 16-row product holds, to attention_some up to 64 (32) by the rule of calls that it is for, else to tiles of
// 256 (128 at a head_dim of more than 128).  Where the tiles do not
// fill the chip, the keys are split, as far as a part holds enough keys to be worth its output's way through memory.
Cut cut_of(const CacheView &c, uint32_t window, const CutRule &rule, bool tree = false)
{
    Cut p{};
    const uint64_t rows = (uint64_t)c.total_q * c.group;
    const uint32_t tile_rows = row_waves(c.head_dim) * 32;
    const bool few = (uint64_t)c.max_q * c.group <= rule.few_rows;
    p.few = few ? std::max(1u, c.max_q * c.group) : 0;
    if (!rows) return p.splits = 1, p.split_keys = kTileKeys, p;
    p.tiles = few            ? c.n_seq
              : c.n_seq == 1 ? (uint32_t)((rows + tile_rows - 1) / tile_rows)
                             : (uint32_t)(rows / tile_rows + c.n_seq);
    // new tokens whose keys a workgroup goes over: those of its rows, or with a mask among them all
    const uint64_t tile_tokens = few || tree ? c.max_q : std::min<uint64_t>(c.max_q, tile_rows / c.group + 2);
    uint64_t span = c.max_kv;
    if (window) span = std::min<uint64_t>(span, (uint64_t)window + tile_tokens + kTileKeys);
    // workgroups that have work: a sequence's last tile is half full, if it has another one
    const uint64_t units = (few              ? c.n_seq
                            : c.n_seq == 1 ? (rows + tile_rows - 1) / tile_rows
                                           : std::max<uint64_t>(c.n_seq, rows / tile_rows + c.n_seq / 2)) * c.kv_heads;
    uint64_t keys = span;                            // of a part
    if (few) {
        // about 1024 parts of 16-bit pages, which read the cache at its full rate (512 by the rule of other calls), and not
        // above 1024 keys where lengths may differ, so that none is left alone at the end.  32 sequences of up to 16K: 191 us
        // at 1024 keys, 210 at 512, 223 at 4096; one of 128K: 47 us at 1024, 49 at 512, 67 at 128.  256 keys stay whole: 8.5
        // us, where two parts and their join take 10.8.
        if (span > 256) {
            keys = std::max<uint64_t>(128, units * span / rule.parts);
            if (c.n_seq > 1) keys = std::min<uint64_t>(keys, 1024);
            keys = std::max(keys, units * span / kMostParts);
        }
    } else if (units < 512) {
        // The fewest parts that keep 19 of 20 CUs busy, of 512 keys or more: parts are written and read again, and a
        // workgroup takes some us to begin.  512 new tokens over 128K: 1064 us at 4 parts (256 workgroups), 1096 at 16,
        // 1293 at 64.
        auto fewest = [&](uint64_t units, uint64_t most) {
            uint64_t best = 1, filled = 0;           // of 1000
            for (uint64_t n = 1; n <= most && filled < 950; ++n) {
                const uint64_t f = units * n * 1000 / ((units * n + 255) / 256 * 256);
                if (f > filled) best = n, filled = f;
            }
            return best;
        };
        auto most_of = [&](uint64_t units) { return std::min(1024 / units, span / 512); };
        uint64_t best = fewest(units, most_of(units));
        if (c.n_seq > 1 && c.n_seq <= 64 && !window) {
            // Tiles that fill the chip stay whole: a join and more workgroups cost more than they give, whether lengths
            // differ or not.  32 x 8 new tokens over 1K (32 heads, 8 KV heads, 128) 43 us, 53 in up to two parts; over up to
            // 4K 117 and 125; 16 x 96 over 1K 48 and 64, over up to 16K 441 and 453.
            if (best > 1)                            // a batch of different lengths may want more, which its workgroups find
                best = std::min(2 * best, most_of(units));
            else if (c.total_q < 2 * (uint64_t)c.max_q && span >= 16384) {
                // A chunk among single tokens has more tiles than counted, of which a few would be left for a round of
                // their own.  31 single tokens and 512 new ones over 16K: 885 us whole, 761 in parts; where the single ones
                // are over 2K to 16K 504 and 520, and over 1K 75 and 84.
                const uint64_t chunk = ((uint64_t)c.max_q * c.group + tile_rows - 1) / tile_rows;
                const uint64_t all = (chunk + c.n_seq - 1) * c.kv_heads;
                if (all < 512) best = fewest(all, most_of(all));
            }
        }
        keys = (span + best - 1) / best;
    }
    // no more parts than without a window: the workspace is asked for without one
    if (window) keys = std::max(keys, (span + cut_of(c, 0, rule).splits - 1) / cut_of(c, 0, rule).splits);
    const uint64_t unit = few ? 128 : kTileKeys;
    keys = std::max(unit, (keys + unit - 1) / unit * unit);
    p.splits = (uint32_t)std::max<uint64_t>(1, (span + keys - 1) / keys);
    p.split_keys = (uint32_t)keys;
    p.uneven = p.splits > 1 && c.n_seq > 1 && c.n_seq <= 64 && (few ? c.max_q * c.group > kFewRows : !window);
    if (p.splits > 1) p.bytes = (uint64_t)p.splits * c.total_q * c.heads * (c.head_dim + 2) * 4;
    return p;
}

Cut attention_cut(const CacheView &c, uint32_t window) { return cut_of(c, window, {kFewRows, 1024}); }

// Half as many parts: they move half the bytes of 8-bit pages, or join the outputs of more rows.  One token over 128K in 8
// bits (32 heads, 8 KV heads, 128) 51.7 us, 56.3 at 1024 parts; trees of 8 and of 16 tokens over 128K 57 and 88, 65 and 107;
// the same over 16-bit pages 93 and 130, 100 and 149.
Cut pages_cut(const CacheView &c, uint32_t window, bool tree = false)
{
    return cut_of(c, window, {some_rows(c.head_dim), 512}, tree);
}

uint32_t row_exponents(uint32_t head_dim) { return (head_dim + 127) / 128 * 4; }

// A slot's bytes; a cache of less than 2^32 rows has less than 2^43.
uint64_t slot_bytes(const CacheView &c, uint32_t kind)
{
    const uint64_t rows = (uint64_t)c.kv_heads * c.block;
    if (kind == KVP_PAGES_16BIT) return rows * c.head_dim * 2;
    return (rows * (c.head_dim + row_exponents(c.head_dim)) + 15) / 16 * 16;
}

void need_kind(uint32_t kind) { need(kind == KVP_PAGES_16BIT || kind == KVP_PAGES_E4M3, "unknown kind of pages"); }

// Checks the pages; buffers says whether they are looked at.
PageView pages_of(const CacheView &c, const kvp_pages *p, uint32_t num_slots, bool buffers)
{
    need(p, "pages is null");
    need_kind(p->kind);
    need(p->reserved == 0, "reserved fields are not 0");
    if (buffers) {
        need_pointer(p->k, 16, "k pages");
        need_pointer(p->v, 16, "v pages");
    }
    PageView v{};
    v.k = static_cast<uint8_t *>(p->k);
    v.v = static_cast<uint8_t *>(p->v);
    v.slot_bytes = slot_bytes(c, p->kind);
    if (p->kind == KVP_PAGES_E4M3) {
        const uint64_t elements = (uint64_t)c.kv_heads * c.block * c.head_dim;
        need(elements <= 0x7FFFFFFFull, "a slot of 2^31 elements or more");
        v.exponents = (uint32_t)elements;
        v.row_exponents = row_exponents(c.head_dim);
    }
    v.num_slots = num_slots;
    return v;
}

// Lanes of 8 elements to a head, a power of two of them.
uint32_t lanes_log2(uint32_t head_dim)
{
    uint32_t n = 0;
    while ((8u << n) < head_dim) ++n;
    return n;
}

// Words of workspace to a list: four of counts, two per token (candidates, then moves), a bit per token, and for
// long lists the counts of 2^11 digits per part and of four waves' candidates.
uint64_t evict_words(const CacheView &c)
{
    const uint64_t n = c.max_kv;
    return 4 + 2 * n + 2 * ((n + 63) / 64) + (n > kEvictShort ? kEvictParts * (2048 + 4) : 0);
}
uint64_t evict_bytes(const CacheView &c) { return (uint64_t)c.n_seq * c.kv_heads * evict_words(c) * 4; }

void need_scale(float scale) { need(std::isfinite(scale) && scale > 0, "scale is not a positive number"); }

}  // namespace

namespace {

// What every attention call checks and says to its kernels, but for the tensors that the cut makes launches of.
void fill_attention(AttentionArgs &a, const void *q, uint64_t q_stride, const void *k, const void *v, float scale,
                    uint32_t window, const float *sinks, void *out, uint64_t out_stride, float *lse, const Cut &p,
                    void *workspace, uint64_t workspace_bytes, const char *too_small)
{
    const uint64_t row = (uint64_t)a.c.heads * a.c.head_dim;
    need_rows(q, q_stride, 0, "q");
    need_rows(out, out_stride, row, "out");
    need_pointer(k, 16, "k_cache");
    need_pointer(v, 16, "v_cache");
    need(aligned(sinks, 4), "sinks is not aligned to 4 bytes");
    need(aligned(lse, 4), "lse is not aligned to 4 bytes");
    if (p.bytes) {
        need_pointer(workspace, 16, "workspace");
        need(workspace_bytes >= p.bytes, too_small);
    }
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.q_stride = q_stride;
    a.out = static_cast<uint16_t *>(out);
    a.out_stride = out_stride;
    a.lse = lse;
    a.sinks = sinks;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window;
    a.few_rows = p.few;
    a.tiles = p.tiles;
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    a.uneven = p.uneven;
    const uint64_t parts = (uint64_t)p.splits * a.c.total_q * a.c.heads;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = a.part_o ? a.part_o + parts * a.c.head_dim : nullptr;
}

}  // namespace

void op_attention_workspace(const kvp_cache_shape *s, const kvp_batch *b, uint64_t *bytes)
{
    need(bytes, "bytes is null");
    *bytes = attention_cut(view_of(s, b, true, false), 0).bytes;
}

void op_attention(const kvp_cache_shape *s, const kvp_batch *b, const void *q, uint64_t q_stride, const void *k,
                  const void *v, float scale, uint32_t window, const float *sinks, void *out, uint64_t out_stride,
                  float *lse, void *workspace, uint64_t workspace_bytes, void *stream)
{
    AttentionArgs a{};
    a.c = view_of(s, b, true);
    need_scale(scale);
    if (a.c.total_q == 0) return;
    fill_attention(a, q, q_stride, k, v, scale, window, sinks, out, out_stride, lse, attention_cut(a.c, window), workspace,
                   workspace_bytes, "workspace is smaller than kv_attention_workspace says");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    check_hip(launch_attention(a, s->dtype, st), "attention launch");
    if (a.splits > 1) check_hip(launch_attention_join(a, s->dtype, st), "attention join launch");
}

void op_attention_pages_workspace(const kvp_cache_shape *s, const kvp_batch *b, uint64_t *bytes)
{
    need(bytes, "bytes is null");
    const CacheView c = view_of(s, b, true, false);
    *bytes = std::max(attention_cut(c, 0).bytes, pages_cut(c, 0).bytes);   // causal ones of 16 bits are kv_attention's
}

void op_attention_pages(const kvp_cache_shape *s, const kvp_batch *b, const kvp_pages *pages, const uint64_t *tree,
                        uint32_t tree_words, const void *q, uint64_t q_stride, float scale, uint32_t window,
                        const float *sinks, void *out, uint64_t out_stride, float *lse, void *workspace,
                        uint64_t workspace_bytes, void *stream)
{
    AttentionArgs a{};
    a.c = view_of(s, b, true);
    need_scale(scale);
    const PageView p = pages_of(a.c, pages, a.c.num_slots, a.c.total_q != 0);
    need(aligned(tree, 8), "tree is not aligned to 8 bytes");
    need(tree ? (uint64_t)tree_words * 64 >= a.c.max_q && tree_words <= 1u << 20 : tree_words == 0,
         "tree_words is not from ceil(max_q / 64) to 2^20, or not 0 without a tree");
    if (a.c.total_q == 0) return;
    const bool eight = pages->kind == KVP_PAGES_E4M3;
    // 16-bit pages under a causal mask are kv_attention's
    const Cut cut = eight || tree ? pages_cut(a.c, window, tree) : attention_cut(a.c, window);
    fill_attention(a, q, q_stride, p.k, p.v, scale, window, sinks, out, out_stride, lse, cut, workspace, workspace_bytes,
                   "workspace is smaller than kv_attention_pages_workspace says");
    a.exponents = p.exponents;
    a.row_exponents = p.row_exponents;
    a.slot_bytes = p.slot_bytes;
    a.tree = tree;
    a.tree_words = tree_words;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    check_hip(eight  ? launch_attention_e4m3(a, s->dtype, st)
              : tree ? launch_attention_tree(a, s->dtype, st)
                     : launch_attention(a, s->dtype, st),
              "attention launch");
    if (a.splits > 1) check_hip(launch_attention_join(a, s->dtype, st), "attention join launch");
}

void op_page_bytes(const kvp_cache_shape *s, uint32_t kind, uint64_t *bytes)
{
    need(bytes, "bytes is null");
    const kvp_batch none{};
    const CacheView c = view_of(s, &none, false, false);
    need_kind(kind);
    *bytes = slot_bytes(c, kind);
}

void op_norm_rope_append(const kvp_cache_shape *s, const kvp_batch *b, const kvp_pages *pages, const kvp_head_norm *norm,
                         const kvp_rope_axes *axes, const float *angles, uint32_t n_positions, uint32_t rot, uint32_t flags,
                         const int32_t *positions, const void *q, uint64_t q_stride, void *q_out, uint64_t q_out_stride,
                         const void *k, uint64_t k_stride, const void *v, uint64_t v_stride, int32_t *pos,
                         uint32_t pos_stride, void *stream)
{
    AppendArgs a{};
    a.c = view_of(s, b, true);
    a.pages = pages_of(a.c, pages, a.c.num_slots, a.c.total_q != 0);
    need(!(flags & ~KVP_ROPE_INTERLEAVED), "unknown flags");
    need(rot % 2 == 0 && rot <= a.c.head_dim, "rot_dim is odd or more than head_dim");
    need(!q == !q_out, "one of q and q_out is null");
    a.axes = 1;
    if (axes) {
        need(axes->num_axes >= 1 && axes->num_axes <= kMostAxes, "num_axes is not from 1 to 4");
        need(axes->reserved == 0, "reserved fields are not 0");
        a.axes = axes->num_axes;
        for (uint32_t j = 0; j < rot / 2; ++j) {
            need(axes->axis_of[j] < a.axes, "a pair's axis is not below num_axes");
            a.axis_of[j] = axes->axis_of[j];
        }
    }
    if (norm) {
        need(norm->reserved == 0, "reserved fields are not 0");
        need(std::isfinite(norm->eps) && norm->eps >= 0, "eps is negative or no number");
        need(aligned(norm->q_weight, 16) && aligned(norm->k_weight, 16), "q_weight or k_weight is not aligned to 16 bytes");
        a.norm = 1;
        a.eps = norm->eps;
        a.q_weight = static_cast<const uint16_t *>(norm->q_weight);
        a.k_weight = static_cast<const uint16_t *>(norm->k_weight);
    }
    if (a.c.total_q == 0) return;
    need(n_positions > 0, "an empty table of angles");
    if (rot) need_pointer(angles, 8, "angles");
    need_pointer(positions, 4, "positions");
    const uint64_t row = (uint64_t)a.c.heads * a.c.head_dim;
    if (q) {
        need_rows(q, q_stride, 0, "q");
        need_rows(q_out, q_out_stride, row, "q_out");
        need(q != q_out, "q_out is q");
    }
    need_rows(k, k_stride, 0, "k");
    need_rows(v, v_stride, 0, "v");
    if (pos) {
        need_pointer(pos, 4, "pos");
        need(pos_stride >= a.c.max_kv, "pos_stride is less than max_kv");
    }
    need(a.c.total_q < 1u << 24, "2^24 new tokens or more in one call");
    a.angles = angles;
    a.positions = positions;
    a.n_positions = n_positions;
    a.rot = rot;
    a.interleaved = flags & KVP_ROPE_INTERLEAVED ? 1 : 0;
    a.lanes_log2 = lanes_log2(a.c.head_dim);
    a.per_dim = 1.0f / (float)a.c.head_dim;
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.q_out = static_cast<uint16_t *>(q_out);
    a.q_stride = q_stride;
    a.q_out_stride = q_out_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pos = pos;
    a.pos_stride = pos_stride;
    check_hip(launch_append(a, s->dtype, static_cast<hipStream_t>(stream)), "append launch");
}

void op_convert_pages(const kvp_cache_shape *s, const kvp_batch *b, const kvp_pages *from, const kvp_pages *to,
                      const int32_t *to_table, uint32_t to_stride, uint32_t to_slots, const int32_t *first, void *stream)
{
    ConvertArgs a{};
    a.c = view_of(s, b, false);
    const bool any = a.c.n_seq && a.c.max_kv;
    a.from = pages_of(a.c, from, a.c.num_slots, any);
    a.to = pages_of(a.c, to, to_slots, any);
    need(from->kind != to->kind, "pages of the same kind");
    need(to_slots > 0, "to_slots is 0");
    need((uint64_t)to_slots * a.c.kv_heads <= 0xFFFFFFFEull / a.c.block, "a cache of 2^32 rows or more");
    need((uint64_t)to_stride * a.c.block >= a.c.max_kv, "to_stride * block_size is less than max_kv");
    need(aligned(first, 4), "first is not aligned to 4 bytes");
    need(((uint64_t)a.c.max_kv + kConvertTokens - 1) / kConvertTokens * a.c.n_seq * a.c.kv_heads < 1u << 24,
         "too many tokens for one call");
    if (!any) return;
    need_pointer(to_table, 4, "to_table");
    a.to_table = to_table;
    a.to_stride = to_stride;
    a.first = first;
    a.lanes_log2 = lanes_log2(a.c.head_dim);
    check_hip(launch_convert(a, s->dtype, static_cast<hipStream_t>(stream)), "page conversion launch");
}

void op_tree_commit(const kvp_cache_shape *s, const kvp_batch *b, const kvp_pages *pages, const int32_t *path,
                    const int32_t *accepted, int32_t *pos, uint32_t pos_stride, int32_t *len_out, void *stream)
{
    CommitArgs a{};
    a.c = view_of(s, b, true);
    a.pages = pages_of(a.c, pages, a.c.num_slots, a.c.n_seq != 0);
    if (a.c.n_seq == 0) return;
    need_pointer(accepted, 4, "accepted");
    need_pointer(len_out, 4, "len_out");
    if (a.c.total_q) need_pointer(path, 4, "path");
    if (pos) {
        need_pointer(pos, 4, "pos");
        need(pos_stride >= a.c.max_kv, "pos_stride is less than max_kv");
    }
    a.path = path;
    a.accepted = accepted;
    a.pos = pos;
    a.pos_stride = pos_stride;
    a.lanes_log2 = lanes_log2(a.c.head_dim);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool in_place = len_out == b->kv_len;   // the move still reads the old lengths
    a.len_out = in_place ? nullptr : len_out;
    check_hip(launch_commit(a, st), "commit launch");
    if (in_place) check_hip(launch_commit_lengths(a, len_out, st), "commit lengths launch");
}

void op_attention_mass(const kvp_cache_shape *s, const kvp_batch *b, const void *q, uint64_t q_stride, const void *k,
                       float scale, uint32_t window, const float *lse, uint32_t last, const float *score_in,
                       float *score_out, uint32_t score_stride, void *stream)
{
    MassArgs a{};
    a.c = view_of(s, b, true);
    need_scale(scale);
    if (a.c.n_seq == 0 || a.c.max_kv == 0) return;
    if (a.c.total_q) {
        need_rows(q, q_stride, 0, "q");
        need_pointer(lse, 4, "lse");
    }
    need_pointer(k, 16, "k_cache");
    need_pointer(score_out, 4, "score_out");
    need(aligned(score_in, 4), "score_in is not aligned to 4 bytes");
    need(score_stride >= a.c.max_kv, "score_stride is less than max_kv");
    need(((uint64_t)a.c.max_kv + 127) / 128 * a.c.n_seq * a.c.kv_heads < 1u << 24, "too many tokens for one call");
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.q_stride = q_stride;
    a.lse = lse;
    a.score_in = score_in;
    a.score_out = score_out;
    a.score_stride = score_stride;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window;
    a.last = last;
    check_hip(launch_mass(a, s->dtype, static_cast<hipStream_t>(stream)), "attention mass launch");
}

void op_rope_append(const kvp_cache_shape *s, const kvp_batch *b, const float *angles, uint32_t n_positions,
                    uint32_t rot, uint32_t flags, const int32_t *positions, const void *q, uint64_t q_stride,
                    void *q_out, uint64_t q_out_stride, const void *k, uint64_t k_stride, const void *v,
                    uint64_t v_stride, void *k_cache, void *v_cache, int32_t *pos, uint32_t pos_stride, void *stream)
{
    RopeArgs a{};
    a.c = view_of(s, b, true);
    need(!(flags & ~KVP_ROPE_INTERLEAVED), "unknown flags");
    need(rot % 2 == 0 && rot <= a.c.head_dim, "rot_dim is odd or more than head_dim");
    need(!q == !q_out, "one of q and q_out is null");
    if (a.c.total_q == 0) return;
    need(n_positions > 0, "an empty table of angles");
    if (rot) need_pointer(angles, 8, "angles");
    need_pointer(positions, 4, "positions");
    const uint64_t row = (uint64_t)a.c.heads * a.c.head_dim;
    if (q) {
        need_rows(q, q_stride, 0, "q");
        need_rows(q_out, q_out_stride, row, "q_out");
        need(q != q_out, "q_out is q");
    }
    need_rows(k, k_stride, 0, "k");
    need_rows(v, v_stride, 0, "v");
    need_pointer(k_cache, 16, "k_cache");
    need_pointer(v_cache, 16, "v_cache");
    if (pos) {
        need_pointer(pos, 4, "pos");
        need(pos_stride >= a.c.max_kv, "pos_stride is less than max_kv");
    }
    need(a.c.total_q < 1u << 24, "2^24 new tokens or more in one call");
    a.angles = angles;
    a.positions = positions;
    a.n_positions = n_positions;
    a.rot = rot;
    a.interleaved = flags & KVP_ROPE_INTERLEAVED ? 1 : 0;
    // 16-byte pieces, or pairs of them where both of a pair are whole
    a.per_head = a.c.head_dim / 8 - (!a.interleaved && rot % 16 == 0 ? rot / 16 : 0);
    divide_by(a.per_head, &a.per_magic, &a.per_shift);
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.q_out = static_cast<uint16_t *>(q_out);
    a.k_cache = static_cast<uint16_t *>(k_cache);
    a.v_cache = static_cast<uint16_t *>(v_cache);
    a.q_stride = q_stride;
    a.q_out_stride = q_out_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pos = pos;
    a.pos_stride = pos_stride;
    check_hip(launch_rope(a, s->dtype, static_cast<hipStream_t>(stream)), "rotary append launch");
}

void op_rope_table(float *angles, uint32_t n_positions, uint32_t rot, const kvp_rope_scaling *r, void *stream)
{
    need(r, "scaling is null");
    need(rot >= 2 && rot % 2 == 0 && rot <= kMostRotary, "rot_dim is no even number from 2 to 256");
    need(n_positions <= 1u << 30, "more than 2^30 positions");
    need(r->kind <= KVP_ROPE_BY_PARTS_INDEX && r->reserved == 0, "unknown kind of scaling, or reserved is not 0");
    need(std::isfinite(r->base) && r->base > 0, "base is not a positive number");
    need(std::isfinite(r->magnitude) && r->magnitude > 0, "magnitude is not a positive number");
    const bool parts = r->kind == KVP_ROPE_BY_PARTS || r->kind == KVP_ROPE_BY_PARTS_INDEX;
    if (r->kind != KVP_ROPE_PLAIN) need(std::isfinite(r->factor) && r->factor >= 1, "factor is less than 1");
    if (parts) {
        need(std::isfinite(r->original_length) && r->original_length > 0, "original_length is not a positive number");
        need(std::isfinite(r->alpha) && std::isfinite(r->beta) && r->alpha > 0 && r->beta > r->alpha,
             "alpha and beta are not 0 < alpha < beta");
        need(r->kind != KVP_ROPE_BY_PARTS_INDEX || r->base > 1, "base is not more than 1");
    }
    if (n_positions == 0) return;
    need_pointer(angles, 8, "angles");
    RopeTableArgs a{};
    a.angles = angles;
    a.n_positions = n_positions;
    a.half = rot / 2;
    a.magnitude = r->magnitude;
    const double tau = 6.283185307179586476925286766559;
    // the index whose frequency makes `turns` revolutions over the original length
    auto index_of = [&](double turns) { return rot * std::log(r->original_length / (turns * tau)) / (2 * std::log(r->base)); };
    for (uint32_t j = 0; j < a.half; ++j) {
        const double f = std::pow(r->base, -2.0 * j / rot) / tau;   // revolutions per position
        double keep = 1;                                            // share of the frequency that is not scaled
        if (r->kind == KVP_ROPE_LINEAR) keep = 0;
        if (r->kind == KVP_ROPE_BY_PARTS) keep = (r->original_length * f - r->alpha) / (r->beta - r->alpha);
        if (r->kind == KVP_ROPE_BY_PARTS_INDEX) {
            const double lo = index_of(r->beta), hi = index_of(r->alpha);
            keep = (hi - j) / (hi - lo);
        }
        keep = std::min(1.0, std::max(0.0, keep));
        a.turns[j] = r->kind == KVP_ROPE_PLAIN ? f : f * keep + f / r->factor * (1 - keep);
    }
    check_hip(launch_rope_table(a, static_cast<hipStream_t>(stream)), "rotary table launch");
}

void op_evict_workspace(const kvp_cache_shape *s, const kvp_batch *b, uint64_t *bytes)
{
    need(bytes, "bytes is null");
    *bytes = evict_bytes(view_of(s, b, false, false));
}

void op_evict(const kvp_cache_shape *s, const kvp_batch *b, const int32_t *keep, const int32_t *protect,
              const float *score_in, float *score_out, uint32_t score_stride, const int32_t *pos_in, int32_t *pos_out,
              uint32_t pos_stride, void *k_cache, void *v_cache, int32_t *len_out, void *workspace,
              uint64_t workspace_bytes, void *stream)
{
    EvictArgs a{};
    a.c = view_of(s, b, false);
    if (a.c.n_seq == 0) return;
    need_pointer(keep, 4, "keep");
    need_pointer(len_out, 4, "len_out");
    need(aligned(protect, 4), "protect is not aligned to 4 bytes");
    if (a.c.max_kv) {
        need_pointer(score_in, 4, "score_in");
        need_pointer(score_out, 4, "score_out");
        need(score_stride >= a.c.max_kv, "score_stride is less than max_kv");
        need_pointer(k_cache, 16, "k_cache");
        need_pointer(v_cache, 16, "v_cache");
        need(aligned(pos_in, 4) && aligned(pos_out, 4), "pos_in or pos_out is not aligned to 4 bytes");
        need((!pos_in && !pos_out) || pos_stride >= a.c.max_kv, "pos_stride is less than max_kv");
    }
    need_pointer(workspace, 16, "workspace");
    need(workspace_bytes >= evict_bytes(a.c), "workspace is smaller than kv_evict_workspace says");
    a.keep = keep;
    a.protect = protect;
    a.score_in = score_in;
    a.score_out = score_out;
    a.pos_in = pos_in;
    a.pos_out = pos_out;
    a.score_stride = score_stride;
    a.pos_stride = pos_stride;
    a.k_cache = static_cast<uint16_t *>(k_cache);
    a.v_cache = static_cast<uint16_t *>(v_cache);
    a.len_out = len_out;
    a.moves = static_cast<uint32_t *>(workspace);
    a.list_words = evict_words(a.c);
    check_hip(launch_evict(a, static_cast<hipStream_t>(stream)), "eviction launch");
}

}  // namespace kvp
