// Internal declarations of the operators that work on a filled pool (attention, eviction).
#pragma once

#include <vector>

#include "pdkv_internal.h"

namespace pdkv {

// Where a pool keeps the row (layer, K/V, head) of a token: bytes.
struct PoolView {
    char *base;
    int64_t block_stride, lc_stride, head_stride, tok_stride;
    int32_t block_tokens;
};
PoolView pool_view(const pdkv_pool &p);

// A list of cached tokens: the own tokens of a sequence, or a prefix.
struct AttnSeg {
    int64_t tbl;            // first entry in the device block table
    int32_t len;
    int32_t seq;            // own tokens: the sequence; prefix: -1
    int32_t member_begin;   // prefix: its sequences are members[member_begin ..)
    int32_t before;         // own tokens: tokens of the prefix in front of them
};

// (segment, row tile, KV head): the rows whose parts are joined.
struct AttnUnit {
    int64_t part_row;   // first partial row; part p starts at part_row + p * rows
    int32_t n_parts;
    int32_t rows;
};

// What one CTA does in one go: rows [row0, row0 + rows) of one head against tokens [tok0, tok1) of a
// segment.  Carries what it needs of the segment, so that a kernel starts on it after one load.
struct alignas(16) AttnItem {
    int64_t part_row;
    int64_t tbl;
    int32_t seq, member_begin, len;   // of the segment
    int32_t head;
    int32_t row0, rows;
    int32_t tok0, tok1;
    int32_t direct;     // 1: the only part of its rows, the item writes the result itself
    int32_t next;       // the CTA's next item, -1: none
    int32_t pad[2];
};

// What the joining kernel has to know about a sequence.
struct AttnSeq {
    int64_t logits;          // first logit of the sequence in the scratch: [head][row][logit_stride]
    int32_t own_unit;        // unit of (row tile 0, head 0), -1: no own tokens
    int32_t own_tile;        // rows per row tile
    int32_t prefix_unit;     // as own_unit, of the prefix; -1: none
    int32_t prefix_tile;
    int32_t prefix_row0;     // first row of this sequence among the rows of its prefix
    int32_t len;             // own tokens at most
    int32_t logit_stride;
    int32_t direct;          // 1: nothing to join
};

// The status word of a handle on which an append or accept was given a length above the handle's.
constexpr unsigned long long kStatusLength = 2;

// tanh(x) / x for |x| <= 0.65 as a polynomial in (2 x log2 e)^2, that of degree 4 with the least largest relative error (a weighted fit, reweighted
// until the extremes are level): off by 2^-22.6 at most.
constexpr double kCapTerms[5] = {0.99999985, -0.04003555, 1.918510e-3, -8.927525e-5, 3.044123e-6};
constexpr float kCapNear = 1.8755036f;   // 2 * 0.65 log2 e

struct AttnParams {
    PoolView pool;
    const int32_t *tbl;
    const AttnSeg *segs;
    const AttnUnit *units;
    const AttnSeq *seqs;
    const int32_t *members;
    const AttnItem *items;           // CTA c starts with item c
    int32_t n_ctas;
    const AttnItem *tile_items;      // the same for the tile kernel
    int32_t n_tile_ctas;
    int32_t use_map;                 // the warp kernel loads through the tensor map
    int32_t map_box, tile_box;       // tokens of a box of the two maps
    int32_t map_layer_major;         // order of the coordinates of the pool's tensor map
    unsigned long long *status;      // [0] != 0: a bounded wait gave up, or kStatusLength
    int32_t n_seq, H, G, D, q_tokens;
    const void *q;
    void *out;
    int64_t q_stride[3], out_stride[3];
    float *lse;
    float scale_log2;           // scale * log2(e): logits are kept in the base-2 domain
    const int32_t *seq_len;     // device, or null
    float *part_o;              // [part row][D], unnormalised, relative to the part's maximum
    float *part_ml;             // [part row][2]: maximum (base 2), sum
    int32_t with_scores;
    int64_t own_tiles;          // tiles of 128 own tokens, over all sequences and heads
    int32_t sm_count;
    float *logits;              // null: no scores wanted, or the weighing kernel finds them
    const float *scores_in;
    float *scores_out;
    int64_t scores_in_stride[2], scores_out_stride[2];
    int32_t max_len;
    int32_t layer;
    int32_t block_shift;        // log2 of block_tokens, -1: not a power of two
    // another form than plain causal (pdkv_attend_form): a variant of each kernel
    int32_t formed;             // 1: masks alone, 2: caps too, 3: biases too (and caps, where there are)
    // logits (base 2) of products z of the scale's sign: cap_out tanh(z cap_in / (2 log2 e)), which up to |z cap_in| = kCapNear is
    // z (cap_terms[0] + cap_terms[1] (z cap_unit)^2 + ...); cap_out 0: z scale_log2
    float cap_in, cap_out, cap_unit, cap_terms[5];
    const float *slopes;
    const uint32_t *mask;
    int64_t mask_stride[2];
    const int32_t *n_new, *offset;
    int64_t offset_stride;
};

int attend_ctas_per_sm(int head_dim);
bool attend_map_supported(const pdkv_pool_desc &d);
int attend_map_box(const pdkv_pool_desc &d);
cudaError_t launch_attend(const AttnParams &p, const void *map, int dtype, cudaStream_t stream);
// (its variants for other forms than plain causal)
cudaError_t launch_attend_masked(const AttnParams &p, const void *map, int dtype, cudaStream_t stream);
cudaError_t launch_attend_capped(const AttnParams &p, const void *map, int dtype, cudaStream_t stream);
cudaError_t launch_attend_sloped(const AttnParams &p, const void *map, int dtype, cudaStream_t stream);
// The tile kernel (tcgen05): segments with many rows.  `map` is a CUtensorMap of the pool.
constexpr int kMapBytes = 128;
bool attend_tile_supported(const pdkv_pool_desc &d);
int attend_tile_box(const pdkv_pool_desc &d);
bool make_attend_map(const pdkv_pool &pool, int box_tokens, void *out);
cudaError_t launch_attend_tile(const AttnParams &p, const void *map, int dtype, cudaStream_t stream);
cudaError_t launch_attend_weigh(const AttnParams &p, const void *map, int dtype, cudaStream_t stream);
cudaError_t launch_attend_join(const AttnParams &p, int dtype, bool join, int most_parts, cudaStream_t stream);

struct EvictParams {
    PoolView src, dst;
    const int32_t *src_tbl, *dst_tbl;
    const AttnSeg *src_segs, *dst_segs;   // own tokens of sequence r are segment r
    int32_t n_seq, H, row_bytes;
    int32_t layer_begin, n_layers;
    int32_t in_place;
    int32_t budget, sink, recent;
    const int32_t *seq_len;
    const float *scores;
    int64_t scores_stride[3];
    int32_t *kept;
    float *kept_scores;
    int64_t kept_scores_stride[3];
    int32_t kept_scores_len;
    int32_t *new_len;
    int32_t max_len;       // longest sequence of the handle
    int32_t vec_bytes;     // alignment every row of both pools has
    int32_t src_shift, dst_shift;   // log2 of block_tokens, -1: not a power of two
};
cudaError_t launch_evict(const EvictParams &p, int sm_count, cudaStream_t stream);

}  // namespace pdkv

struct pdkv_seqs {
    pdkv_pool pool{};
    int device = 0;
    int sm_count = 148;
    int32_t n_seq = 0, n_prefix = 0;
    std::vector<int32_t> len;
    int32_t max_len = 0;
    bool unique_blocks = true;   // no block belongs to two sequences or to a prefix as well
    int32_t Hq = 0, G = 0, q_tokens = 0, dtype = 0;
    // host copies of the work lists (inspection), one list
    std::vector<pdkv::AttnSeg> segs;
    std::vector<pdkv::AttnUnit> units;
    std::vector<pdkv::AttnSeq> seqs;
    std::vector<pdkv::AttnItem> items[2];      // warp kernel, tile kernel
    std::vector<int32_t> item_cta[2];
    int32_t n_ctas[2] = {0, 0};
    alignas(64) char map[2][pdkv::kMapBytes] = {};   // tensor maps of the pool, for the two kernels
    bool use_map = false;        // the warp kernel loads through its map
    bool own_tiles = false;      // the tile kernel has the own tokens (all sequences have the same number of rows)
    std::vector<pdkv_attend_item> listing;
    int64_t part_rows = 0, logit_floats = 0;
    bool join = false;           // some rows have several parts, or none
    int32_t most_parts = 0;      // of a row behind one segment
    // device arrays
    void *dev_mem = nullptr;
    size_t dev_bytes = 0;
    bool owns_dev_mem = true;
    unsigned long long *d_status = nullptr;
    const int32_t *d_tbl = nullptr, *d_members = nullptr;
    const pdkv::AttnSeg *d_segs = nullptr;
    const pdkv::AttnUnit *d_units = nullptr;
    const pdkv::AttnSeq *d_seqs = nullptr;
    const pdkv::AttnItem *d_items[2] = {nullptr, nullptr};
};
