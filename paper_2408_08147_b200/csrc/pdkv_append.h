// Internal declarations of the calls that put tokens into a filled pool and settle drafted ones.
#pragma once

#include "pdkv_seqs.h"

namespace pdkv {

struct AppendParams {
    PoolView pool;
    const int32_t *tbl;
    const AttnSeg *segs;          // own tokens of sequence r are segment r
    int32_t layer, n_seq;
    int32_t Hq, H, D;             // Hq 0: no queries
    int32_t rows, per;            // rows of q, k, v; rows of a sequence where row_begin is null
    const int32_t *row_begin, *n_new, *seq_len;
    const void *q, *k, *v;
    void *q_out;
    int64_t q_stride[3], k_stride[3], v_stride[3], q_out_stride[3];
    const float *q_norm, *k_norm;
    float eps;
    const int32_t *position;
    int64_t position_stride;      // between axes
    int32_t rotated, adjacent, axes;
    const uint64_t *turns;
    const uint8_t *axis;
    float rotary_scale;
    int32_t block_shift;          // log2 of block_tokens, -1: not a power of two
    unsigned long long *status;
    // set by the launcher: a row is `parts` pieces of work of `steps` steps each; steps of its queries, of its keys
    int32_t parts, steps, q_steps, k_steps;
    float inv_D;
};
cudaError_t launch_append(AppendParams p, int dtype, int sm_count, cudaStream_t stream);

struct AcceptParams {
    PoolView pool;
    const int32_t *tbl;
    const AttnSeg *segs;
    int32_t n_seq, H, row_bytes;
    int32_t lc_begin, n_lc;       // (layer, K/V) strips
    const int32_t *path;
    int64_t path_stride;
    int32_t path_len, new_tokens;
    const int32_t *n_new, *seq_len;
    int32_t *new_len;
    int32_t vec_bytes;            // alignment every row of the pool has, 16 at most
    int32_t block_shift;
    unsigned long long *status;
};
cudaError_t launch_accept(const AcceptParams &p, cudaStream_t stream);

}  // namespace pdkv
