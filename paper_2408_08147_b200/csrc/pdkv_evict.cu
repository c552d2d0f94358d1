// Eviction: which tokens of a (layer, sequence, KV head) stay, and the move of their rows.
#include <cmath>

#include "pdkv_seqs.h"

namespace pdkv {

namespace {

__device__ __forceinline__ int own_len(const EvictParams &p, int seq)
{
    const int cap = p.src_segs[seq].len;
    if (!p.seq_len) return cap;
    const int n = p.seq_len[seq];
    return n < 0 ? 0 : (n < cap ? n : cap);
}

// Order of the scores as unsigned numbers: NaN below everything, -0 equal to +0.
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

}  // namespace

// One block per (layer, sequence, head): the key of the last token to keep is found bit by bit.
__global__ void __launch_bounds__(256) evict_select_kernel(const EvictParams p)
{
    __shared__ int counts[8];
    __shared__ int warp_keep[8], warp_tie[8];
    const int head = blockIdx.x % p.H, seq = blockIdx.x / p.H % p.n_seq, layer = blockIdx.x / p.H / p.n_seq;
    const int len = own_len(p, seq), lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int32_t *kept = p.kept + (int64_t)blockIdx.x * p.budget;
    for (int j = min(len, p.budget) + threadIdx.x; j < p.budget; j += 256) kept[j] = -1;
    if (len <= p.budget) {
        for (int j = threadIdx.x; j < len; j += 256) kept[j] = j;
        return;
    }
    const float *row = p.scores + layer * p.scores_stride[0] + seq * p.scores_stride[1] + head * p.scores_stride[2];
    const int lo = p.sink, hi = len - p.recent, want = p.budget - p.sink - p.recent;
    auto count = [&](uint32_t at_least) {
        int n = 0;
        for (int t = lo + threadIdx.x; t < hi; t += 256) n += order_key(row[t]) >= at_least;
        for (int o = 16; o; o /= 2) n += __shfl_xor_sync(~0u, n, o);
        __syncthreads();
        if (lane == 0) counts[warp] = n;
        __syncthreads();
        n = 0;
        for (int w = 0; w < 8; ++w) n += counts[w];
        return n;
    };
    uint32_t key = 0;   // largest key that at least `want` tokens reach
    if (want > 0)
        for (int b = 31; b >= 0; --b)
            if (count(key | 1u << b) >= want) key |= 1u << b;
    const int above = want > 0 && key != 0xffffffffu ? count(key + 1) : 0;
    const int ties = want - above;   // of the tokens at the key itself, the first ones
    int done = p.sink, tied = 0;
    for (int j = threadIdx.x; j < p.sink; j += 256) kept[j] = j;
    for (int t0 = lo; t0 < hi; t0 += 256) {
        const int t = t0 + threadIdx.x;
        const uint32_t k = t < hi ? order_key(row[t]) : 0u;
        const bool over = want > 0 && t < hi && k > key, tie = want > 0 && t < hi && k == key;
        const unsigned tie_mask = __ballot_sync(~0u, tie);
        __syncthreads();
        if (lane == 0) warp_tie[warp] = __popc(tie_mask);
        __syncthreads();
        int tie_rank = tied + __popc(tie_mask & ((1u << lane) - 1));
        for (int w = 0; w < 8; ++w) {
            if (w < warp) tie_rank += warp_tie[w];
            tied += warp_tie[w];
        }
        const bool keep = over || (tie && tie_rank < ties);
        const unsigned mask = __ballot_sync(~0u, keep);
        if (lane == 0) warp_keep[warp] = __popc(mask);
        __syncthreads();
        int at = done + __popc(mask & ((1u << lane) - 1));
        for (int w = 0; w < 8; ++w) {
            if (w < warp) at += warp_keep[w];
            done += warp_keep[w];
        }
        if (keep) kept[at] = t;
    }
    for (int j = threadIdx.x; j < p.recent; j += 256) kept[p.budget - p.recent + j] = hi + j;
}

namespace {

__device__ __forceinline__ char *row_at(const PoolView &v, const int32_t *tbl, const AttnSeg &seg, int lc, int head, int t)
{
    const int64_t blk = tbl[seg.tbl + t / v.block_tokens];
    return v.base + blk * v.block_stride + lc * v.lc_stride + head * v.head_stride + (int64_t)(t % v.block_tokens) * v.tok_stride;
}

}  // namespace

// One block per (layer, sequence, head, K/V) walks the kept tokens in order.  Token kept[j] >= j goes
// to slot j, so slots written for chunk j hold sources of chunks <= j only: in place it is enough
// that a chunk is read whole before it is written.
template <typename V>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictParams p)
{
    const int c = blockIdx.x & 1, stream = blockIdx.x >> 1;
    const int head = stream % p.H, seq = stream / p.H % p.n_seq, layer = stream / p.H / p.n_seq;
    const int32_t *kept = p.kept + (int64_t)stream * p.budget;
    const AttnSeg from = p.src_segs[seq], to = p.dst_segs[seq];
    const int lc = 2 * (p.layer_begin + layer) + c, vecs = p.row_bytes / (int)sizeof(V);
    const int top = min(min(p.budget, from.len), to.len);
    float *scores_to = c == 0 && p.kept_scores
                           ? p.kept_scores + layer * p.kept_scores_stride[0] + seq * p.kept_scores_stride[1] + head * p.kept_scores_stride[2]
                           : nullptr;
    const float *scores = p.scores + layer * p.scores_stride[0] + seq * p.scores_stride[1] + head * p.scores_stride[2];
    int n_kept = 0;
    for (int j0 = 0; j0 < top; j0 += 256) {   // scores and the count
        const int j = j0 + threadIdx.x;
        const int t = j < top ? kept[j] : -1;
        float s = 0.f;
        if (t >= 0 && scores_to) s = scores[t];
        n_kept += __syncthreads_count(t >= 0);
        if (t >= 0 && scores_to) scores_to[j] = s;
    }
    if (scores_to)
        for (int j = n_kept + threadIdx.x; j < p.kept_scores_len; j += 256) scores_to[j] = 0.f;
    if (p.new_len && c == 0 && layer == 0 && head == 0 && threadIdx.x == 0) p.new_len[seq] = n_kept;
    const int64_t work = (int64_t)n_kept * vecs;
    for (int64_t i0 = 0; i0 < work; i0 += 256) {
        const int64_t i = i0 + threadIdx.x;
        const int j = (int)(i / vecs), at = (int)(i % vecs);
        V v{};
        if (i < work) v = reinterpret_cast<const V *>(row_at(p.src, p.src_tbl, from, lc, head, kept[j]))[at];
        __syncthreads();
        if (i < work) reinterpret_cast<V *>(row_at(p.dst, p.dst_tbl, to, lc, head, j))[at] = v;
    }
}

cudaError_t launch_evict(const EvictParams &p, int sm_count, cudaStream_t stream)
{
    (void)sm_count;
    const int64_t rows = (int64_t)p.n_layers * p.n_seq * p.H;
    if (2 * rows > INT32_MAX) return cudaErrorInvalidConfiguration;
    evict_select_kernel<<<(unsigned)rows, 256, 0, stream>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)(2 * rows);
    switch (p.vec_bytes) {
    case 16: evict_move_kernel<uint4><<<grid, 256, 0, stream>>>(p); break;
    case 8: evict_move_kernel<uint2><<<grid, 256, 0, stream>>>(p); break;
    case 4: evict_move_kernel<uint32_t><<<grid, 256, 0, stream>>>(p); break;
    case 2: evict_move_kernel<uint16_t><<<grid, 256, 0, stream>>>(p); break;
    default: evict_move_kernel<uint8_t><<<grid, 256, 0, stream>>>(p); break;
    }
    return cudaGetLastError();
}

}  // namespace pdkv
