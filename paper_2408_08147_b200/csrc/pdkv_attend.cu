// Attention of a batch's newest tokens over a paged pool, and the join of its parts.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "pdkv_seqs.h"

namespace pdkv {

namespace {

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ int own_len(const AttnParams &p, int seq, int cap)
{
    if (!p.seq_len) return cap;
    const int n = p.seq_len[seq];
    return n < 0 ? 0 : (n < cap ? n : cap);
}

struct RowId {
    int seq, token, g;
};
// Row `row` of a segment: which query token of which sequence, and which of the G heads.
__device__ __forceinline__ RowId row_id(const AttnParams &p, const AttnSeg &seg, int row)
{
    const int R = p.G * p.q_tokens;
    RowId id;
    if (seg.seq >= 0) {
        id.seq = seg.seq;
    } else {
        id.seq = p.members[seg.member_begin + row / R];
        row %= R;
    }
    id.token = row / p.G;
    id.g = row % p.G;
    return id;
}

}  // namespace

// One work item per pass: a warp walks the tokens of one row at a time.
template <typename T>
__global__ void __launch_bounds__(128) attend_items_kernel(const AttnParams p)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int i = p.cta_items[blockIdx.x]; i < p.cta_items[blockIdx.x + 1]; ++i) {
        const AttnItem it = p.items[i];
        const AttnSeg seg = p.segs[it.seg];
        for (int r = warp; r < it.rows; r += 4) {
            const RowId id = row_id(p, seg, it.row0 + r);
            const int head = it.head * p.G + id.g;
            const T *q = static_cast<const T *>(p.q) + id.seq * p.q_stride[0] + id.token * p.q_stride[1] + head * p.q_stride[2];
            int len = seg.len, sees = len;
            if (seg.seq >= 0) {
                len = own_len(p, seg.seq, seg.len);
                sees = len - (p.q_tokens - 1 - id.token);
            }
            float qf[8], acc[8];
            for (int k = 0; k < 8; ++k) {
                qf[k] = lane + 32 * k < p.D ? to_float(q[lane + 32 * k]) : 0.f;
                acc[k] = 0.f;
            }
            float m = -INFINITY, l = 0.f;
            for (int t = it.tok0; t < min(it.tok1, len); ++t) {
                const int64_t blk = p.tbl[seg.tbl + t / p.pool.block_tokens];
                const char *row = p.pool.base + blk * p.pool.block_stride + (2 * (int64_t)p.layer) * p.pool.lc_stride +
                                  it.head * p.pool.head_stride + (t % p.pool.block_tokens) * p.pool.tok_stride;
                float z = -INFINITY;
                if (t < sees) {
                    const T *k_row = reinterpret_cast<const T *>(row), *v_row = reinterpret_cast<const T *>(row + p.pool.lc_stride);
                    float dot = 0.f;
                    for (int k = 0; k < 8; ++k)
                        if (lane + 32 * k < p.D) dot += qf[k] * to_float(k_row[lane + 32 * k]);
                    for (int o = 16; o; o /= 2) dot += __shfl_xor_sync(~0u, dot, o);
                    z = dot * p.scale_log2;
                    const float top = fmaxf(m, z), base = top == -INFINITY ? 0.f : top;
                    const float keep = exp2f(m - base), w = exp2f(z - base);
                    l = l * keep + w;
                    for (int k = 0; k < 8; ++k)
                        if (lane + 32 * k < p.D) acc[k] = acc[k] * keep + w * to_float(v_row[lane + 32 * k]);
                    m = top;
                }
                if (p.logits && seg.seq >= 0 && lane == 0) {
                    const AttnSeq s = p.seqs[seg.seq];
                    p.logits[s.logits + ((int64_t)it.head * p.G * p.q_tokens + it.row0 + r) * s.logit_stride + t] = z;
                }
            }
            if (it.direct) {
                T *out = static_cast<T *>(p.out) + id.seq * p.out_stride[0] + id.token * p.out_stride[1] + head * p.out_stride[2];
                for (int k = 0; k < 8; ++k)
                    if (lane + 32 * k < p.D) out[lane + 32 * k] = from_float<T>(l > 0.f || l != l ? acc[k] / l : 0.f);
                if (p.lse && lane == 0)
                    p.lse[((int64_t)id.seq * p.q_tokens + id.token) * p.G * p.H + head] = (m + log2f(l)) * kLn2;
            } else {
                for (int k = 0; k < 8; ++k)
                    if (lane + 32 * k < p.D) p.part_o[(it.part_row + r) * p.D + lane + 32 * k] = acc[k];
            }
            if ((!it.direct || p.logits) && lane == 0) {
                p.part_ml[2 * (it.part_row + r)] = m;
                p.part_ml[2 * (it.part_row + r) + 1] = l;
            }
        }
    }
}

namespace {

// The parts of row `row` of (sequence, head): np0 parts of own tokens, then those of the prefix.
struct Parts {
    int64_t first[2], step[2];
    int n[2];
};

__device__ __forceinline__ Parts parts_of(const AttnParams &p, const AttnSeq &s, int head, int row)
{
    Parts x;
    x.n[0] = x.n[1] = 0;
    x.first[0] = x.first[1] = x.step[0] = x.step[1] = 0;
    if (s.own_unit >= 0) {
        const AttnUnit u = p.units[s.own_unit + row / s.own_tile * p.H + head];
        x.first[0] = u.part_row + row % s.own_tile;
        x.step[0] = u.rows;
        x.n[0] = u.n_parts;
    }
    if (s.prefix_unit >= 0) {
        const int pr = s.prefix_row0 + row;
        const AttnUnit u = p.units[s.prefix_unit + pr / s.prefix_tile * p.H + head];
        x.first[1] = u.part_row + pr % s.prefix_tile;
        x.step[1] = u.rows;
        x.n[1] = u.n_parts;
    }
    return x;
}

__device__ __forceinline__ int64_t part_at(const Parts &x, int i)
{
    return i < x.n[0] ? x.first[0] + i * x.step[0] : x.first[1] + (i - x.n[0]) * x.step[1];
}

// Maximum and sum of a row over all of its parts; whole warp, every lane gets both.
__device__ __forceinline__ float2 joined_ml(const AttnParams &p, const Parts &x, int lane)
{
    const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml);
    float m = -INFINITY, l = 0.f;
    for (int i = lane; i < x.n[0] + x.n[1]; i += 32) {
        const float2 v = ml[part_at(x, i)];
        const float top = fmaxf(m, v.x), base = top == -INFINITY ? 0.f : top;
        l = l * exp2f(m - base) + v.y * exp2f(v.x - base);
        m = top;
    }
    for (int o = 16; o; o /= 2) {
        const float m2 = __shfl_xor_sync(~0u, m, o), l2 = __shfl_xor_sync(~0u, l, o);
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
        l = l * exp2f(m - base) + l2 * exp2f(m2 - base);
        m = top;
    }
    return make_float2(m, l);
}

constexpr int kScoreChunk = 512;   // tokens of one block of the score part
constexpr int kScoreRows = 64;     // rows whose lse is held at a time

}  // namespace

// Blocks (sequence, head, 0) join the parts of the rows: m = max m_p, l = sum l_p 2^(m_p - m),
// O = sum O_p 2^(m_p - m).  Blocks (sequence, head, 1 + c) turn the logits of token chunk c into
// weights 2^(z - lse) and add them to the scores; they take the lse from the parts themselves, so
// no block waits for another.
template <typename T>
__global__ void __launch_bounds__(128) attend_join_kernel(const AttnParams p, const int chunks)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int x = blockIdx.x % (1 + chunks), head = blockIdx.x / (1 + chunks) % p.H, seq = blockIdx.x / (1 + chunks) / p.H;
    const AttnSeq s = p.seqs[seq];
    const int R = p.G * p.q_tokens;
    if (x == 0) {
        if (s.direct) return;
        for (int row = warp; row < R; row += 4) {
            const Parts parts = parts_of(p, s, head, row);
            const float2 ml = joined_ml(p, parts, lane);
            const float base = ml.x == -INFINITY ? 0.f : ml.x;
            float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
            for (int i = 0; i < parts.n[0] + parts.n[1]; ++i) {
                const int64_t at = part_at(parts, i);
                const float m = p.part_ml[2 * at];
                if (m == -INFINITY) continue;   // nothing was written for this part
                const float w = exp2f(m - base);
                const float4 *o = reinterpret_cast<const float4 *>(p.part_o + at * p.D);
                for (int k = 0; k < 2; ++k)
                    if (4 * (lane + 32 * k) < p.D) {
                        const float4 v = o[lane + 32 * k];
                        acc[k].x += w * v.x;
                        acc[k].y += w * v.y;
                        acc[k].z += w * v.z;
                        acc[k].w += w * v.w;
                    }
            }
            const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
            const int token = row / p.G, h = head * p.G + row % p.G;
            T *out = static_cast<T *>(p.out) + seq * p.out_stride[0] + token * p.out_stride[1] + h * p.out_stride[2];
            for (int k = 0; k < 2; ++k)
                if (4 * (lane + 32 * k) < p.D) {
                    T v[4] = {from_float<T>(acc[k].x * inv), from_float<T>(acc[k].y * inv), from_float<T>(acc[k].z * inv),
                              from_float<T>(acc[k].w * inv)};
                    *reinterpret_cast<uint2 *>(out + 4 * (lane + 32 * k)) = *reinterpret_cast<uint2 *>(v);
                }
            if (p.lse && lane == 0) p.lse[((int64_t)seq * p.q_tokens + token) * p.G * p.H + h] = (ml.x + log2f(ml.y)) * kLn2;
        }
        return;
    }
    __shared__ float lse[kScoreRows];
    const int len = own_len(p, seq, s.len), t0 = (x - 1) * kScoreChunk + 4 * threadIdx.x;
    // past the sequence's end there is no weight: nothing to do in place, else the row is carried over
    const int width = p.scores_in == p.scores_out ? len : p.max_len;
    if ((x - 1) * kScoreChunk >= width) return;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < R; r0 += kScoreRows) {
        const int n = min(kScoreRows, R - r0);
        __syncthreads();
        for (int row = warp; row < n; row += 4) {
            const float2 ml = joined_ml(p, parts_of(p, s, head, r0 + row), lane);
            // an empty row gives no weight to anything: 2^(z - inf) = 0
            if (lane == 0) lse[row] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
        }
        __syncthreads();
        const float *z = p.logits + s.logits + ((int64_t)head * R + r0) * s.logit_stride + t0;
        if (t0 < len)
            for (int row = 0; row < n; ++row) {
                const float4 v = *reinterpret_cast<const float4 *>(z + (int64_t)row * s.logit_stride);
                sum[0] += exp2f(v.x - lse[row]);
                if (t0 + 1 < len) sum[1] += exp2f(v.y - lse[row]);
                if (t0 + 2 < len) sum[2] += exp2f(v.z - lse[row]);
                if (t0 + 3 < len) sum[3] += exp2f(v.w - lse[row]);
            }
    }
    for (int k = 0; k < 4; ++k)
        if (t0 + k < width) {
            const float in = p.scores_in ? p.scores_in[seq * p.scores_in_stride[0] + head * p.scores_in_stride[1] + t0 + k] : 0.f;
            p.scores_out[seq * p.scores_out_stride[0] + head * p.scores_out_stride[1] + t0 + k] = in + sum[k];
        }
}

cudaError_t launch_attend(const AttnParams &p, int dtype, cudaStream_t stream)
{
    if (dtype == PDKV_DTYPE_BF16)
        attend_items_kernel<__nv_bfloat16><<<p.n_ctas, 128, 0, stream>>>(p);
    else
        attend_items_kernel<__half><<<p.n_ctas, 128, 0, stream>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_attend_join(const AttnParams &p, int dtype, cudaStream_t stream)
{
    const int chunks = p.logits ? (p.max_len + kScoreChunk - 1) / kScoreChunk : 0;
    const int64_t blocks = (int64_t)p.n_seq * p.H * (1 + chunks);
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    if (dtype == PDKV_DTYPE_BF16)
        attend_join_kernel<__nv_bfloat16><<<(unsigned)blocks, 128, 0, stream>>>(p, chunks);
    else
        attend_join_kernel<__half><<<(unsigned)blocks, 128, 0, stream>>>(p, chunks);
    return cudaGetLastError();
}

}  // namespace pdkv
