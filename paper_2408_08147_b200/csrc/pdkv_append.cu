// New tokens into a paged pool, their queries and keys normalised and rotated on the way; and the tokens of an accepted path
// to the place behind what they follow.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pdkv_append.h"

namespace pdkv {

namespace {

constexpr int kAppendThreads = 64;   // (128: 57.4 us instead of 56.8 for 13262 rows of 48 heads, 3.1 instead of 2.8 for 64)
// Steps of a warp in its ring, one of them at work.  Measured on 13262 rows of 48 heads of 128 dims: 3 59.3 us, 4 57.2, 6 57.8 (with 128 threads a block).
constexpr int kRing = 4;

__device__ __forceinline__ int own_tokens(const int32_t *seq_len, int seq, int most)
{
    if (!seq_len) return most;
    const int n = seq_len[seq];
    return n < 0 ? 0 : (n < most ? n : most);
}

// A length above the handle's is taken as the handle's, and the tokens of the call take the places of cached ones: reported.
__device__ __forceinline__ void report_length(const int32_t *seq_len, int seq, int most, unsigned long long *status)
{
    if (seq_len && seq_len[seq] > most) atomicCAS(status, 0ull, kStatusLength);
}

// Bytes from the pool's base to (layer 0, K, head 0) of token `slot` of a list.
__device__ __forceinline__ int64_t slot_offset(const PoolView &pool, const int32_t *tbl, int64_t list, int slot, int block_shift)
{
    const int b = block_shift >= 0 ? slot >> block_shift : slot / pool.block_tokens;
    return tbl[list + b] * pool.block_stride + (int64_t)(slot - b * pool.block_tokens) * pool.tok_stride;
}

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t x);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t x) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x)); }
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2 *>(&x)); }
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Two 32-bit numbers at a time.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t &>(d)) : "l"(reinterpret_cast<uint64_t &>(a)),
        "l"(reinterpret_cast<uint64_t &>(b)), "l"(reinterpret_cast<uint64_t &>(c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t &>(d)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)));
    return d;
}

// Eight 16-bit numbers of which the first n are there, as four words.  PIECES: their address is a multiple of 2 only.
template <bool PIECES> __device__ __forceinline__ uint4 load8(const uint16_t *from, int n)
{
    if constexpr (!PIECES) {
        return n > 0 ? *reinterpret_cast<const uint4 *>(from) : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? from[i] : 0;
        return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
    }
}
template <bool PIECES> __device__ __forceinline__ void store8(uint16_t *to, int n, const uint4 &v)
{
    if constexpr (!PIECES) {
        if (n > 0) *reinterpret_cast<uint4 *>(to) = v;
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) to[i] = (uint16_t)(w[i / 2] >> 16 * (i % 2));
    }
}

// The sequence that row `row` belongs to: the last one that begins at or before it, by 32 probes a round.  -1: none.
__device__ __forceinline__ int sequence_of(const int32_t *row_begin, int n_seq, int row)
{
    const int lane = threadIdx.x % 32;
    int lo = 0, hi = n_seq;
    while (true) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t before = __ballot_sync(~0u, at < hi && row_begin[at] <= row);
        if (before == 0) return -1;
        lo += (31 - __clz(before)) * step;
        if (step == 1) return lo;
        hi = min(lo + step, hi);
    }
}

}  // namespace

// A warp has one row (token) and, a step at a time, 32 / W heads of its queries, then of its keys, then of its values.  W lanes have a
// head, each two runs of eight dims, chosen so that both members of a rotated pair lie in one lane, which then has eight pairs:
//     y = x w / sqrt(mean x^2 + eps)      (a, b) -> (a cos - b sin, b cos + a sin), the angle position * frequency
// The sines serve all heads of the row, each found by one lane.  The angle is kept in turns as a 64-bit fraction: position * frequency
// wraps at whole turns by itself, and its upper 32 bits are right to 2^-32 of a turn at any position (position * frequency in 32-bit
// floating point is off by 0.004 at 100000).  Everything between load and store is 32 bits, two numbers at a time, rounded once; the
// weights are multiplied into the cosines and sines, so a result is two products and one by 1 / sqrt.
//
// Bound by the issue of instructions and memory in about equal parts: 13262 rows of 48 heads of 128 dims, normalised, into blocks of 16 tokens
// 55.5 us (5.9 TB/s; 207 instructions a step, four warps a scheduler busy for 55% of the time).  With the values' way through
// registers instead of shared memory 68 us (they crowd the tables out), with weights and sines multiplied one after the other 78.
// 64 rows: 2.8 us in a recorded graph, the latency of the lookups.
//
// Where all dims turn in split pairs, the lanes of a head load 16 bytes side by side.  Where pairs are adjacent, or dims do not turn, a lane's two
// runs are neighbours and the lanes load every other 16 bytes: the same prompts 86 us with adjacent pairs, 69 with 64 of 128 dims turning, 81 with none.
// Between its widths lanes idle: 96 dims 56 us, 80 dims 55 (for 0.75 and 0.63 of the bytes).
//
// ODD: half of the rotated dims is no multiple of eight.  Pairs (i, i + half) then lie in runs that are not aligned: a lane takes up
// to eight pairs, or up to sixteen of the dims behind them, in 16-bit pieces; a warp has one head a step, and nothing is loaded ahead.
// Slow: the same prompts with 24 of 96 dims turning 300 us, with 20 of 80 298.
template <typename T, int W, bool ODD, bool ADJACENT>
__global__ void __launch_bounds__(kAppendThreads, 8) append_kernel(const __grid_constant__ AppendParams p)
{
    constexpr int kHeads = 32 / W;   // of a step
    __shared__ __align__(16) float sines[kAppendThreads / 32][2][8 * W];
    __shared__ uint4 ring[kAppendThreads / 32][ODD ? 1 : kRing][2][32];
    const int lane = threadIdx.x % 32, sub = lane / W, i = lane % W;
    const int64_t item = (int64_t)blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32;
    const int row = (int)(item / p.parts), part = (int)(item - (int64_t)row * p.parts);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    if (row >= p.rows) return;   // (whole warps)

    // which dims are this lane's: na from a, nb from b
    const int half = p.rotated / 2;
    int a, b, na, nb;
    if (ADJACENT) {
        a = 16 * i;
        b = a + 8;
        na = p.D - a;
        nb = p.D - b;
    } else {
        const int turning = (half + 7) / 8;   // lanes with pairs
        if (i < turning) {
            a = 8 * i;
            b = half + a;
            na = nb = half - a;
        } else {
            a = p.rotated + 16 * (i - turning);
            b = a + 8;
            na = p.D - a;
            nb = p.D - b;
        }
    }
    na = max(0, min(8, na));
    nb = max(0, min(8, nb));
    a = na > 0 ? a : 0;
    b = nb > 0 ? b : 0;

    const int first = part * p.steps, last = min(first + p.steps, p.q_steps + 2 * p.k_steps);   // the warp's steps
    const int outer = p.row_begin ? 0 : row / p.per, lead = row - outer * p.per;   // where the row lies in q, k and v
    uint16_t *q_out = static_cast<uint16_t *>(p.q_out) + outer * p.q_out_stride[0] + lead * p.q_out_stride[1];
    // Walks the values of the warp's steps: queries (kind 0), then keys (1), then values (2).
    struct Walk {
        const uint16_t *src;
        int64_t stride;      // elements between steps
        int h, heads, left;  // the lane's head, heads of the kind, steps of the kind that are left
        int kind;
    };
    const auto enter = [&](Walk &w, int kind, int skip) {   // `skip` steps of the kind are not the warp's
        const int64_t *stride = kind == 0 ? p.q_stride : kind == 1 ? p.k_stride : p.v_stride;
        w.kind = kind;
        w.heads = kind == 0 ? p.Hq : p.H;
        w.h = skip * kHeads + sub;
        w.left = (kind == 0 ? p.q_steps : p.k_steps) - skip;
        w.stride = stride[2] * kHeads;
        w.src = static_cast<const uint16_t *>(kind == 0 ? p.q : kind == 1 ? p.k : p.v) + outer * stride[0] + lead * stride[1] + w.h * stride[2];
    };
    Walk load;
    if (first < p.q_steps)
        enter(load, 0, first);
    else if (first < p.q_steps + p.k_steps)
        enter(load, 1, first - p.q_steps);
    else
        enter(load, 2, first - p.q_steps - p.k_steps);
    const int first_kind = load.kind, first_skip = first - (load.kind == 0 ? 0 : load.kind == 1 ? p.q_steps : p.q_steps + p.k_steps);
    // The next kRing - 1 steps are on their way into shared memory (a lane copies and reads its own runs: no barrier), the first of them
    // before it is known where the row goes.  (ODD: the runs are not aligned, a step is loaded when its turn comes.)
    const bool has_a = na > 0, has_b = nb > 0;
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&ring[threadIdx.x / 32][0][0][lane]);
    uint32_t load_at = 0, read_at = 0;   // places in the ring
    int to_load = last - first;
    auto issue = [&]() {
        if constexpr (!ODD) {
            if (to_load > 0) {
                --to_load;
                if (load.left == 0) enter(load, load.kind + 1, 0);
                const bool there = load.h < load.heads;
                if (there && has_a) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + load_at), "l"(load.src + a) : "memory");
                if (there && has_b) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + load_at + 512), "l"(load.src + b) : "memory");
                load.src += load.stride;
                load.h += kHeads;
                --load.left;
                load_at = (load_at + 1024) % (kRing * 1024);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
#pragma unroll 1
    for (int k = 0; k < kRing - 1; ++k) issue();

    // whose row is it, and which of its tokens
    int seq = outer, at = lead, count;
    if (p.row_begin) {
        seq = sequence_of(p.row_begin, p.n_seq, row);
        at = seq < 0 ? 0 : row - p.row_begin[seq];
        count = seq < 0 ? 0 : p.row_begin[seq + 1] - p.row_begin[seq];
    } else
        count = p.n_new ? max(0, min(p.n_new[seq], p.per)) : p.per;
    if (at >= count) {   // not a token
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    const AttnSeg seg = p.segs[seq];
    const int64_t slot = (int64_t)own_tokens(p.seq_len, seq, seg.len) - count + at;
    if (at == 0 && part == 0 && lane == 0) report_length(p.seq_len, seq, seg.len, p.status);
    const bool cached = slot >= 0 && slot < seg.len;   // (a sequence shorter than its new tokens has no place for the first of them)
    char *place = nullptr;
    if (cached && last > p.q_steps)
        place = p.pool.base + 2 * (int64_t)p.layer * p.pool.lc_stride + slot_offset(p.pool, p.tbl, seg.tbl, (int)slot, p.block_shift);

    // cos and sin of the row's pairs, lane, lane + 32 ... by each lane
    float (&sc)[2][8 * W] = sines[threadIdx.x / 32];
    if (half > 0 && first < p.q_steps + p.k_steps) {
#pragma unroll
        for (int e = 0; e < W / 4; ++e) {
            const int pair = lane + 32 * e;
            if (pair < half) {
                const int axis = p.axis ? min((int)p.axis[pair], p.axes - 1) : 0;
                const int64_t pos = p.position ? p.position[axis * p.position_stride + row] : seg.before + slot;
                const int32_t turn = (int32_t)(((uint64_t)pos * p.turns[pair]) >> 32);
                float s, c;
                sincospif((float)turn * 0x1p-31f, &s, &c);   // half turns
                sc[0][pair] = c * p.rotary_scale;
                sc[1][pair] = s * p.rotary_scale;
            }
        }
        __syncwarp();
    }

    int steps = last - first;
#pragma unroll 1
    for (int kind = first_kind, skip = first_skip; steps > 0; ++kind, skip = 0) {
        const int count = min(steps, (kind == 0 ? p.q_steps : p.k_steps) - skip);
        steps -= count;
        if (count == 0) continue;
        const int heads = kind == 0 ? p.Hq : p.H;
        int h = skip * kHeads + sub;
        const int64_t out_stride = kind == 0 ? p.q_out_stride[2] : p.pool.head_stride / 2;   // elements between heads
        uint16_t *dst = (kind == 0 ? q_out : reinterpret_cast<uint16_t *>(place + (kind - 1) * p.pool.lc_stride)) + h * out_stride;
        const bool store = kind == 0 || cached, store_a = store && has_a, store_b = store && has_b;
        Walk odd;
        if constexpr (ODD) enter(odd, kind, skip);
        // y = x A + z B, z the other member of each pair
        float2 A[8], B[8];
        const float *norm = kind == 0 ? p.q_norm : kind == 1 ? p.k_norm : nullptr;
        if (kind < 2) {
            float w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = 1.f;
            if (norm) {
                if constexpr (ODD) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        w[e] = e < na ? norm[a + e] : 0.f;
                        w[8 + e] = e < nb ? norm[b + e] : 0.f;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4 *>(w + e) = *reinterpret_cast<const float4 *>(norm + (e < 8 ? a + e : b + e - 8));
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                A[e] = make_float2(w[2 * e], w[2 * e + 1]);
                B[e] = make_float2(0.f, 0.f);
            }
            if (8 * i < half) {
                float c[8], s[8];
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    *reinterpret_cast<float4 *>(c + e) = *reinterpret_cast<const float4 *>(&sc[0][8 * i + e]);
                    *reinterpret_cast<float4 *>(s + e) = *reinterpret_cast<const float4 *>(&sc[1][8 * i + e]);
                }
                if (ADJACENT) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!ODD || 8 * i + e < half) {
                            A[e] = make_float2(c[e] * w[2 * e], c[e] * w[2 * e + 1]);
                            B[e] = make_float2(-s[e] * w[2 * e + 1], s[e] * w[2 * e]);
                        }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        A[e] = make_float2(c[2 * e] * w[2 * e], c[2 * e + 1] * w[2 * e + 1]);
                        B[e] = make_float2(-s[2 * e] * w[8 + 2 * e], -s[2 * e + 1] * w[9 + 2 * e]);
                        A[4 + e] = make_float2(c[2 * e] * w[8 + 2 * e], c[2 * e + 1] * w[9 + 2 * e]);
                        B[4 + e] = make_float2(s[2 * e] * w[2 * e], s[2 * e + 1] * w[2 * e + 1]);
                    }
                }
            }
        }
#pragma unroll 1
        for (int n = count; n > 0; --n) {
            uint4 xa, xb;
            const bool there = h < heads;
            if constexpr (ODD) {
                xa = load8<true>(odd.src + a, there ? na : 0);
                xb = load8<true>(odd.src + b, there ? nb : 0);
                odd.src += odd.stride;
            } else {
                issue();
                asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
                // (what is not there holds anything, and stays in its lane but for the sum of squares)
                const char *at_ring = reinterpret_cast<const char *>(&ring[threadIdx.x / 32][0][0][lane]) + read_at;
                xa = *reinterpret_cast<const uint4 *>(at_ring);
                xb = *reinterpret_cast<const uint4 *>(at_ring + 512);
                read_at = (read_at + 1024) % (kRing * 1024);
            }
            if (kind < 2) {
                const uint32_t words[8] = {xa.x, xa.y, xa.z, xa.w, xb.x, xb.y, xb.z, xb.w};
                float2 x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = unpack2<T>(words[e]);
                float r = 1.f;
                if (norm) {
                    float2 sum_a = make_float2(0.f, 0.f), sum_b = sum_a;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sum_a = fma2(x[e], x[e], sum_a);
                        sum_b = fma2(x[4 + e], x[4 + e], sum_b);
                    }
                    float sum = (has_a ? sum_a.x + sum_a.y : 0.f) + (has_b ? sum_b.x + sum_b.y : 0.f);
#pragma unroll
                    for (int o = W / 2; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
                    r = rsqrtf(fmaf(sum, p.inv_D, p.eps));
                }
                if (8 * i < half) {
                    if (ADJACENT) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            y[e] = mul2(x[e], A[e]);
                            if (!ODD || 8 * i + e < half) y[e] = fma2(make_float2(x[e].y, x[e].x), B[e], y[e]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            y[e] = fma2(x[4 + e], B[e], mul2(x[e], A[e]));
                            y[4 + e] = fma2(x[e], B[4 + e], mul2(x[4 + e], A[4 + e]));
                        }
                    }
                } else {   // dims that do not turn are not mixed: 0 * infinity
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = mul2(x[e], A[e]);
                }
                if (norm) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = mul2(y[e], make_float2(r, r));
                }
                xa = make_uint4(pack2<T>(y[0].x, y[0].y), pack2<T>(y[1].x, y[1].y), pack2<T>(y[2].x, y[2].y), pack2<T>(y[3].x, y[3].y));
                xb = make_uint4(pack2<T>(y[4].x, y[4].y), pack2<T>(y[5].x, y[5].y), pack2<T>(y[6].x, y[6].y), pack2<T>(y[7].x, y[7].y));
            }
            store8<ODD>(dst + a, there && store_a ? na : 0, xa);
            store8<ODD>(dst + b, there && store_b ? nb : 0, xb);
            dst += kHeads * out_stride;
            h += kHeads;
        }
    }
}

namespace {

template <typename T, int W, bool ODD, bool ADJACENT> cudaError_t launch_append_as(AppendParams p, int sm_count, cudaStream_t stream)
{
    // A warp takes all heads of a row, which finds the row's sines once, where that gives each SM 16 warps; else it takes fewer (64 rows of
    // 48 heads: a step a warp 2.8 us, all 12 steps a warp would be 64 warps for 148 SMs; 4547 rows of 36 heads: all 9 steps 19.6 us, three 23.7).
    constexpr int heads = 32 / W;
    p.q_steps = (p.Hq + heads - 1) / heads;
    p.k_steps = (p.H + heads - 1) / heads;
    p.inv_D = 1.f / (float)p.D;
    const int steps = p.q_steps + 2 * p.k_steps;
    const int64_t most = (int64_t)p.rows * steps / (16 * sm_count);
    p.steps = (int)std::max<int64_t>(1, std::min<int64_t>(steps, most));
    p.parts = (steps + p.steps - 1) / p.steps;
    const int64_t blocks = ((int64_t)p.rows * p.parts + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kAppendThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // set up while the work before ends
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, append_kernel<T, W, ODD, ADJACENT>, p);
}

template <typename T, bool ADJACENT> cudaError_t launch_append_dims(const AppendParams &p, int sm_count, cudaStream_t stream)
{
    if (p.rotated / 2 % 8) return launch_append_as<T, 32, true, ADJACENT>(p, sm_count, stream);
    if (p.D <= 64) return launch_append_as<T, 4, false, ADJACENT>(p, sm_count, stream);
    if (p.D <= 128) return launch_append_as<T, 8, false, ADJACENT>(p, sm_count, stream);
    return launch_append_as<T, 16, false, ADJACENT>(p, sm_count, stream);
}
template <typename T> cudaError_t launch_append_type(const AppendParams &p, int sm_count, cudaStream_t stream)
{
    return p.adjacent ? launch_append_dims<T, true>(p, sm_count, stream) : launch_append_dims<T, false>(p, sm_count, stream);
}

}  // namespace

cudaError_t launch_append(AppendParams p, int dtype, int sm_count, cudaStream_t stream)
{
    return dtype == PDKV_DTYPE_BF16 ? launch_append_type<__nv_bfloat16>(p, sm_count, stream) : launch_append_type<__half>(p, sm_count, stream);
}

namespace {

constexpr int kAcceptThreads = 128;

// Accepted tokens of a sequence, 32 at a time: lane's entry of the path where the path reaches that far, -1 else.
__device__ __forceinline__ int path_entry(const AcceptParams &p, int seq, int from, int n_new, int last, int *count)
{
    const int lane = threadIdx.x % 32, j = from + lane;
    const int x = j < p.path_len ? p.path[seq * p.path_stride + j] : -1;
    int before = __shfl_up_sync(~0u, x, 1);
    if (lane == 0) before = last;
    const uint32_t ends = __ballot_sync(~0u, !(x > before && x < n_new));   // ascending, of the sequence's tokens
    *count = ends ? __ffs(ends) - 1 : 32;
    return lane < *count ? x : -1;
}

__device__ __forceinline__ int new_tokens_of(const AcceptParams &p, int seq)
{
    return p.n_new ? max(0, min(p.n_new[seq], p.new_tokens)) : p.new_tokens;
}

}  // namespace

// A CTA has one sequence and a run of 128 columns (V bytes of a head of a (layer, K/V) strip) of it.  Its first warp finds where the
// accepted tokens lie and where they go; a thread then moves its column of up to 32 tokens, all loads of eight before their stores.  In
// place that is safe without a barrier: entry j of an ascending path is at least j, so a place is written after the
// entries that might lie there were read, by the same thread.
// Bound by latency: lengths, path, table, rows, one after the other.  7 sequences of 13 drafted tokens, 5 layers of 5 heads of 80 dims
// 2.3 us in a recorded graph; 48 of up to 32, 32 layers of 8 heads of 128 dims 6.4 us (26.5 MB at 4.2 TB/s).
template <typename V> __global__ void __launch_bounds__(kAcceptThreads) accept_kernel(const __grid_constant__ AcceptParams p)
{
    __shared__ int64_t from[32], to[32];
    __shared__ int moves, state[2];   // accepted so far, last entry
    const int seq = blockIdx.x, lane = threadIdx.x % 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const AttnSeg seg = p.segs[seq];
    const int n_new = new_tokens_of(p, seq), first = own_tokens(p.seq_len, seq, seg.len) - n_new;
    const int vecs = p.row_bytes / (int)sizeof(V), columns = vecs * p.H;   // of a strip
    const int64_t column = (int64_t)blockIdx.y * kAcceptThreads + threadIdx.x;
    const bool mine = column < (int64_t)columns * p.n_lc;
    const int lc = (int)(column / columns), rest = (int)(column - (int64_t)lc * columns), head = rest / vecs;
    char *base = p.pool.base + (int64_t)(p.lc_begin + lc) * p.pool.lc_stride + head * p.pool.head_stride + (rest - head * vecs) * (int)sizeof(V);
    int accepted = 0, last = -1;
    while (true) {
        if (threadIdx.x < 32) {
            int count;
            const int x = path_entry(p, seq, accepted, n_new, last, &count);
            const int j = accepted + lane;
            // (tokens of a sequence shorter than its new tokens that have no place are not there)
            const bool moves_it = x > j && first + j >= 0;
            const uint32_t any = __ballot_sync(~0u, moves_it);
            if (moves_it) {
                const int k = __popc(any & ((1u << lane) - 1));
                from[k] = slot_offset(p.pool, p.tbl, seg.tbl, first + x, p.block_shift);
                to[k] = slot_offset(p.pool, p.tbl, seg.tbl, first + j, p.block_shift);
            }
            const int top = __shfl_sync(~0u, x, max(count - 1, 0));
            if (lane == 0) {
                moves = __popc(any);
                state[0] = accepted + count;
                state[1] = top;
            }
        }
        __syncthreads();
        const int n = moves, now = state[0];
        const bool more = now == accepted + 32 && now < p.path_len;
        last = state[1];
        if (mine)
            for (int j0 = 0; j0 < n; j0 += 8) {
                V x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j0 + j < n) x[j] = *reinterpret_cast<const V *>(base + from[j0 + j]);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j0 + j < n) *reinterpret_cast<V *>(base + to[j0 + j]) = x[j];
            }
        accepted = now;
        if (!more) break;
        __syncthreads();
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) {
        report_length(p.seq_len, seq, seg.len, p.status);
        if (p.new_len) p.new_len[seq] = max(0, first + accepted);
    }
}

// The new lengths alone, a warp a sequence: where they replace the lengths that the moves go by.
__global__ void __launch_bounds__(kAcceptThreads) accept_lens_kernel(const __grid_constant__ AcceptParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int seq = blockIdx.x * (kAcceptThreads / 32) + threadIdx.x / 32;
    if (seq >= p.n_seq) return;
    const int n_new = new_tokens_of(p, seq), first = own_tokens(p.seq_len, seq, p.segs[seq].len) - n_new;
    int accepted = 0, last = -1, count;
    do {
        const int x = path_entry(p, seq, accepted, n_new, last, &count);
        last = __shfl_sync(~0u, x, max(count - 1, 0));
        accepted += count;
    } while (count == 32 && accepted < p.path_len);
    if (threadIdx.x % 32 == 0) p.new_len[seq] = max(0, first + accepted);
}

namespace {

template <typename V> cudaError_t launch_accept_as(const AcceptParams &p, cudaStream_t stream)
{
    const int64_t columns = (int64_t)(p.row_bytes / (int)sizeof(V)) * p.H * p.n_lc, groups = (columns + kAcceptThreads - 1) / kAcceptThreads;
    if (groups > 65535) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kAcceptThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    AcceptParams moves = p;
    const bool in_place = p.new_len && p.new_len == p.seq_len;
    if (in_place) moves.new_len = nullptr;
    cfg.gridDim = dim3((unsigned)p.n_seq, (unsigned)groups);
    cudaError_t e = cudaLaunchKernelEx(&cfg, accept_kernel<V>, moves);
    if (e != cudaSuccess || !in_place) return e;
    cfg.gridDim = dim3((unsigned)((p.n_seq + kAcceptThreads / 32 - 1) / (kAcceptThreads / 32)));
    return cudaLaunchKernelEx(&cfg, accept_lens_kernel, p);
}

}  // namespace

cudaError_t launch_accept(const AcceptParams &p, cudaStream_t stream)
{
    switch (p.vec_bytes) {
    case 16: return launch_accept_as<uint4>(p, stream);
    case 8: return launch_accept_as<uint2>(p, stream);
    case 4: return launch_accept_as<uint32_t>(p, stream);
    case 2: return launch_accept_as<uint16_t>(p, stream);
    default: return launch_accept_as<uint8_t>(p, stream);
    }
}

}  // namespace pdkv
