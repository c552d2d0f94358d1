// New tokens into a paged pool, their queries and keys normalised and rotated on the way; and the tokens of an accepted path
// to the place behind what they follow.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pdkv_append.h"

namespace pdkv {

namespace {

constexpr int kAppendThreads = 128;
constexpr int kBatch = 4;          // steps whose loads are on their way together

__device__ __forceinline__ int own_tokens(const int32_t *seq_len, int seq, int most)
{
    if (!seq_len) return most;
    const int n = seq_len[seq];
    return n < 0 ? 0 : (n < most ? n : most);
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

// A warp has one row (token) and, a step at a time, 32 / W of its heads: queries, then keys, then values.  W lanes have a head, each
// two runs of eight dims, chosen so that both members of a rotated pair lie in one lane, which then has eight pairs:
//     y = x w / sqrt(mean x^2 + eps)      (a, b) -> (a cos - b sin, b cos + a sin), the angle position * frequency
// The sines serve all heads of the row; the lanes of one step share the work of finding them.  The angle is kept in turns as a 64-bit
// fraction, position * frequency wraps at whole turns by itself, and its upper 32 bits are exact to 2^-32 of a turn at any position
// (position * frequency in 32-bit floating point is off by 0.004 at 100000).  Everything between load and store is 32 bits, rounded once.
//
// ODD: half of the rotated dims is no multiple of eight.  Pairs (i, i + half) then lie in runs that are not aligned: a lane takes up
// to eight pairs, or up to sixteen of the dims behind them, in 16-bit pieces.
template <typename T, int W, bool ODD>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendParams p)
{
    constexpr int kHeads = 32 / W;   // of a step
    const int lane = threadIdx.x % 32, sub = lane / W, i = lane % W;
    const int64_t item = (int64_t)blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32;
    const int row = (int)(item / p.parts), part = (int)(item - (int64_t)row * p.parts);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    if (row >= p.rows) return;   // (whole warps)

    // which dims are this lane's: na from a, nb from b
    const int half = p.rotated / 2;
    int a, b, na, nb;
    if (p.adjacent) {
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

    const int first = part * p.steps * kHeads, slots = p.Hq + 2 * p.H;
    const int last = min(slots, first + p.steps * kHeads);   // heads [first, last) of the row

    // whose row is it, and which of its tokens
    int seq, at, count;
    if (p.row_begin) {
        seq = sequence_of(p.row_begin, p.n_seq, row);
        if (seq < 0) return;
        at = row - p.row_begin[seq];
        count = p.row_begin[seq + 1] - p.row_begin[seq];
    } else {
        seq = row / p.per;
        at = row - seq * p.per;
        count = p.n_new ? max(0, min(p.n_new[seq], p.per)) : p.per;
    }
    if (at >= count) return;   // not a token
    const int64_t lead = p.row_begin ? row : at, outer = p.row_begin ? 0 : seq;
    const uint16_t *q = static_cast<const uint16_t *>(p.q) + outer * p.q_stride[0] + lead * p.q_stride[1];
    const uint16_t *k = static_cast<const uint16_t *>(p.k) + outer * p.k_stride[0] + lead * p.k_stride[1];
    const uint16_t *v = static_cast<const uint16_t *>(p.v) + outer * p.v_stride[0] + lead * p.v_stride[1];
    uint16_t *q_out = static_cast<uint16_t *>(p.q_out) + outer * p.q_out_stride[0] + lead * p.q_out_stride[1];
    // values of step s: head `first + s * kHeads + sub` of queries, keys, values
    auto source = [&](int h) {
        return h < p.Hq ? q + h * p.q_stride[2] : h < p.Hq + p.H ? k + (h - p.Hq) * p.k_stride[2] : v + (h - p.Hq - p.H) * p.v_stride[2];
    };
    uint4 xa[kBatch], xb[kBatch];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int s = 0; s < kBatch; ++s) {
            const int h = h0 + s * kHeads + sub;
            const bool there = h < last;
            const uint16_t *from = source(there ? h : first);
            xa[s] = load8<ODD>(from + (na > 0 ? a : 0), there ? na : 0);
            xb[s] = load8<ODD>(from + (nb > 0 ? b : 0), there ? nb : 0);
        }
    };
    fetch(first);

    const AttnSeg seg = p.segs[seq];
    const int64_t slot = (int64_t)own_tokens(p.seq_len, seq, seg.len) - count + at;
    const bool cached = slot >= 0 && slot < seg.len;   // (a sequence shorter than its new tokens has no place for the first of them)
    char *place = nullptr;
    if (cached && last > p.Hq)
        place = p.pool.base + 2 * (int64_t)p.layer * p.pool.lc_stride + slot_offset(p.pool, p.tbl, seg.tbl, (int)slot, p.block_shift);

    // cos and sin of the lane's pairs 8i..8i+7; the kHeads lanes with the same dims find 8 / kHeads each
    float cosine[8], sine[8];
    const bool turns = p.rotated > 0 && first < p.Hq + p.H;
    if (turns) {
        constexpr int kMine = 8 / kHeads;
        float c[kMine], s[kMine];
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
            const int pair = 8 * i + sub * kMine + e;
            c[e] = 1.f;
            s[e] = 0.f;
            if (pair < half) {
                const int axis = p.axis ? min((int)p.axis[pair], p.axes - 1) : 0;
                const int64_t pos = p.position ? p.position[axis * p.position_stride + row] : seg.before + slot;
                const int32_t turn = (int32_t)(((uint64_t)pos * p.turns[pair]) >> 32);
                sincospif((float)turn * 0x1p-31f, &s[e], &c[e]);   // half turns
                c[e] *= p.rotary_scale;
                s[e] *= p.rotary_scale;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            cosine[e] = __shfl_sync(~0u, c[e % kMine], e / kMine * W + i);
            sine[e] = __shfl_sync(~0u, s[e % kMine], e / kMine * W + i);
        }
    }
    float w[16];
    const float *have = nullptr;   // whose weights w are
    for (int h0 = first; h0 < last; h0 += kBatch * kHeads) {
        if (h0 > first) fetch(h0);
#pragma unroll
        for (int s = 0; s < kBatch; ++s) {
            const int h = h0 + s * kHeads + sub;
            if (h0 + s * kHeads >= last) break;   // (the whole warp)
            const bool value = h >= p.Hq + p.H, query = h < p.Hq;
            uint4 ya = xa[s], yb = xb[s];
            if (h0 + s * kHeads < p.Hq + p.H) {   // (the whole warp: some lanes have queries or keys)
                float x[16];   // a in the first eight, b in the others
                const uint32_t words[8] = {ya.x, ya.y, ya.z, ya.w, yb.x, yb.y, yb.z, yb.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 f = unpack2<T>(words[e]);
                    x[2 * e] = f.x;
                    x[2 * e + 1] = f.y;
                }
                const float *norm = query ? p.q_norm : value ? nullptr : p.k_norm;
                if (__any_sync(~0u, norm != nullptr)) {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
                    for (int o = W / 2; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
                    if (norm) {
                        if (norm != have) {
                            have = norm;
                            if (ODD) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    w[e] = e < na ? norm[a + e] : 0.f;
                                    w[8 + e] = e < nb ? norm[b + e] : 0.f;
                                }
                            } else {
#pragma unroll
                                for (int e = 0; e < 16; e += 4)
                                    *reinterpret_cast<float4 *>(w + e) = (e < 8 ? na : nb) > 0 ? *reinterpret_cast<const float4 *>(norm + (e < 8 ? a + e : b + e - 8))
                                                                                              : make_float4(0.f, 0.f, 0.f, 0.f);
                            }
                        }
                        const float r = 1.f / sqrtf(sum / p.D + p.eps);
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] *= r * w[e];
                    }
                }
                if (turns && 8 * i < half) {
                    if (p.adjacent) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (!ODD || 8 * i + e < half) {
                                const float u = x[2 * e], t = x[2 * e + 1];
                                x[2 * e] = u * cosine[e] - t * sine[e];
                                x[2 * e + 1] = t * cosine[e] + u * sine[e];
                            }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float u = x[e], t = x[8 + e];
                            x[e] = u * cosine[e] - t * sine[e];
                            x[8 + e] = t * cosine[e] + u * sine[e];
                        }
                    }
                }
                if (!value) {
                    ya = make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
                    yb = make_uint4(pack2<T>(x[8], x[9]), pack2<T>(x[10], x[11]), pack2<T>(x[12], x[13]), pack2<T>(x[14], x[15]));
                }
            }
            if (h < last) {
                uint16_t *to = nullptr;
                if (query)
                    to = q_out + h * p.q_out_stride[2];
                else if (cached)
                    to = reinterpret_cast<uint16_t *>(place + (value ? p.pool.lc_stride : 0) + (h - p.Hq - (value ? p.H : 0)) * p.pool.head_stride);
                if (to) {
                    store8<ODD>(to + (na > 0 ? a : 0), na, ya);
                    store8<ODD>(to + (nb > 0 ? b : 0), nb, yb);
                }
            }
        }
    }
}

namespace {

template <typename T, int W, bool ODD> cudaError_t launch_append_as(AppendParams p, int sm_count, cudaStream_t stream)
{
    // A warp takes all heads of a row, which finds the row's sines once, where that gives each SM 16 warps; else it takes fewer.
    const int heads = 32 / W, steps = (p.Hq + 2 * p.H + heads - 1) / heads;
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
    return cudaLaunchKernelEx(&cfg, append_kernel<T, W, ODD>, p);
}

template <typename T> cudaError_t launch_append_type(const AppendParams &p, int sm_count, cudaStream_t stream)
{
    if (p.rotated / 2 % 8) return launch_append_as<T, 32, true>(p, sm_count, stream);
    if (p.D <= 64) return launch_append_as<T, 4, false>(p, sm_count, stream);
    if (p.D <= 128) return launch_append_as<T, 8, false>(p, sm_count, stream);
    return launch_append_as<T, 16, false>(p, sm_count, stream);
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
// Bound by latency: lengths, path, table, rows, one after the other.
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
    if (p.new_len && blockIdx.y == 0 && threadIdx.x == 0) p.new_len[seq] = max(0, first + accepted);
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
