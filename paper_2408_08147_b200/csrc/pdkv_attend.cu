// Attention of a batch's newest tokens over a paged pool, and the join of its parts.
#include <numeric>
#include <type_traits>

#include "pdkv_attend_warp.cuh"

namespace pdkv {

namespace {

// Tokens of one block of the score part: four a thread, and either each warp has tokens of its own, or -- many
// rows -- all warps have the same and share the rows.
constexpr int kSharedRows = 12;
__host__ __device__ constexpr int score_chunk(int rows) { return rows > kSharedRows ? 128 : 512; }
constexpr int kScoreRows = 64;     // rows whose lse is held at a time

}  // namespace

// The first `row_blocks` blocks of a (sequence, head) join the parts of four rows each, a warp per row, or (WIDE: rows in
// many parts) of one row, each warp every fourth part:
// m = max m_p, l = sum l_p 2^(m_p - m), O = sum O_p 2^(m_p - m).  The others turn the logits of a chunk of
// tokens into weights 2^(z - lse) and add them to the scores; they take the lse from the parts themselves, so no
// block waits for another.  Bound by the latency of its few dependent loads: 4096 rows of 128 dims in four parts each 10 us
// alone, about 4 us behind the kernel that left them, since it is set up while that one ends.
template <typename T, bool WIDE, bool FORM>
__global__ void __launch_bounds__(128) attend_join_kernel(const AttnParams p, const int row_blocks, const int chunks)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, per = row_blocks + chunks;
    const int x = blockIdx.x % per, head = blockIdx.x / per % p.H, seq = blockIdx.x / per / p.H;
    const AttnSeq s = p.seqs[seq];
    const int R = p.G * p.q_tokens;
    constexpr int ways = WIDE ? 4 : 1;
    const int row = WIDE ? x : 4 * x + warp, way = WIDE ? warp : 0;
    const bool mine = x < row_blocks && !s.direct && row < R;
    Parts parts{};
    if (mine) parts = parts_of(p, s, head, row);         // where they are is known before they are written
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the parts are written by the kernels before
    asm volatile("griddepcontrol.launch_dependents;");
    if (x < row_blocks) {
        if (!mine) return;
        const bool absent = FORM && row / p.G >= newest_of(p, seq);   // a query token that is not there: nothing, and its parts may hold anything
        const int n = absent ? 0 : (parts.n[0] + parts.n[1] - way + ways - 1) / ways;   // of this warp: way, way + ways, ...
        const float2 ml = absent ? make_float2(-INFINITY, 0.f) : joined_ml<32>(p, parts, lane);
        const float base = ml.x == -INFINITY ? 0.f : ml.x;
        float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        for (int i0 = 0; i0 < n; i0 += 32) {
            const float w = i0 + lane < n ? pow2(p.part_ml[2 * part_at(parts, (i0 + lane) * ways + way)] - base) : 0.f;
            const int top = min(32, n - i0);
#pragma unroll 8
            for (int i = 0; i < top; ++i) {
                const float wi = __shfl_sync(~0u, w, i);
                const float4 *o = reinterpret_cast<const float4 *>(p.part_o + part_at(parts, (i0 + i) * ways + way) * p.D);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (4 * (lane + 32 * k) < p.D) {
                        const float4 v = o[lane + 32 * k];
                        acc[k].x += wi * v.x;
                        acc[k].y += wi * v.y;
                        acc[k].z += wi * v.z;
                        acc[k].w += wi * v.w;
                    }
            }
        }
        if (WIDE) {
            __shared__ float4 others[3][64];
            if (warp > 0) {
                others[warp - 1][lane] = acc[0];
                others[warp - 1][lane + 32] = acc[1];
            }
            __syncthreads();   // (a block has one row: all warps come here)
            if (warp > 0) return;
#pragma unroll
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float4 v = others[w][lane + 32 * k];
                    acc[k].x += v.x;
                    acc[k].y += v.y;
                    acc[k].z += v.z;
                    acc[k].w += v.w;
                }
        }
        const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
        const int token = row / p.G, h = head * p.G + row % p.G;
        T *out = static_cast<T *>(p.out) + seq * p.out_stride[0] + token * p.out_stride[1] + h * p.out_stride[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (4 * (lane + 32 * k) < p.D)
                *reinterpret_cast<uint2 *>(out + 4 * (lane + 32 * k)) =
                    make_uint2(pack<T>(acc[k].x * inv, acc[k].y * inv), pack<T>(acc[k].z * inv, acc[k].w * inv));
        if (p.lse && lane == 0) p.lse[((int64_t)seq * p.q_tokens + token) * p.G * p.H + h] = (ml.x + log2f(ml.y)) * kLn2;
        return;
    }
    __shared__ float lse[kScoreRows];
    __shared__ float4 sums[4][32];
    const bool shared = R > kSharedRows;
    const int begin = (x - row_blocks) * score_chunk(R), len = own_len(p, seq, s.len), t0 = begin + (shared ? 0 : 128 * warp) + 4 * lane;
    // past the sequence's end there is no weight: nothing to do in place, else the row is carried over
    const int width = p.scores_in == p.scores_out ? len : p.max_len;
    if (begin >= width) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    // Rows of query tokens that are not there, the last ones, weigh nothing, and their logits may never have been written.
    const int rows = FORM ? min(R, newest_of(p, seq) * p.G) : R;
    // (a token that a row does not see weighs nothing even where the row's sum is NaN)
    auto weight = [](float z, float e) { return z == -INFINITY ? 0.f : pow2(z - e); };
    for (int r0 = 0; r0 < rows; r0 += kScoreRows) {
        const int n = min(kScoreRows, rows - r0);
        __syncthreads();
        for (int r = warp; WIDE && r < n; r += 4) {
            const float2 ml = joined_ml<32>(p, parts_of(p, s, head, r0 + r), lane);
            if (lane == 0) lse[r] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
        }
        for (int r = warp * 8; !WIDE && r < n; r += 32) {
            const int row = r + lane / 4;
            const float2 ml = joined_ml<4>(p, parts_of(p, s, head, r0 + min(row, n - 1)), lane);
            // an empty row gives no weight to anything: 2^(z - inf) = 0
            if (lane % 4 == 0 && row < n) lse[row] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
        }
        __syncthreads();
        const float *z = p.logits + s.logits + ((int64_t)head * R + r0) * s.logit_stride + t0;
        if (t0 < len) {
#pragma unroll 4
            for (int row = shared ? warp : 0; row < n; row += shared ? 4 : 1) {
                const float4 v = *reinterpret_cast<const float4 *>(z + (int64_t)row * s.logit_stride);
                const float e = lse[row];
                sum.x += weight(v.x, e);
                sum.y += weight(v.y, e);
                sum.z += weight(v.z, e);
                sum.w += weight(v.w, e);
            }
        }
    }
    auto put = [&](int t, float add) {
        if (t >= width) return;
        const float in = p.scores_in ? p.scores_in[seq * p.scores_in_stride[0] + head * p.scores_in_stride[1] + t] : 0.f;
        // (what lies in the scratch behind the last token is no logit)
        p.scores_out[seq * p.scores_out_stride[0] + head * p.scores_out_stride[1] + t] = t < len ? in + add : in;
    };
    sums[warp][lane] = sum;
    if (shared) {
        __syncthreads();
        float add = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) add += reinterpret_cast<const float *>(sums[w])[threadIdx.x];
        put(begin + threadIdx.x, add);
    } else {   // neighbouring lanes store neighbouring tokens
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) put(begin + 128 * warp + 32 * k + lane, reinterpret_cast<const float *>(sums[warp])[32 * k + lane]);
    }
}

int attend_ctas_per_sm(int head_dim) { return head_dim <= 128 ? 2 : 1; }

// Blocks of a multiple of 8 tokens, rows that fill at least a box of 64 dims.  A box holds as many tokens as
// divide both a block and a slice (8 at least: the period of the swizzle), so it lies within one block.
bool attend_map_supported(const pdkv_pool_desc &d)
{
    return d.elem_bytes == 2 && d.head_dim >= 64 && d.head_dim <= 256 && d.head_dim % 8 == 0 && d.num_blocks <= 0x7fffffff && d.block_tokens % 8 == 0;
}
int attend_map_box(const pdkv_pool_desc &d) { return std::gcd(d.block_tokens, kSlice); }

cudaError_t launch_attend(const AttnParams &p, const void *map, int dtype, cudaStream_t stream)
{
    switch (p.formed) {
    case kMasked: return launch_attend_masked(p, map, dtype, stream);
    case kCapped: return launch_attend_capped(p, map, dtype, stream);
    case kSloped: return launch_attend_sloped(p, map, dtype, stream);
    default: return launch_warp_kernel<kPlain>(p, map, dtype, stream);
    }
}

cudaError_t launch_attend_join(const AttnParams &p, int dtype, bool join, int most_parts, cudaStream_t stream)
{
    // A row in hundreds of parts would keep one warp waiting for them: 12 rows in 290 parts each 51 us a call, 23 with four warps a row
    const bool wide = most_parts > 16;
    const int rows = p.G * p.q_tokens, row_blocks = join ? (wide ? rows : (rows + 3) / 4) : 0;
    const int per = score_chunk(p.G * p.q_tokens), chunks = p.logits ? (p.max_len + per - 1) / per : 0;
    const int64_t blocks = (int64_t)p.n_seq * p.H * (row_blocks + chunks);
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    if (blocks == 0) return cudaSuccess;
    // May be launched before the kernel in front of it has finished; it waits on the device for its results.
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(128);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    auto launch = [&](auto type, auto formed) {
        using T = decltype(type);
        constexpr bool FORM = decltype(formed)::value;
        return cudaLaunchKernelEx(&cfg, wide ? attend_join_kernel<T, true, FORM> : attend_join_kernel<T, false, FORM>, p, row_blocks, chunks);
    };
    if (dtype == PDKV_DTYPE_BF16) return p.formed ? launch(__nv_bfloat16(), std::true_type()) : launch(__nv_bfloat16(), std::false_type());
    return p.formed ? launch(__half(), std::true_type()) : launch(__half(), std::false_type());
}

}  // namespace pdkv
