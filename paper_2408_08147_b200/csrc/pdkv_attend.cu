// Attention of a batch's newest tokens over a paged pool, and the join of its parts.
#include <cmath>

#include "pdkv_attend_device.cuh"

namespace pdkv {

namespace {

constexpr int kThreads = 128;
constexpr int kSlice = 16;   // tokens of one pipeline slice: the depth of one matrix instruction in the product with V

// Shared memory of a CTA: a ring of slices, each 16 rows of K and 16 of V.  Rows are padded by 16
// bytes, an odd number of 16-byte pieces, so that the eight rows of a matrix load lie in different banks.
// About 100 KB of slices per CTA and two CTAs per SM up to 128 dims, 200 KB and one CTA above: 130 to
// 150 KB of loads in flight on each SM, twice what 6.5 TB/s at a microsecond of latency need.
template <int DP> struct Ring {
    static constexpr int kRow = 2 * DP + 16;
    static constexpr int kSliceBytes = 2 * kSlice * kRow;
    static constexpr int kSlices = DP <= 64 ? 20 : DP <= 96 ? 16 : DP <= 128 ? 12 : DP <= 192 ? 16 : 12;
    static constexpr int kBytes = kSlices * kSliceBytes;
    static constexpr int kCtas = DP <= 128 ? 2 : 1;
};

// 16 bytes to shared memory; with `there` false zeros are written and nothing is read.
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_trans(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <typename T> __device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void multiply<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void multiply<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int N> __device__ __forceinline__ void group_sync(int id)
{
    if (N == 32)
        __syncwarp();
    else
        asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(N) : "memory");
}

// One work item with WM warps along the rows (16 each) and 4 / WM groups of warps along the tokens.
//
// Every group runs its own pipeline over its slices (group, group + groups, ...): wait for a slice,
// issue the load of the one `stages - 1` later, multiply.  S = Q K^T and O += P V go through
// m16n8k16 matrix instructions with the rows (heads of one KV head, query tokens, sequences behind one
// prefix) as M; the maximum and sum of each row are kept per slice in 32 bits, and O is only rescaled
// when a maximum moved.  The weights are rounded to 16 bits for the product with V (the matrix
// instruction takes no wider operand beside a 16-bit V); their sum is taken before that.
template <typename T, int DP, int WM>
__device__ __forceinline__ void attend_item(const AttnParams &p, const AttnItem &it, char *smem)
{
    using R = Ring<DP>;
    constexpr int kGroups = 4 / WM, kGroupThreads = 32 * WM, kStages = R::kSlices / kGroups, kCols = DP / 8;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, wm = warp % WM, group = warp / WM;
    const int tid = wm * 32 + lane;
    const AttnSeg seg = p.segs[it.seg];
    const bool own = seg.seq >= 0;
    const int len = own ? own_len(p, seg.seq, seg.len) : seg.len;
    const int limit = min(it.tok1, len);
    const int n_slices = limit > it.tok0 ? (limit - it.tok0 + kSlice - 1) / kSlice : 0;
    const int count = n_slices > group ? (n_slices - group + kGroups - 1) / kGroups : 0;
    const int cols = (p.D + 15) / 16 * 2;   // 16-byte pieces of a row; one past the row's end is filled with zeros
    char *ring = smem + group * kStages * R::kSliceBytes;
    const char *base = p.pool.base + 2 * (int64_t)p.layer * p.pool.lc_stride + it.head * p.pool.head_stride;

    // byte offset of token (slice, lane) from `base`, -1: past the end
    auto offset_of = [&](int slice) -> int64_t {
        const int t = it.tok0 + (group + slice * kGroups) * kSlice + lane % kSlice;
        if (slice >= count || t >= limit) return -1;
        const int b = p.block_shift >= 0 ? t >> p.block_shift : t / p.pool.block_tokens;
        return p.tbl[seg.tbl + b] * p.pool.block_stride + (int64_t)(t - b * p.pool.block_tokens) * p.pool.tok_stride;
    };
    auto load = [&](int slice, int64_t offset) {
        const uint32_t to = smem_u32(ring + (slice % kStages) * R::kSliceBytes);
#pragma unroll
        for (int i = 0; i < (kSlice * kCols + kGroupThreads - 1) / kGroupThreads; ++i) {
            const int x = tid + i * kGroupThreads, row = x / kCols, col = x % kCols;
            const int64_t o = __shfl_sync(~0u, offset, row % kSlice);
            if (row < kSlice && col < cols) {
                const bool there = o >= 0 && col * 8 < p.D;
                const char *k = base + (there ? o + col * 16 : 0);
                copy_async(to + row * R::kRow + col * 16, k, there);
                copy_async(to + kSlice * R::kRow + row * R::kRow + col * 16, k + p.pool.lc_stride, there);
            }
        }
    };

    int64_t offset = offset_of(0);
#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) {
        const int64_t next = offset_of(i + 1);
        if (i < count) load(i, offset);
        copy_commit();
        offset = next;
    }

    // this lane's two rows: lane / 4 and lane / 4 + 8 of the warp's sixteen
    uint32_t q[DP / 16][4];
    int sees[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = wm * 16 + lane / 4 + 8 * half;
        const bool live = r < it.rows;
        const RowId id = row_id(p, seg, it.row0 + (live ? r : 0));
        sees[half] = own ? min(limit, len - (p.q_tokens - 1 - id.token)) : limit;
        const T *row = static_cast<const T *>(p.q) + id.seq * p.q_stride[0] + id.token * p.q_stride[1] + (it.head * p.G + id.g) * p.q_stride[2];
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int d = 16 * k + 8 * j + 2 * (lane % 4);
                q[k][half + 2 * j] = live && d < p.D ? *reinterpret_cast<const uint32_t *>(row + d) : 0u;
            }
    }
    const int safe = own ? min(limit, len - (p.q_tokens - 1)) : limit;   // tokens before this one are seen by every row
    float *logits = nullptr;
    int64_t logit_row8 = 0;
    bool store[2] = {false, false};
    if (p.logits && own) {
        const AttnSeq s = p.seqs[seg.seq];
        logits = p.logits + s.logits + ((int64_t)it.head * p.G * p.q_tokens + it.row0 + wm * 16 + lane / 4) * s.logit_stride;
        logit_row8 = 8 * (int64_t)s.logit_stride;
        store[0] = wm * 16 + lane / 4 < it.rows;
        store[1] = wm * 16 + lane / 4 + 8 < it.rows;
    }

    float o[DP / 8][4];
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[n][j] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    // addresses of the matrix loads of this lane inside a slice
    const uint32_t k_at = ((lane / 16) * 8 + lane % 8) * R::kRow + (lane / 8 % 2) * 16;
    const uint32_t v_at = kSlice * R::kRow + ((lane / 8 % 2) * 8 + lane % 8) * R::kRow + (lane / 16) * 16;

#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        copy_wait<kStages - 2>();
        group_sync<kGroupThreads>(1 + group);
        {
            const int64_t next = offset_of(i + kStages);
            if (i + kStages - 1 < count) load(i + kStages - 1, offset);
            copy_commit();
            offset = next;
        }
        const uint32_t slice = smem_u32(ring + (i % kStages) * R::kSliceBytes);
        float z[2][4] = {};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
            if (16 * k < p.D) {
                uint32_t b[4];
                load_matrices(b, slice + k_at + k * 32);
                multiply<T>(z[0], q[k], b[0], b[1]);
                multiply<T>(z[1], q[k], b[2], b[3]);
            }
        const int t0 = it.tok0 + (group + i * kGroups) * kSlice;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) z[n][j] *= p.scale_log2;
        if (t0 + kSlice > safe)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t0 + 8 * n + 2 * (lane % 4) + (j & 1) >= sees[j >> 1]) z[n][j] = -INFINITY;
        if (logits)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int t = t0 + 8 * n + 2 * (lane % 4);
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (store[half] && t < limit)
                        *reinterpret_cast<float2 *>(logits + half * logit_row8 + t) = make_float2(z[n][2 * half], z[n][2 * half + 1]);
            }
        float top[2], base2[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float x = fmaxf(fmaxf(z[0][2 * half], z[0][2 * half + 1]), fmaxf(z[1][2 * half], z[1][2 * half + 1]));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
            top[half] = fmaxf(m[half], x);
            base2[half] = top[half] == -INFINITY ? 0.f : top[half];
        }
        if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
            const float f0 = pow2(m[0] - base2[0]), f1 = pow2(m[1] - base2[1]);
            l[0] *= f0;
            l[1] *= f1;
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                o[n][0] *= f0;
                o[n][1] *= f0;
                o[n][2] *= f1;
                o[n][3] *= f1;
            }
            m[0] = top[0];
            m[1] = top[1];
        }
        uint32_t w[4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float a = pow2(z[n][2 * half] - base2[half]), b = pow2(z[n][2 * half + 1] - base2[half]);
                l[half] += a + b;
                w[2 * n + half] = pack<T>(a, b);
            }
        }
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
            if (16 * k < p.D) {
                uint32_t b[4];
                load_matrices_trans(b, slice + v_at + k * 32);
                multiply<T>(o[2 * k], w, b[0], b[1]);
                multiply<T>(o[2 * k + 1], w, b[2], b[3]);
            }
    }

    // join the groups through the ring's memory: [warp][16 rows][DP + 4] and [warp][16 rows][2]
    copy_wait<0>();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        l[half] += __shfl_xor_sync(~0u, l[half], 1);
        l[half] += __shfl_xor_sync(~0u, l[half], 2);
    }
    __syncthreads();
    constexpr int kOut = DP + 4;
    float *so = reinterpret_cast<float *>(smem), *sml = so + 4 * 16 * kOut;
    static_assert((4 * 16 * kOut + 4 * 16 * 2) * 4 <= R::kBytes, "the join fits the ring");
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = warp * 16 + lane / 4 + 8 * half;
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
            *reinterpret_cast<float2 *>(so + r * kOut + 8 * n + 2 * (lane % 4)) = make_float2(o[n][2 * half], o[n][2 * half + 1]);
        if (lane % 4 == 0) *reinterpret_cast<float2 *>(sml + 2 * r) = make_float2(m[half], l[half]);
    }
    __syncthreads();
    for (int r = warp; r < it.rows; r += 4) {
        float mt = -INFINITY, lt = 0.f, f[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) mt = fmaxf(mt, sml[2 * (g * WM * 16 + r)]);
        const float b2 = mt == -INFINITY ? 0.f : mt;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            f[g] = pow2(sml[2 * (g * WM * 16 + r)] - b2);
            lt += f[g] * sml[2 * (g * WM * 16 + r) + 1];
        }
        const RowId id = row_id(p, seg, it.row0 + r);
        const int head = it.head * p.G + id.g;
        const float inv = lt == 0.f ? 0.f : 1.f / lt;
        T *out = static_cast<T *>(p.out) + id.seq * p.out_stride[0] + id.token * p.out_stride[1] + head * p.out_stride[2];
        for (int d = 4 * lane; d < p.D; d += 128) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const float4 x = *reinterpret_cast<const float4 *>(so + (g * WM * 16 + r) * kOut + d);
                v.x += f[g] * x.x;
                v.y += f[g] * x.y;
                v.z += f[g] * x.z;
                v.w += f[g] * x.w;
            }
            if (it.direct)
                *reinterpret_cast<uint2 *>(out + d) = make_uint2(pack<T>(v.x * inv, v.y * inv), pack<T>(v.z * inv, v.w * inv));
            else
                *reinterpret_cast<float4 *>(p.part_o + (it.part_row + r) * p.D + d) = v;
        }
        if (lane == 0) {
            if (it.direct && p.lse) p.lse[((int64_t)id.seq * p.q_tokens + id.token) * p.G * p.H + head] = (mt + log2f(lt)) * kLn2;
            if (!it.direct || p.logits) *reinterpret_cast<float2 *>(p.part_ml + 2 * (it.part_row + r)) = make_float2(mt, lt);
        }
    }
    __syncthreads();
}

}  // namespace

// Every CTA walks its stretch of the work list.  Warps are laid along the rows as far as there are rows,
// the rest of them along the tokens.
template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, Ring<DP>::kCtas) attend_items_kernel(const AttnParams p)
{
    extern __shared__ __align__(128) char smem[];
    asm volatile("griddepcontrol.launch_dependents;");
    const int end = p.cta_items[blockIdx.x + 1];
    for (int i = p.cta_items[blockIdx.x]; i < end; ++i) {
        const AttnItem it = p.items[i];
        if (it.rows <= 16)
            attend_item<T, DP, 1>(p, it, smem);
        else if (it.rows <= 32)
            attend_item<T, DP, 2>(p, it, smem);
        else
            attend_item<T, DP, 4>(p, it, smem);
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

// Maximum and sum of a row over all of its parts, by W neighbouring lanes; each of them gets both.
template <int W> __device__ __forceinline__ float2 joined_ml(const AttnParams &p, const Parts &x, int lane)
{
    const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml);
    float m = -INFINITY, l = 0.f;
    for (int i = lane % W; i < x.n[0] + x.n[1]; i += W) {
        const float2 v = ml[part_at(x, i)];
        const float top = fmaxf(m, v.x), base = top == -INFINITY ? 0.f : top;
        l = l * pow2(m - base) + v.y * pow2(v.x - base);
        m = top;
    }
#pragma unroll
    for (int o = W / 2; o; o /= 2) {
        const float m2 = __shfl_xor_sync(~0u, m, o), l2 = __shfl_xor_sync(~0u, l, o);
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
        l = l * pow2(m - base) + l2 * pow2(m2 - base);
        m = top;
    }
    return make_float2(m, l);
}

constexpr int kScoreChunk = 512;   // tokens of one block of the score part
constexpr int kScoreRows = 64;     // rows whose lse is held at a time

}  // namespace

// The first `row_blocks` blocks of a (sequence, head) join the parts of four rows each, a warp per row:
// m = max m_p, l = sum l_p 2^(m_p - m), O = sum O_p 2^(m_p - m).  The others turn the logits of a chunk of
// tokens into weights 2^(z - lse) and add them to the scores; they take the lse from the parts themselves
// (eight lanes a row), so no block waits for another.
template <typename T>
__global__ void __launch_bounds__(128) attend_join_kernel(const AttnParams p, const int row_blocks, const int chunks)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, per = row_blocks + chunks;
    const int x = blockIdx.x % per, head = blockIdx.x / per % p.H, seq = blockIdx.x / per / p.H;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the parts are written by the kernel before
    const AttnSeq s = p.seqs[seq];
    const int R = p.G * p.q_tokens;
    if (x < row_blocks) {
        const int row = 4 * x + warp;
        if (s.direct || row >= R) return;
        const Parts parts = parts_of(p, s, head, row);
        const int n = parts.n[0] + parts.n[1];
        const float2 ml = joined_ml<32>(p, parts, lane);
        const float base = ml.x == -INFINITY ? 0.f : ml.x;
        float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        for (int i0 = 0; i0 < n; i0 += 32) {
            const float w = i0 + lane < n ? pow2(p.part_ml[2 * part_at(parts, i0 + lane)] - base) : 0.f;
            const int top = min(32, n - i0);
#pragma unroll 8
            for (int i = 0; i < top; ++i) {
                const float wi = __shfl_sync(~0u, w, i);
                const float4 *o = reinterpret_cast<const float4 *>(p.part_o + part_at(parts, i0 + i) * p.D);
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
    const int chunk = x - row_blocks, len = own_len(p, seq, s.len), t0 = chunk * kScoreChunk + 4 * threadIdx.x;
    // past the sequence's end there is no weight: nothing to do in place, else the row is carried over
    const int width = p.scores_in == p.scores_out ? len : p.max_len;
    if (chunk * kScoreChunk >= width) return;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < R; r0 += kScoreRows) {
        const int n = min(kScoreRows, R - r0);
        __syncthreads();
        for (int r = warp * 4; r < n; r += 16) {
            const int row = r + lane / 8;
            const float2 ml = joined_ml<8>(p, parts_of(p, s, head, r0 + min(row, n - 1)), lane);
            // an empty row gives no weight to anything: 2^(z - inf) = 0
            if (lane % 8 == 0 && row < n) lse[row] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
        }
        __syncthreads();
        const float *z = p.logits + s.logits + ((int64_t)head * R + r0) * s.logit_stride + t0;
        if (t0 < len) {
#pragma unroll 4
            for (int row = 0; row < n; ++row) {
                const float4 v = *reinterpret_cast<const float4 *>(z + (int64_t)row * s.logit_stride);
                const float e = lse[row];
                sum[0] += pow2(v.x - e);
                sum[1] += pow2(v.y - e);
                sum[2] += pow2(v.z - e);
                sum[3] += pow2(v.w - e);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (t0 + k < width) {
            const float in = p.scores_in ? p.scores_in[seq * p.scores_in_stride[0] + head * p.scores_in_stride[1] + t0 + k] : 0.f;
            // (what lies in the scratch behind the last token is no logit)
            p.scores_out[seq * p.scores_out_stride[0] + head * p.scores_out_stride[1] + t0 + k] = t0 + k < len ? in + sum[k] : in;
        }
}

namespace {

template <typename T, int DP> cudaError_t launch_dims(const AttnParams &p, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(attend_items_kernel<T, DP>, Ring<DP>::kBytes, ready);
    if (e != cudaSuccess) return e;
    attend_items_kernel<T, DP><<<p.n_ctas, kThreads, Ring<DP>::kBytes, stream>>>(p);
    return cudaGetLastError();
}

template <typename T> cudaError_t launch_type(const AttnParams &p, cudaStream_t stream)
{
    if (p.D <= 64) return launch_dims<T, 64>(p, stream);
    if (p.D <= 96) return launch_dims<T, 96>(p, stream);
    if (p.D <= 128) return launch_dims<T, 128>(p, stream);
    if (p.D <= 192) return launch_dims<T, 192>(p, stream);
    return launch_dims<T, 256>(p, stream);
}

}  // namespace

int attend_ctas_per_sm(int head_dim) { return head_dim <= 128 ? 2 : 1; }

cudaError_t launch_attend(const AttnParams &p, int dtype, cudaStream_t stream)
{
    return dtype == PDKV_DTYPE_BF16 ? launch_type<__nv_bfloat16>(p, stream) : launch_type<__half>(p, stream);
}

cudaError_t launch_attend_join(const AttnParams &p, int dtype, bool join, cudaStream_t stream)
{
    const int row_blocks = join ? (p.G * p.q_tokens + 3) / 4 : 0;
    const int chunks = p.logits ? (p.max_len + kScoreChunk - 1) / kScoreChunk : 0;
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
    cfg.numAttrs = p.n_ctas > 0 || p.n_tile_ctas > 0 ? 1 : 0;
    if (dtype == PDKV_DTYPE_BF16) return cudaLaunchKernelEx(&cfg, attend_join_kernel<__nv_bfloat16>, p, row_blocks, chunks);
    return cudaLaunchKernelEx(&cfg, attend_join_kernel<__half>, p, row_blocks, chunks);
}

}  // namespace pdkv
