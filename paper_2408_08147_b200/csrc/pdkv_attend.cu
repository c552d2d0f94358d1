// Attention of a batch's newest tokens over a paged pool, and the join of its parts.
#include <cmath>

#include "pdkv_attend_device.cuh"

namespace pdkv {

namespace {

constexpr int kConsumers = 128, kThreads = 160;   // four warps that compute, one that loads
constexpr int kSlice = 16;   // tokens of one ring slot: the depth of one matrix instruction in the product with V

// Shared memory of a CTA: a ring of slices, each 16 rows of K and 16 of V, in pieces of 64 dims whose 16-byte
// chunks are swizzled (chunk c of row r lies at c ^ (r mod 8): the TMA unit's 128-byte swizzle, and the eight
// rows of a matrix load lie in different banks); behind it the space through which warps join their
// results.  About 100 KB and two CTAs per SM up to 128 dims, 210 KB and one CTA above: 130 to 150 KB of
// loads in flight on each SM, twice what 6.5 TB/s at a microsecond of latency need.
template <int DP> struct Ring {
    static constexpr int kSubs = DP / 64;
    static constexpr int kSubBytes = kSlice * 128;
    static constexpr int kHalf = kSubs * kSubBytes;            // K or V of a slice
    static constexpr int kSliceBytes = 2 * kHalf;
    static constexpr int kSlots = DP == 64 ? 24 : DP == 192 ? 16 : 12;
    static constexpr int kQuarter = DP / 4;                    // dims that one warp of four joins
    static constexpr int kXchRow = kQuarter + 4;               // floats
    static constexpr int kXch = 4 * 16 * kXchRow * 4;
    static constexpr int kBytes = kSlots * kSliceBytes + kXch + 1024;
    static constexpr int kCtas = DP <= 128 ? 2 : 1;
};

struct RingBarriers {
    uint64_t full[24], empty[24];
};

// 16 bytes to shared memory; with `there` false zeros are written and nothing is read.
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
// This thread's arrival, once its copies so far have landed.
__device__ __forceinline__ void copy_arrive(uint64_t *b)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void mbar_arrive_many(uint64_t *b, uint32_t n)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}

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
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

__device__ __forceinline__ int slices_of(const AttnParams &p, const AttnItem &it, int *len, int *limit)
{
    *len = it.seq >= 0 ? own_len(p, it.seq, it.len) : it.len;
    *limit = min(it.tok1, *len);
    return *limit > it.tok0 ? (*limit - it.tok0 + kSlice - 1) / kSlice : 0;
}

// The loading warp: slices of all items in order, into the ring.  Where a slice lies within one block
// (block sizes that are multiples of 16) it is fetched by the TMA unit, a box of 64 dims per instruction; else
// by 16-byte asynchronous copies, each row looked up by its own lane.  It runs ahead of the computing warps
// across items, so memory stays busy while they join their results.
template <int DP>
__device__ __forceinline__ void load_slices(const AttnParams &p, const CUtensorMap *map, uint32_t ring, RingBarriers &bar, int first, int end)
{
    using R = Ring<DP>;
    const int lane = threadIdx.x % 32;
    const int cols = (p.D + 15) / 16 * 2;   // 16-byte pieces of a row; one past the row's end is filled with zeros
    bool dead = false;
    uint32_t slot = 0, parity = 1;
    for (int i = first; i < end; ++i) {
        const AttnItem it = p.items[i];
        int len, limit;
        const int count = slices_of(p, it, &len, &limit);
        if (p.use_map) {
            int block = 0;
            for (int s = 0; s < count; ++s) {
                const int t = it.tok0 + s * kSlice;
                if (s % 32 == 0) {   // blocks of the next 32 slices
                    const int tl = t + lane * kSlice;
                    if (tl < limit) block = p.tbl[it.tbl + (p.block_shift >= 0 ? tl >> p.block_shift : tl / p.pool.block_tokens)];
                }
                const int b = __shfl_sync(~0u, block, s % 32);
                const int tt = p.block_shift >= 0 ? t & (p.pool.block_tokens - 1) : t % p.pool.block_tokens;
                mbar_wait(&bar.empty[slot], parity, dead, p.status);
                dead = __any_sync(~0u, dead);
                if (!dead) {
                    if (lane == 0) mbar_expect(&bar.full[slot], R::kSliceBytes);
                    __syncwarp();
                    if (lane < 2 * R::kSubs) {
                        const int kv = lane / R::kSubs, sub = lane % R::kSubs, lc = 2 * p.layer + kv;
                        const uint32_t to = ring + slot * R::kSliceBytes + lane * R::kSubBytes;
                        if (p.map_layer_major)
                            load_box(to, map, 64 * sub, tt, it.head, b, lc, &bar.full[slot]);
                        else
                            load_box(to, map, 64 * sub, it.head, tt, lc, b, &bar.full[slot]);
                    }
                }
                if (++slot == R::kSlots) {
                    slot = 0;
                    parity ^= 1;
                }
            }
            continue;
        }
        const char *base = p.pool.base + 2 * (int64_t)p.layer * p.pool.lc_stride + it.head * p.pool.head_stride;
        // byte offset of token `lane` of a slice from `base`, -1: past the end
        auto offset_of = [&](int s) -> int64_t {
            const int t = it.tok0 + s * kSlice + lane % kSlice;
            if (t >= limit) return -1;
            const int b = p.block_shift >= 0 ? t >> p.block_shift : t / p.pool.block_tokens;
            return p.tbl[it.tbl + b] * p.pool.block_stride + (int64_t)(t - b * p.pool.block_tokens) * p.pool.tok_stride;
        };
        int64_t next = offset_of(0);
        for (int s = 0; s < count; ++s) {
            const int64_t offset = next;
            next = offset_of(s + 1);
            mbar_wait(&bar.empty[slot], parity, dead, p.status);
            dead = __any_sync(~0u, dead);
            const uint32_t to = ring + slot * R::kSliceBytes;
            if (!dead) {
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {   // 16 rows x DP / 8 pieces, 32 lanes
                    constexpr int kCols = DP / 8;
                    const int x = lane + 32 * k, row = x / kCols, col = x % kCols;
                    const int64_t o = __shfl_sync(~0u, offset, row);
                    if (col < cols) {
                        const bool there = o >= 0 && col * 8 < p.D;
                        const char *from = base + (there ? o + col * 16 : 0);
                        const uint32_t at = to + col / 8 * R::kSubBytes + row * 128 + (((col % 8) ^ (row % 8)) * 16);
                        copy_async(at, from, there);
                        copy_async(at + R::kHalf, from + p.pool.lc_stride, there);
                    }
                }
                copy_arrive(&bar.full[slot]);
            }
            if (++slot == R::kSlots) {
                slot = 0;
                parity ^= 1;
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// One work item with WM warps along the rows (16 each) and 4 / WM groups of warps along the tokens: group g
// takes slices g, g + groups, ...  `n` is the number of slices that went through the ring before.
//
// S = Q K^T and O += P V go through m16n8k16 matrix instructions with the rows (heads of one KV head,
// query tokens, sequences behind one prefix) as M; the maximum and sum of each row are kept per slice in 32
// bits, and O is only rescaled when a maximum moved.  The weights are rounded to 16 bits for the product
// with V (the matrix instruction takes no wider operand beside a 16-bit V); their sum is taken before that.
template <typename T, int DP, int WM>
__device__ __forceinline__ void attend_item(const AttnParams &p, const AttnItem &it, int n_slices, int len, int limit, char *smem,
                                            float (*sml)[16][2], RingBarriers &bar, uint32_t n, bool &dead)
{
    using R = Ring<DP>;
    constexpr int kGroups = 4 / WM;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, wm = warp % WM, group = warp / WM;
    const bool own = it.seq >= 0;
    const uint32_t ring = smem_u32(smem);

    // this lane's two rows: lane / 4 and lane / 4 + 8 of the warp's sixteen
    uint32_t q[DP / 16][4];
    int sees[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = wm * 16 + lane / 4 + 8 * half;
        const bool live = r < it.rows;
        const RowId id = row_id(p, it, it.row0 + (live ? r : 0));
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
        const AttnSeq s = p.seqs[it.seq];
        logits = p.logits + s.logits + ((int64_t)it.head * p.G * p.q_tokens + it.row0 + wm * 16 + lane / 4) * s.logit_stride;
        logit_row8 = 8 * (int64_t)s.logit_stride;
        store[0] = wm * 16 + lane / 4 < it.rows;
        store[1] = wm * 16 + lane / 4 + 8 < it.rows;
    }

    float o[DP / 8][4];
#pragma unroll
    for (int k = 0; k < DP / 8; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[k][j] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    // matrix loads: this lane's row of a slice, and which of the two 16-byte pieces of a step of 16 dims
    const uint32_t k_row = (lane / 16) * 8 + lane % 8, k_piece = lane / 8 % 2;
    const uint32_t v_row = (lane / 8 % 2) * 8 + lane % 8, v_piece = lane / 16;
    const uint32_t k_at = k_row * 128, v_at = R::kHalf + v_row * 128, turn = lane % 8;   // (row mod 8 is lane mod 8 for both)

    uint32_t slot = (n + group) % R::kSlots, parity = (n + group) / R::kSlots & 1;
#pragma unroll 1
    for (int s = group; s < n_slices; s += kGroups) {
        mbar_wait(&bar.full[slot], parity, dead, p.status);
        __syncwarp();
        const uint32_t slice = ring + slot * R::kSliceBytes;
        const int t0 = it.tok0 + s * kSlice;
        if (p.use_map && t0 + kSlice > limit) {
            // a box brings whole pages: rows of V past the end may hold anything, and 0 * NaN is NaN
            for (int x = lane; x < (t0 + kSlice - limit) * 8 * R::kSubs; x += 32) {
                const int row = limit - t0 + x / (8 * R::kSubs), piece = x % (8 * R::kSubs);
                *reinterpret_cast<uint4 *>(smem + slot * R::kSliceBytes + R::kHalf + piece / 8 * R::kSubBytes + row * 128 + piece % 8 * 16) =
                    make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();
            __syncwarp();
        }
        float z[2][4] = {};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
            if (16 * k < p.D) {
                uint32_t b[4];
                load_matrices(b, slice + k_at + k / 4 * R::kSubBytes + ((((k % 4) * 2 + k_piece) ^ turn) * 16));
                multiply<T>(z[0], q[k], b[0], b[1]);
                multiply<T>(z[1], q[k], b[2], b[3]);
            }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) z[i][j] *= p.scale_log2;
        if (t0 + kSlice > safe)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t0 + 8 * i + 2 * (lane % 4) + (j & 1) >= sees[j >> 1]) z[i][j] = -INFINITY;
        if (logits)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = t0 + 8 * i + 2 * (lane % 4);
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (store[half] && t < limit)
                        *reinterpret_cast<float2 *>(logits + half * logit_row8 + t) = make_float2(z[i][2 * half], z[i][2 * half + 1]);
            }
        float top[2], base[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float x = fmaxf(fmaxf(z[0][2 * half], z[0][2 * half + 1]), fmaxf(z[1][2 * half], z[1][2 * half + 1]));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
            top[half] = fmaxf(m[half], x);
            base[half] = top[half] == -INFINITY ? 0.f : top[half];
        }
        if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
            const float f0 = pow2(m[0] - base[0]), f1 = pow2(m[1] - base[1]);
            l[0] *= f0;
            l[1] *= f1;
#pragma unroll
            for (int k = 0; k < DP / 8; ++k) {
                o[k][0] *= f0;
                o[k][1] *= f0;
                o[k][2] *= f1;
                o[k][3] *= f1;
            }
            m[0] = top[0];
            m[1] = top[1];
        }
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float a = pow2(z[i][2 * half] - base[half]), b = pow2(z[i][2 * half + 1] - base[half]);
                l[half] += a + b;
                w[2 * i + half] = pack<T>(a, b);
            }
        }
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
            if (16 * k < p.D) {
                uint32_t b[4];
                load_matrices_trans(b, slice + v_at + k / 4 * R::kSubBytes + ((((k % 4) * 2 + v_piece) ^ turn) * 16));
                multiply<T>(o[2 * k], w, b[0], b[1]);
                multiply<T>(o[2 * k + 1], w, b[2], b[3]);
            }
        __syncwarp();
        if (lane == 0) mbar_arrive_many(&bar.empty[slot], kGroups);   // a slot is free after four arrivals
        slot += kGroups;
        if (slot >= R::kSlots) {
            slot -= R::kSlots;
            parity ^= 1;
        }
    }

#pragma unroll
    for (int half = 0; half < 2; ++half) {
        l[half] += __shfl_xor_sync(~0u, l[half], 1);
        l[half] += __shfl_xor_sync(~0u, l[half], 2);
    }
    // Join the groups: all take the largest maximum, then each warp collects its share of the dims -- a quarter
    // with four groups, two with two -- from the others, one quarter a round.
    constexpr int kTiles = R::kQuarter / 8;   // accumulator tiles of a quarter
    if (kGroups > 1) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
            if (lane % 4 == 0) *reinterpret_cast<float2 *>(sml[warp][lane / 4 + 8 * half]) = make_float2(m[half], l[half]);
        consumer_sync();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float mt = -INFINITY, lt = 0.f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) mt = fmaxf(mt, sml[g * WM + wm][lane / 4 + 8 * half][0]);
            const float b = mt == -INFINITY ? 0.f : mt;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const float *x = sml[g * WM + wm][lane / 4 + 8 * half];
                lt += pow2(x[0] - b) * x[1];
            }
            const float f = pow2(m[half] - b);
            m[half] = mt;
            l[half] = lt;
#pragma unroll
            for (int k = 0; k < DP / 8; ++k) {
                o[k][2 * half] *= f;
                o[k][2 * half + 1] *= f;
            }
        }
        float *xch = reinterpret_cast<float *>(smem + R::kSlots * R::kSliceBytes);
        float *mine = xch + (warp * 16 + lane / 4) * R::kXchRow + 2 * (lane % 4);
        constexpr int kRounds = kGroups == 4 ? 3 : 2;
#pragma unroll 1
        for (int round = 0; round < kRounds; ++round) {
            // the quarter that is given away, the one that is received, and from which warp
            const int away = kGroups == 4 ? (group + 1 + round) % 4 : 2 * (1 - group) + round;
            const int here = kGroups == 4 ? group : 2 * group + round;
            const int peer = kGroups == 4 ? (group + 3 - round) % 4 : (1 - group) * WM + wm;
#pragma unroll
            for (int quarter = 0; quarter < 4; ++quarter)
                if (quarter == away)
#pragma unroll
                    for (int k = 0; k < kTiles; ++k)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            *reinterpret_cast<float2 *>(mine + 8 * half * R::kXchRow + 8 * k) =
                                make_float2(o[quarter * kTiles + k][2 * half], o[quarter * kTiles + k][2 * half + 1]);
            consumer_sync();
            const float *theirs = xch + (peer * 16 + lane / 4) * R::kXchRow + 2 * (lane % 4);
#pragma unroll
            for (int quarter = 0; quarter < 4; ++quarter)
                if (quarter == here)
#pragma unroll
                    for (int k = 0; k < kTiles; ++k)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const float2 x = *reinterpret_cast<const float2 *>(theirs + 8 * half * R::kXchRow + 8 * k);
                            o[quarter * kTiles + k][2 * half] += x.x;
                            o[quarter * kTiles + k][2 * half + 1] += x.y;
                        }
            consumer_sync();
        }
    }
    if (dead) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = wm * 16 + lane / 4 + 8 * half;
        if (r >= it.rows) continue;
        const RowId id = row_id(p, it, it.row0 + r);
        const int head = it.head * p.G + id.g;
        const float inv = l[half] == 0.f ? 0.f : 1.f / l[half];
        T *out = static_cast<T *>(p.out) + id.seq * p.out_stride[0] + id.token * p.out_stride[1] + head * p.out_stride[2] + 2 * (lane % 4);
        float *part = p.part_o + (it.part_row + r) * p.D + 2 * (lane % 4);
#pragma unroll
        for (int k = 0; k < DP / 8; ++k) {
            const int quarter = k / kTiles;
            if ((kGroups == 1 || quarter / (4 / kGroups) == group) && 8 * k < p.D) {
                if (it.direct)
                    *reinterpret_cast<uint32_t *>(out + 8 * k) = pack<T>(o[k][2 * half] * inv, o[k][2 * half + 1] * inv);
                else
                    *reinterpret_cast<float2 *>(part + 8 * k) = make_float2(o[k][2 * half], o[k][2 * half + 1]);
            }
        }
        if (lane % 4 == 0 && group == 0) {
            if (it.direct && p.lse) p.lse[((int64_t)id.seq * p.q_tokens + id.token) * p.G * p.H + head] = (m[half] + log2f(l[half])) * kLn2;
            if (!it.direct || p.logits) *reinterpret_cast<float2 *>(p.part_ml + 2 * (it.part_row + r)) = make_float2(m[half], l[half]);
        }
    }
}

}  // namespace

// Every CTA walks its stretch of the work list.  Warps are laid along the rows as far as there are rows,
// the rest of them along the tokens.
template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, Ring<DP>::kCtas) attend_items_kernel(const __grid_constant__ CUtensorMap map, const AttnParams p)
{
    using R = Ring<DP>;
    extern __shared__ char raw[];
    __shared__ RingBarriers bar;
    __shared__ __align__(16) float sml[4][16][2];
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(raw) + 1023) / 1024 * 1024);
    const int first = p.cta_items[blockIdx.x], end = p.cta_items[blockIdx.x + 1];
    asm volatile("griddepcontrol.launch_dependents;");
    if (threadIdx.x < R::kSlots) {
        mbar_init(&bar.full[threadIdx.x], p.use_map ? 1 : 32);
        mbar_init(&bar.empty[threadIdx.x], 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (threadIdx.x >= kConsumers) {
        load_slices<DP>(p, &map, smem_u32(smem), bar, first, end);
        return;
    }
    bool dead = false;
    uint32_t n = 0;
    for (int i = first; i < end; ++i) {
        const AttnItem it = p.items[i];
        int len, limit;
        const int slices = slices_of(p, it, &len, &limit);
        if (it.rows <= 16)
            attend_item<T, DP, 1>(p, it, slices, len, limit, smem, sml, bar, n, dead);
        else if (it.rows <= 32)
            attend_item<T, DP, 2>(p, it, slices, len, limit, smem, sml, bar, n, dead);
        else
            attend_item<T, DP, 4>(p, it, slices, len, limit, smem, sml, bar, n, dead);
        n += slices;
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

template <typename T, int DP> cudaError_t launch_dims(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(attend_items_kernel<T, DP>, Ring<DP>::kBytes, ready);
    if (e != cudaSuccess) return e;
    attend_items_kernel<T, DP><<<p.n_ctas, kThreads, Ring<DP>::kBytes, stream>>>(map, p);
    return cudaGetLastError();
}

template <typename T> cudaError_t launch_type(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    if (p.D <= 64) return launch_dims<T, 64>(p, map, stream);
    if (p.D <= 128) return launch_dims<T, 128>(p, map, stream);
    if (p.D <= 192) return launch_dims<T, 192>(p, map, stream);
    return launch_dims<T, 256>(p, map, stream);
}

}  // namespace

int attend_ctas_per_sm(int head_dim) { return head_dim <= 128 ? 2 : 1; }

// Slices that lie within a block, rows that fill at least a box of 64 dims.
bool attend_map_supported(const pdkv_pool_desc &d)
{
    return d.elem_bytes == 2 && d.head_dim >= 64 && d.head_dim <= 256 && d.head_dim % 8 == 0 && d.block_tokens % kSlice == 0 &&
           d.num_blocks <= 0x7fffffff;
}
int attend_map_tokens() { return kSlice; }

cudaError_t launch_attend(const AttnParams &p, const void *map, int dtype, cudaStream_t stream)
{
    const CUtensorMap &m = *static_cast<const CUtensorMap *>(map);
    return dtype == PDKV_DTYPE_BF16 ? launch_type<__nv_bfloat16>(p, m, stream) : launch_type<__half>(p, m, stream);
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
