// The attention kernel of few rows and its launches.  Each form of attention is compiled in a file of its own.
#pragma once

#include <cmath>

#include "pdkv_attend_device.cuh"

namespace pdkv {

namespace {

constexpr int kConsumers = 128, kThreads = 160;   // four warps that compute, one that loads
constexpr int kSlice = 32;                        // tokens of one ring slot, the work of a warp between two waits

// Shared memory of a CTA: a ring of slices, each 32 rows of K and 32 of V, in pieces of 64 dims whose 16-byte
// chunks are swizzled (chunk c of row r lies at c ^ (r mod 8): the TMA unit's 128-byte swizzle, and the eight
// rows of a matrix load lie in different banks); behind it the space through which warps join their
// results.  80 to 96 KB of slices per CTA and two CTAs per SM up to 128 dims, 160 to 168 KB and one CTA above:
// twice the bytes in flight that 6.5 TB/s at a microsecond of latency need.
template <int DP> struct Ring {
    static constexpr int kSubs = DP / 64;
    static constexpr int kSubBytes = kSlice * 128;
    static constexpr int kHalf = kSubs * kSubBytes;            // K or V of a slice
    static constexpr int kSliceBytes = 2 * kHalf;
    static constexpr int kSlots = DP == 64 ? 12 : DP == 128 ? 5 : DP == 192 ? 7 : 5;
    static constexpr int kXchRow = DP + 4;                     // floats; 4 mod 16, so that a warp's stores do not collide
    static constexpr int kXch = 4 * 8 * kXchRow * 4;
    static constexpr int kBytes = kSlots * kSliceBytes + kXch + 1024;
    static constexpr int kCtas = DP <= 128 ? 2 : 1;
};

struct RingBarriers {
    uint64_t full[12], empty[12];
};

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
// Transposes an 8 x 8 tile of 16-bit numbers between the lanes of a warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int FORM> __device__ __forceinline__ int slices_of(const AttnParams &p, const AttnItem &it, int *len, int *limit)
{
    *len = it.seq >= 0 ? own_len(p, it.seq, it.len) : it.len;
    *limit = min(it.tok1, *len);
    if (FORM && nobody_there(p, it)) *limit = min(*limit, it.tok0);
    return *limit > it.tok0 ? (*limit - it.tok0 + kSlice - 1) / kSlice : 0;
}

// The loading warp: slices of all items in order, into the ring.  Where pages and slices divide one another
// they are fetched by the TMA unit, a box of 64 dims per instruction; else by 16-byte asynchronous copies,
// each row looked up by its own lane.  It runs ahead of the computing warps across items, so memory stays
// busy while they join their results.
template <int DP, int FORM>
__device__ __forceinline__ void load_slices(const AttnParams &p, const CUtensorMap *map, uint32_t ring, RingBarriers &bar, AttnItem it)
{
    using R = Ring<DP>;
    const int lane = threadIdx.x % 32;
    bool dead = false;
    uint32_t slot = 0, parity = 1;
    for (bool more = true; more;) {
        const AttnItem next_it = fetch_item(p.items, max(it.next, 0));   // in flight while this one is worked on
        more = it.next >= 0;
        int len, limit;
        const int count = slices_of<FORM>(p, it, &len, &limit);
        if (p.use_map) {
            // lane: page, then piece of 64 dims of K or V
            const int box = p.map_box, page = lane / (2 * R::kSubs), kv = lane / R::kSubs % 2, sub = lane % R::kSubs;
            auto block_of = [&](int s) {
                const int t = it.tok0 + s * kSlice + page * box;
                return page * box < kSlice && t < limit ? p.tbl[it.tbl + (p.block_shift >= 0 ? t >> p.block_shift : t / p.pool.block_tokens)] : -1;
            };
            int next = block_of(0);
            for (int s = 0; s < count; ++s) {
                const int block = next, t = it.tok0 + s * kSlice + page * box;
                next = block_of(s + 1);
                const int tt = p.block_shift >= 0 ? t & (p.pool.block_tokens - 1) : t % p.pool.block_tokens;
                const int boxes = __popc(__ballot_sync(~0u, block >= 0));   // pages past the end are not loaded
                mbar_wait(&bar.empty[slot], parity, dead, p.status);
                dead = __any_sync(~0u, dead);
                if (!dead) {
                    if (lane == 0) mbar_expect(&bar.full[slot], boxes * box * 128);
                    __syncwarp();
                    if (block >= 0) {
                        const uint32_t to = ring + slot * R::kSliceBytes + kv * R::kHalf + sub * R::kSubBytes + page * box * 128;
                        const int lc = 2 * p.layer + kv;
                        if (p.map_layer_major)
                            load_box(to, map, 64 * sub, tt, it.head, block, lc, &bar.full[slot]);
                        else
                            load_box(to, map, 64 * sub, it.head, tt, lc, block, &bar.full[slot]);
                    }
                }
                if (++slot == R::kSlots) {
                    slot = 0;
                    parity ^= 1;
                }
            }
            it = next_it;
            continue;
        }
        const char *base = p.pool.base + 2 * (int64_t)p.layer * p.pool.lc_stride + it.head * p.pool.head_stride;
        // byte offset of token `lane` of a slice from `base`, -1: past the end
        auto offset_of = [&](int s) -> int64_t {
            const int t = it.tok0 + s * kSlice + lane;
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
#pragma unroll 8
                for (int k = 0; k < kSlice * DP / 8 / 32; ++k) {   // 32 rows x DP / 8 pieces, 32 lanes
                    constexpr int kCols = DP / 8;
                    const int x = lane + 32 * k, row = x / kCols, col = x % kCols;
                    const int64_t o = __shfl_sync(~0u, offset, row);
                    const bool there = o >= 0 && col * 8 < p.D;   // else zeros
                    const char *from = base + (there ? o + col * 16 : 0);
                    const uint32_t at = to + col / 8 * R::kSubBytes + row * 128 + (((col % 8) ^ (row % 8)) * 16);
                    copy_async(at, from, there);
                    copy_async(at + R::kHalf, from + p.pool.lc_stride, there);
                }
                copy_arrive(&bar.full[slot]);
            }
            if (++slot == R::kSlots) {
                slot = 0;
                parity ^= 1;
            }
        }
        it = next_it;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Adds what was left out of the products of an item (see left_out) to its results: a warp a row, the rows and dims that the
// same thread has written.  A direct result has been rounded already, and such pieces of it are rounded twice.
template <typename T, int FORM>
__device__ __noinline__ void add_left_out(const AttnParams &p, const AttnItem it, int len, int limit, const float (*sml)[16][2], int nt, int wm)
{
    const int lane = threadIdx.x % 32, safe = min(limit, FORM ? len - newest_of(p, it.seq) : len - (p.q_tokens - 1));
    for (int r = threadIdx.x / 32; r < it.rows; r += 4) {
        const int w = r / (8 * nt), at = r % (8 * nt);
        float base = -INFINITY, sum = 0.f;
        for (int g = w; g < 4; g += wm) base = fmaxf(base, sml[g][at][0]);
        if (base == -INFINITY) continue;
        for (int g = w; g < 4; g += wm) sum += pow2(sml[g][at][0] - base) * sml[g][at][1];
        const RowId id = row_id(p, it, it.row0 + r);
        const int h = it.head * p.G + id.g, to = min(limit, len - (p.q_tokens - 1 - id.token));
        const T *q = static_cast<const T *>(p.q) + id.seq * p.q_stride[0] + id.token * p.q_stride[1] + h * p.q_stride[2];
        for (int d = 4 * lane; d < p.D; d += 128) {
            float4 y;
            if constexpr (FORM)
                y = left_out_formed<T>(p, q, it, id, len, max(safe, it.tok0), limit, base, d);
            else
                y = left_out<T>(p, q, it.tbl, it.head, max(safe, it.tok0), to, base, d);
            if (it.direct) {
                T *out = static_cast<T *>(p.out) + id.seq * p.out_stride[0] + id.token * p.out_stride[1] + h * p.out_stride[2] + d;
                const float inv = 1.f / sum;
                *reinterpret_cast<uint2 *>(out) = make_uint2(pack<T>(static_cast<float>(out[0]) + y.x * inv, static_cast<float>(out[1]) + y.y * inv),
                                                             pack<T>(static_cast<float>(out[2]) + y.z * inv, static_cast<float>(out[3]) + y.w * inv));
            } else {
                float4 *o = reinterpret_cast<float4 *>(p.part_o + (it.part_row + r) * p.D + d);
                *o = make_float4(o->x + y.x, o->y + y.y, o->z + y.z, o->w + y.w);
            }
        }
    }
}

// One work item with WM warps along the rows (8 NT each) and 4 / WM groups of warps along the tokens: group g
// takes slices g, g + groups, ...  `n` is the number of slices that went through the ring before.
//
// The products are turned round, so that the rows (heads of one KV head, query tokens, sequences behind one
// prefix), of which there are few, are the short side of the m16n8k16 matrix instructions:
//     S^T [token][row] = K Q^T       O^T [dim][row] += V^T P^T
// K and V are the 16-row operands, read from shared memory as they lie (V transposed by the matrix load), and
// eight rows cost half the instructions and registers that they would cost as one side of sixteen.  P^T
// changes from accumulator to operand layout by transposing its 8 x 8 tiles between lanes.
// Base and sum of each row are kept in 32 bits; O is rescaled only when a maximum outgrew its base by
// 2^8.  An instruction takes no wider operand beside a 16-bit V: up to 8 rows the weights go into the product as two 16-bit
// numbers, the second what the rounding to the first left (the tensor pipe has time: 32 x 2048 tokens 43.5 us either way, 256 small
// requests 79 -> 82); with more rows, which its registers and products bound, they are rounded (see kLift).  Their sum is taken
// before that.  KD: steps of 16 dims; behind the last dim Q, K and V are zero (a step that is skipped at run time keeps
// the loads of the next ones from being issued ahead: 40 rows of 256 dims 338 us, without 165).
//
// FORM: another form than plain causal.  The logits, once they are there, become what the form says (capped, biased, hidden by the
// rows' masks); from then on nothing else differs, but that a row may see nothing of what it is multiplied with.  A variant each for masks,
// caps and biases: with all in one (tanh from the exponential alone) 32 sequences of 2048 tokens, 4 rows, capped took 49.6 us instead of 46, 32 rows 92
// instead of 76.  Now, plain, with masks, capped, biased: 43.7, 46.8, 46.9, 47.0 and, 32 rows, 63, 72, 83, 82.  Every form spills registers (below).
template <typename T, int DP, int KD, bool HIDES, int FORM, int NT, int WM>
__device__ __forceinline__ void attend_item(const AttnParams &p, const AttnItem &it, int n_slices, int len, int limit, char *smem,
                                            float (*sml)[16][2], volatile uint32_t *wild, RingBarriers &bar, uint32_t n, bool &dead)
{
    using R = Ring<DP>;
    constexpr int kGroups = 4 / WM;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, wm = warp % WM, group = warp / WM;
    const bool own = it.seq >= 0;
    const uint32_t ring = smem_u32(smem);
    const float scale = FORM >= kCapped ? 1.f : fabsf(p.scale_log2);
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;   // a negative scale: the signs of Q are turned

    // operand Q^T: row lane / 4 of each tile of eight, dims 2 (lane % 4) and 8 further of each sixteen
    uint32_t q[KD][NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = (wm * NT + t) * 8 + lane / 4;
        const bool live = r < it.rows;
        const RowId id = row_id(p, it, it.row0 + (live ? r : 0));
        const T *row = static_cast<const T *>(p.q) + id.seq * p.q_stride[0] + id.token * p.q_stride[1] + (it.head * p.G + id.g) * p.q_stride[2];
#pragma unroll
        for (int k = 0; k < KD; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int d = 16 * k + 8 * j + 2 * (lane % 4);
                const uint32_t x = *reinterpret_cast<const uint32_t *>(row + min(d, p.D - 2));   // (always, so that all are on their way)
                q[k][t][j] = live && d < p.D ? x ^ flip : 0u;
            }
    }
    // accumulators: rows 2 (lane % 4) and the next of each tile of eight
    int sees[NT][2];
    float *logits[NT][2];
    int n_new = 0;           // FORM, own tokens: the newest of the sequence
    Bias bias[NT][2];
    if (FORM && own) n_new = newest_of(p, it.seq);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = (wm * NT + t) * 8 + 2 * (lane % 4) + j;
            const bool live = r < it.rows;
            sees[t][j] = limit;
            logits[t][j] = nullptr;
            if (FORM) {
                const RowId id = row_id(p, it, it.row0 + (live ? r : 0));
                if (id.token >= (own ? n_new : newest_of(p, id.seq))) sees[t][j] = 0;   // the query token is not there
                if (FORM == kSloped) bias[t][j] = bias_of(p, it, id, own ? len : own_len(p, id.seq, p.segs[id.seq].len));
            }
            if (own) {
                if (!FORM) sees[t][j] = min(limit, len - (p.q_tokens - 1 - (it.row0 + (live ? r : 0)) / p.G));
                if (!FORM && p.logits && live) {
                    const AttnSeq s = p.seqs[it.seq];
                    logits[t][j] = p.logits + s.logits + ((int64_t)it.head * p.G * p.q_tokens + it.row0 + r) * s.logit_stride;
                }
            }
        }
    const int safe = own ? min(limit, FORM ? len - n_new : len - (p.q_tokens - 1)) : limit;   // tokens before this one are seen by every row
    const bool with_logits = p.logits && own;

    float o[KD][NT][4];
#pragma unroll
    for (int k = 0; k < KD; ++k)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[k][t][j] = 0.f;
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.f;
    }
    // matrix loads.  K: lanes 0-7 rows 0-7, 8-15 rows 8-15, then the same 8 dims further.  V (transposed): lanes
    // 0-7 tokens 0-7, 8-15 the same 8 dims further, then tokens 8-15.  Row mod 8 is lane mod 8 for both.
    const uint32_t k_at = (lane % 16) * 128, v_at = R::kHalf + ((lane / 16) * 8 + lane % 8) * 128;
    uint32_t k_chunk[4], v_chunk[4];   // swizzled place of step s of 16 dims within a piece of 64
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        k_chunk[s] = ((2 * s + lane / 16) ^ (lane % 8)) * 16;
        v_chunk[s] = ((2 * s + lane / 8 % 2) ^ (lane % 8)) * 16;
    }

    uint32_t slot = (n + group) % R::kSlots, parity = (n + group) / R::kSlots & 1;
#pragma unroll 1
    for (int s = group; s < n_slices; s += kGroups) {
        // The parity of a barrier tells a phase from the next one only.  When the slots are not dealt to the groups
        // evenly, another group had this slot before and may not even have received its slice yet (copies
        // can land out of order): wait until it gave the slot back, then at most one phase is open.
        if (R::kSlots % 4 && n + s >= R::kSlots) mbar_wait(&bar.empty[slot], parity ^ 1, dead, p.status);
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
        if (HIDES && t0 + kSlice > safe) {   // see left_out
            const int row0 = max(safe - t0, 0), pieces = (min(limit - t0, kSlice) - row0) * 8 * R::kSubs;
            for (int x = lane; x < pieces; x += 32) {
                const int row = row0 + x / (8 * R::kSubs), piece = x % (8 * R::kSubs);
                uint4 *at = reinterpret_cast<uint4 *>(smem + slot * R::kSliceBytes + R::kHalf + piece / 8 * R::kSubBytes + row * 128 + piece % 8 * 16);
                if (any_not_finite<T>(*at)) {
                    *at = make_uint4(0, 0, 0, 0);
                    *wild = (uint32_t)it.part_row;
                }
            }
            fence_async_smem();
            __syncwarp();
        }
        float z[2][NT][4] = {};   // [16 tokens][8 rows]: tokens lane / 4 and 8 further
#pragma unroll
        for (int k = 0; k < KD; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t a[4];
                load_matrices(a, slice + k_at + h * 2048 + k / 4 * R::kSubBytes + k_chunk[k % 4]);
#pragma unroll
                for (int t = 0; t < NT; ++t) multiply<T>(z[h][t], a, q[k][t][0], q[k][t][1]);
            }
        if constexpr (FORM >= kCapped) {
            if (FORM == kCapped || p.cap_out != 0.f) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; j += 2) {
                            const float2 x = capped(p, make_float2(z[h][t][j], z[h][t][j + 1]));
                            z[h][t][j] = x.x;
                            z[h][t][j + 1] = x.y;
                        }
            }
        }
        if constexpr (FORM == kSloped) {
            const float in = p.cap_out != 0.f ? 1.f : fabsf(p.scale_log2);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const Bias b = bias[t][j & 1];
                    const int first = t0 + lane / 4 + 8 * (j >> 1) - b.query;
#pragma unroll
                    for (int h = 0; h < 2; ++h) z[h][t][j] = fmaf(b.slope, (float)(first + 16 * h), z[h][t][j] * in);
                }
        }
        if constexpr (FORM != kPlain) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (sees[t][j & 1] == 0) z[0][t][j] = z[1][t][j] = -INFINITY;
            if (own && t0 + kSlice > safe) {
                const int from = t0 - (len - n_new);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = (wm * NT + t) * 8 + 2 * (lane % 4) + j, token = (it.row0 + min(r, it.rows - 1)) / p.G;
                        const uint32_t seen = newest_seen(p, it.seq, token, n_new, from) >> (lane / 4);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {   // tokens lane / 4 + 8 x
                            float &y = z[x / 2][t][x % 2 * 2 + j];
                            if (!(seen >> (8 * x) & 1))
                                y = -INFINITY;
                            else if (FORM == kSloped && p.offset && from + lane / 4 + 8 * x >= 0)   // its place is not its slot
                                y = fmaf(bias[t][j].slope, (float)(offset_of(p, it.seq, from + lane / 4 + 8 * x) - (from + lane / 4 + 8 * x)), y);
                        }
                    }
            }
        }
        if ((FORM ? limit : safe) < t0 + kSlice)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (t0 + 16 * h + lane / 4 + 8 * (j >> 1) >= sees[t][j & 1]) z[h][t][j] = -INFINITY;
        if (with_logits)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int tok = t0 + 16 * h + lane / 4 + 8 * (j >> 1);
                        if constexpr (FORM != kPlain) {   // (where its row lies is found when it is wanted: that takes no registers)
                            const int r = (wm * NT + t) * 8 + 2 * (lane % 4) + (j & 1);
                            if (r < it.rows && tok < limit) {
                                const AttnSeq s = p.seqs[it.seq];
                                p.logits[s.logits + ((int64_t)it.head * p.G * p.q_tokens + it.row0 + r) * s.logit_stride + tok] =
                                    z[h][t][j] == -INFINITY ? -INFINITY : z[h][t][j] * scale;
                            }
                        } else if (logits[t][j & 1] && tok < limit)
                            logits[t][j & 1][tok] = z[h][t][j] == -INFINITY ? -INFINITY : z[h][t][j] * scale;
                    }
        float top[NT][2];
        bool grew = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x = fmaxf(fmaxf(z[0][t][j], z[0][t][j + 2]), fmaxf(z[1][t][j], z[1][t][j + 2]));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                top[t][j] = x == -INFINITY ? x : fmaf(x, scale, -kLift<T>);   // the base that this slice asks for
                grew = grew || top[t][j] > m[t][j] + kGrowth || (m[t][j] == -INFINITY && top[t][j] > m[t][j]);
            }
        if (__any_sync(~0u, grew)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // (FORM: the row's own maximum alone decides on its base, so that its neighbours change no bit of it)
                    const bool mine = top[t][j] > m[t][j] + kGrowth || (m[t][j] == -INFINITY && top[t][j] > m[t][j]);
                    const float new_m = !FORM || mine ? fmaxf(m[t][j], top[t][j]) : m[t][j], f = new_m == -INFINITY ? 1.f : pow2(m[t][j] - new_m);
                    m[t][j] = new_m;
                    l[t][j] *= f;
#pragma unroll
                    for (int k = 0; k < KD; ++k) {
                        o[k][t][j] *= f;
                        o[k][t][j + 2] *= f;
                    }
                }
        }
        constexpr bool kTwo = NT == 1;
        uint32_t w[2][NT][2], rest[2][2];   // operand P^T, and what its rounding left
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float b0 = m[t][0] == -INFINITY ? 0.f : m[t][0], b1 = m[t][1] == -INFINITY ? 0.f : m[t][1];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = pow2(fmaf(z[h][t][j], scale, j & 1 ? -b1 : -b0));
                    l[t][j & 1] += x;
                    z[h][t][j] = x;
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t two = pack<T>(z[h][t][2 * j], z[h][t][2 * j + 1]);
                    w[h][t][j] = transpose8(two);
                    if (kTwo) rest[h][j] = transpose8(pack<T>(z[h][t][2 * j] - unpack<T>(two & 0xffffu), z[h][t][2 * j + 1] - unpack<T>(two >> 16)));
                }
            }
        }
#pragma unroll
        for (int k = 0; k < KD; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t a[4];
                load_matrices_trans(a, slice + v_at + h * 2048 + k / 4 * R::kSubBytes + v_chunk[k % 4]);
#pragma unroll
                for (int t = 0; t < NT; ++t) multiply<T>(o[k][t], a, w[h][t][0], w[h][t][1]);
                if (kTwo) multiply<T>(o[k][0], a, rest[h][0], rest[h][1]);
            }
        __syncwarp();
        if (lane == 0) mbar_arrive_many(&bar.empty[slot], kGroups);   // a slot is free after four arrivals
        slot += kGroups;
        if (slot >= R::kSlots) {
            slot -= R::kSlots;
            parity ^= 1;
        }
    }

    // Join the groups: every warp writes its maxima and sums and, eight rows at a time, its O; a warp per row
    // adds them up and writes the result.
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int x = 4; x < 32; x *= 2) l[t][j] += __shfl_xor_sync(~0u, l[t][j], x);
            if (lane < 4) *reinterpret_cast<float2 *>(sml[warp][t * 8 + 2 * lane + j]) = make_float2(m[t][j], l[t][j]);
        }
    float *xch = reinterpret_cast<float *>(smem + R::kSlots * R::kSliceBytes);
    bool pieces_left_out = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float *mine = xch + (warp * 8 + 2 * (lane % 4)) * R::kXchRow + lane / 4;
#pragma unroll
        for (int k = 0; k < KD; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) mine[(j & 1) * R::kXchRow + 16 * k + 8 * (j >> 1)] = o[k][t][j];
        consumer_sync();
        if (HIDES && t == 0) pieces_left_out = *wild == (uint32_t)it.part_row;   // (the next item may set it after the last barrier here)
#pragma unroll 1
        for (int x = warp; x < WM * 8; x += 4) {
            const int w = x / 8, r = (w * NT + t) * 8 + x % 8;   // row of the item: warp w of each group has it
            if (r >= it.rows) continue;
            float mt = -INFINITY, lt = 0.f, f[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) mt = fmaxf(mt, sml[g * WM + w][t * 8 + x % 8][0]);
            const float b = mt == -INFINITY ? 0.f : mt;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                f[g] = pow2(sml[g * WM + w][t * 8 + x % 8][0] - b);
                lt += f[g] * sml[g * WM + w][t * 8 + x % 8][1];
            }
            if (dead) continue;
            T *out = nullptr;
            float inv = 1.f;
            if (it.direct) {   // own tokens: whose row it is, is known without a load
                const RowId id = row_id(p, it, it.row0 + r);
                const int head = it.head * p.G + id.g;
                inv = lt == 0.f ? 0.f : 1.f / lt;
                out = static_cast<T *>(p.out) + id.seq * p.out_stride[0] + id.token * p.out_stride[1] + head * p.out_stride[2];
                if (p.lse && lane == 0) p.lse[((int64_t)id.seq * p.q_tokens + id.token) * p.G * p.H + head] = (mt + log2f(lt)) * kLn2;
            }
#pragma unroll
            for (int d0 = 0; d0 < DP; d0 += 128) {
                const int d = d0 + 4 * lane;
                if (d >= p.D) continue;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (FORM && lt == 0.f) break;   // a row that saw nothing: its products may be 0 * infinity
                    const float4 y = *reinterpret_cast<const float4 *>(xch + ((g * WM + w) * 8 + x % 8) * R::kXchRow + d);
                    v.x += f[g] * y.x;
                    v.y += f[g] * y.y;
                    v.z += f[g] * y.z;
                    v.w += f[g] * y.w;
                }
                if (it.direct)
                    *reinterpret_cast<uint2 *>(out + d) = make_uint2(pack<T>(v.x * inv, v.y * inv), pack<T>(v.z * inv, v.w * inv));
                else
                    *reinterpret_cast<float4 *>(p.part_o + (it.part_row + r) * p.D + d) = v;
            }
            if (lane == 0 && (!it.direct || p.with_scores)) *reinterpret_cast<float2 *>(p.part_ml + 2 * (it.part_row + r)) = make_float2(mt, lt);
        }
        consumer_sync();
    }
    if (HIDES && pieces_left_out) {
        if (!dead) add_left_out<T, FORM>(p, it, len, limit, sml, NT, WM);
        consumer_sync();
    }
}

}  // namespace

// Every CTA walks its stretch of the work list.  Warps are laid along the rows as far as there are rows,
// the rest of them along the tokens.
// Bound by memory up to 16 rows: 32 sequences of 2048 tokens, 8 heads of 128 dims, 4 rows each 43.6 us (6.2 TB/s of K and V),
// 2 sequences of about 110000 tokens, 8 rows each, 6.4 TB/s.  Above, by the products of the four warps, or eight, of an SM
// (64 rows of 256 dims over 40000 tokens 169 us, 8 rows 60).  Bytes of registers that ptxas spills (bf16; stored), plain, with masks, capped, biased: 64
// dims 0, 112, 120, 220; 96 dims 64, 204, 176, 228; 128 dims 160, 320, 388, 556; 192 dims 24, 68, 76, 52; 256 dims 188, 396, 576, 672.  The matrix instructions of this kind are enough here: 8 rows at full memory rate keep
// them busy for 13% of the time.
template <typename T, int DP, int KD, bool HIDES, int FORM>
__global__ void __launch_bounds__(kThreads, Ring<DP>::kCtas) attend_items_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnParams p)
{
    using R = Ring<DP>;
    extern __shared__ char raw[];
    __shared__ RingBarriers bar;
    __shared__ __align__(16) float sml[4][16][2];
    __shared__ uint32_t wild;   // first partial row (every item has another) of the last item some of whose values were left out
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(raw) + 1023) / 1024 * 1024);
    AttnItem it = fetch_item(p.items, blockIdx.x);
    if (threadIdx.x == 0) wild = ~0u;
    if (threadIdx.x < R::kSlots) {
        mbar_init(&bar.full[threadIdx.x], p.use_map ? 1 : 32);
        mbar_init(&bar.empty[threadIdx.x], 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == kConsumers && p.n_tile_ctas > 0) {   // (see below; for the CTA, by the barrier.  A fence took 3 us of a call of 64)
        unsigned long long any;
        asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(any) : "l"(p.status) : "memory");
    }
    __syncthreads();
    if (threadIdx.x == kConsumers) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
    // The first kernel of a call is set up while the work before it ends.  Behind the tile kernel of the same call it does not
    // wait: it would wait for the whole of that kernel, which it is to run beside.  It starts once every CTA of that kernel has
    // seen the work before the call complete (griddepcontrol.wait) and has said so (launch_dependents).  PTX promises what that
    // work wrote only to a grid that waits itself, so this goes beyond it by one step: a CTA that started after
    // that completion finds the writes in L2, and the acquiring load above and the fence below keep it from anything older.
    if (p.n_tile_ctas == 0)
        asm volatile("griddepcontrol.wait;" ::: "memory");
    else if (threadIdx.x == kConsumers)
        asm volatile("fence.proxy.async.global;" ::: "memory");   // its loads of K and V
    asm volatile("griddepcontrol.launch_dependents;");
    if (threadIdx.x >= kConsumers) {
        load_slices<DP, FORM>(p, &map, smem_u32(smem), bar, it);
    } else {
        bool dead = false;
        uint32_t n = 0;
        for (bool more = true; more;) {
            const AttnItem next_it = fetch_item(p.items, max(it.next, 0));
            more = it.next >= 0;
            int len, limit;
            const int slices = slices_of<FORM>(p, it, &len, &limit);
            if (it.rows <= 8)
                attend_item<T, DP, KD, HIDES, FORM, 1, 1>(p, it, slices, len, limit, smem, sml, &wild, bar, n, dead);
            else if (it.rows <= 16)
                attend_item<T, DP, KD, HIDES, FORM, 2, 1>(p, it, slices, len, limit, smem, sml, &wild, bar, n, dead);
            else if (it.rows <= 32)
                attend_item<T, DP, KD, HIDES, FORM, 2, 2>(p, it, slices, len, limit, smem, sml, &wild, bar, n, dead);
            else
                attend_item<T, DP, KD, HIDES, FORM, 2, 4>(p, it, slices, len, limit, smem, sml, &wild, bar, n, dead);
            n += slices;
            it = next_it;
        }
    }
    // This kernel may run beside the tile kernel launched before it, which it does not depend on; whoever waits for
    // this one has to find both complete.
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

namespace {

template <typename T, int DP, int KD, bool HIDES, int FORM> cudaError_t launch_hides(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(attend_items_kernel<T, DP, KD, HIDES, FORM>, Ring<DP>::kBytes, ready);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.n_ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Ring<DP>::kBytes;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // beside the tile kernel, or early
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_items_kernel<T, DP, KD, HIDES, FORM>, map, p);
}

// With one query token every row sees every token: without the code for tokens that some rows do not see, 256 small requests behind
// a prefix take 79 us instead of 83.
template <typename T, int DP, int KD, int FORM> cudaError_t launch_dims(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    if constexpr (FORM == kPlain)
        if (p.q_tokens == 1) return launch_hides<T, DP, KD, false, FORM>(p, map, stream);
    return launch_hides<T, DP, KD, true, FORM>(p, map, stream);
}

template <typename T, int FORM> cudaError_t launch_type(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    // shared memory in pieces of 64 dims, products in steps that cover the head
    if (p.D <= 64) return launch_dims<T, 64, 4, FORM>(p, map, stream);
    if (p.D <= 96) return launch_dims<T, 128, 6, FORM>(p, map, stream);
    if (p.D <= 128) return launch_dims<T, 128, 8, FORM>(p, map, stream);
    if (p.D <= 192) return launch_dims<T, 192, 12, FORM>(p, map, stream);
    return launch_dims<T, 256, 16, FORM>(p, map, stream);
}

template <int FORM> cudaError_t launch_warp_kernel(const AttnParams &p, const void *map, int dtype, cudaStream_t stream)
{
    const CUtensorMap &m = *static_cast<const CUtensorMap *>(map);
    return dtype == PDKV_DTYPE_BF16 ? launch_type<__nv_bfloat16, FORM>(p, m, stream) : launch_type<__half, FORM>(p, m, stream);
}

}  // namespace

}  // namespace pdkv
