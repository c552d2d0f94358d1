// Device code shared by the attention kernels.
#pragma once

#include <atomic>
#include <cmath>

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pdkv_seqs.h"

namespace pdkv {

constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

__device__ __forceinline__ int own_len(const AttnParams &p, int seq, int cap)
{
    if (!p.seq_len) return cap;
    const int n = p.seq_len[seq];
    return n < 0 ? 0 : (n < cap ? n : cap);
}

__device__ __forceinline__ AttnItem fetch_item(const AttnItem *items, int i)
{
    AttnItem it;
    const uint4 *from = reinterpret_cast<const uint4 *>(items + i);
    uint4 *to = reinterpret_cast<uint4 *>(&it);
#pragma unroll
    for (int k = 0; k < 4; ++k) to[k] = __ldg(from + k);
    return it;
}

struct RowId {
    int seq, token, g;
};
// Row `row` of an item's segment: which query token of which sequence, and which of the G heads.
__device__ __forceinline__ RowId row_id(const AttnParams &p, const AttnItem &seg, int row)
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

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

constexpr float kGrowth = 8.f;                    // log2 of how far a maximum may run ahead of its base
// A row's weights are 2^(z - base), rounded to the pool's type for the product with V (their sum is taken before that).  bf16
// has the exponents of 32 bits: a weight is off by 2^-8 of itself at most, however small.  fp16 ends at 2^16, has
// fewer bits below 2^-14 and none below 2^-25, which a long list of light tokens beside one heavy token can
// notice (131072 tokens 17 nats below it: 0.0078 instead of 0.0054).  So its base lies kLift below the maximum: the
// heaviest weight is at most 2^(kLift + kGrowth) = 2^15, and weights keep all bits down to 2^-21 of the base's, and lose at most
// 2^-32 of it each.
template <typename T> __device__ constexpr float kLift = 0.f;
template <> __device__ constexpr float kLift<__half> = 7.f;
constexpr long long kWaitCycles = 2000000000;   // a wait gives up after a second

__device__ __forceinline__ void mbar_init(uint64_t *b, int count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(uint64_t *b)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint64_t *b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint64_t *b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait.  A thread that gives up records it and waits for nothing any more: every role then runs
// through to the end of its list without touching memory for the results.
__device__ __forceinline__ void mbar_wait(uint64_t *b, uint32_t parity, bool &dead, unsigned long long *status)
{
    if (dead || mbar_try(b, parity)) return;
    const long long start = clock64();
    while (!mbar_try(b, parity))
        if (clock64() - start > kWaitCycles) {
            dead = true;
            atomicExch(status, 1ull);
            return;
        }
}

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap *map, int c0, int c1, int c2, int c3, int c4, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2,%3,%4,%5,%6}], [%7];" ::"r"(to),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(smem_u32(bar)) : "memory");
}

// 16 bytes to shared memory; with `there` false zeros are written and nothing is read.
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Values that are not finite.  A row that does not see a token gives it the weight 0, but 0 * infinity is NaN.  So the
// 16-byte pieces of V that hold such a value, among the tokens that some of an item's rows do not see, become zero before the product,
// and what they would have added is added to the rows that see them once their sums are complete.  (Tokens past the end of a sequence, which
// nobody sees, become zero as well.)
//
// Is one of eight 16-bit numbers infinite or NaN: an exponent of ones, which carries into the sign's place?
template <typename T> __device__ __forceinline__ bool any_not_finite(const uint4 &x);
template <> __device__ __forceinline__ bool any_not_finite<__nv_bfloat16>(const uint4 &x)
{
    auto carry = [](uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; };
    return ((carry(x.x) | carry(x.y) | carry(x.z) | carry(x.w)) & 0x80008000u) != 0;
}
template <> __device__ __forceinline__ bool any_not_finite<__half>(const uint4 &x)
{
    auto carry = [](uint32_t w) { return (w & 0x7c007c00u) + 0x04000400u; };
    return ((carry(x.x) | carry(x.y) | carry(x.z) | carry(x.w)) & 0x80008000u) != 0;
}
// What such pieces of own tokens [from, to) add to dims [d, d + 4) of a row: sum of 2^(z - base) v.  Rare, and slow: one
// thread, from the pool.
template <typename T>
__device__ __forceinline__ float4 left_out(const AttnParams &p, const T *q, int64_t tbl, int head, int from, int to, float base, int d)
{
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (base == -INFINITY) return sum;   // a row without weights
#pragma unroll 1
    for (int t = from; t < to; ++t) {
        const int block = t / p.pool.block_tokens;
        const char *row = p.pool.base + 2 * (int64_t)p.layer * p.pool.lc_stride + head * p.pool.head_stride +
                          p.tbl[tbl + block] * p.pool.block_stride + (int64_t)(t - block * p.pool.block_tokens) * p.pool.tok_stride;
        const T *k = reinterpret_cast<const T *>(row), *v = reinterpret_cast<const T *>(row + p.pool.lc_stride);
        if (!any_not_finite<T>(*reinterpret_cast<const uint4 *>(v + d / 8 * 8))) continue;
        float z = 0.f;
#pragma unroll 1
        for (int i = 0; i < p.D; ++i) z = fmaf(static_cast<float>(q[i]), static_cast<float>(k[i]), z);
        const float w = exp2f(fmaf(z, p.scale_log2, -base));
        sum.x = fmaf(w, static_cast<float>(v[d]), sum.x);
        sum.y = fmaf(w, static_cast<float>(v[d + 1]), sum.y);
        sum.z = fmaf(w, static_cast<float>(v[d + 2]), sum.z);
        sum.w = fmaf(w, static_cast<float>(v[d + 3]), sum.w);
    }
    return sum;
}

template <typename T> __device__ __forceinline__ float unpack(uint32_t low)
{
    const uint16_t bits = (uint16_t)low;
    return static_cast<float>(*reinterpret_cast<const T *>(&bits));
}

// 2^x, off by 2 units in the last place at most; 0 for -infinity.
__device__ __forceinline__ float pow2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

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

// The opt-in to more than 48 KB of shared memory is per kernel and device.
template <typename K> inline cudaError_t allow_shared(K kernel, int bytes, std::atomic<uint64_t> &devices)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (devices.load(std::memory_order_acquire) >> dev & 1)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) devices.fetch_or(1ull << dev, std::memory_order_release);
    return e;
}

}  // namespace pdkv
