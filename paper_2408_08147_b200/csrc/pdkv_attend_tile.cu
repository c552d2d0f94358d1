// Attention of many rows over one list of cached tokens -- the queries of all sequences behind a shared
// prefix, or a window of query tokens over its own sequence -- on the fifth-generation tensor cores.
//
// A CTA holds up to 256 rows (two tiles of 128) of one KV head and runs over tiles of 128 tokens:
//     S = Q K^T      tcgen05.mma, both operands in shared memory, S in tensor memory (128 columns a tile)
//     P = 2^(S - m)  one thread a row, rounded to 16 bits and written over S
//     O += P V       tcgen05.mma, P from tensor memory, O stays in tensor memory
// Two row tiles take turns: while the threads of one turn S into P, the tensor cores work for the
// other, and both use the same K and V, which halves what is read from L2.  When there is only one row tile, the
// two halves of the CTA take every second tile of tokens each, and leave two parts to be joined.  Twelve warps: four per row
// tile for the softmax, one that issues the matrix instructions, one that issues the loads (TMA boxes of one
// page, 64 dims and the 128-byte swizzle that the matrix instructions expect), two that only give up their registers.
//
// O is rescaled only when a row's maximum grew by more than 2^8 since the last time.  Bases and sums are 32 bits, the sums
// taken before the weights are rounded (see kLift).
//
// Bound by the tensor core and by the chain S, P, O of a row tile: 256 rows against 128 tokens of 128 dims take it
// 3024 cycles (125 for 16 dims of Q K^T, whose two operands come from shared memory at 64 bytes a cycle, 64 for 16 tokens
// of P V), and an iteration takes 3700.  Measured on B200, whole calls: 64 rows of each of 8 heads against 65536 tokens
// 70 us (3.8 TB/s), 256 rows 102 us (670 TFLOP/s), 512 rows against 200000 tokens 438 to 453 us (925 to 958 TFLOP/s).  (A row of S does not
// quite fit: ptxas spills 240 bytes a thread.)  Starting and finishing an
// item costs about 8 us, which is what short lists pay (256 rows against 4096 tokens: 26 us).
#include <algorithm>
#include <numeric>
#include <type_traits>

#include <cuda.h>

#include "pdkv_attend_device.cuh"

namespace pdkv {

namespace {

constexpr int kTileRows = 128, kTileTokens = 128;
constexpr int kSoftmaxThreads = 128;                          // of one row tile
constexpr int kMmaWarp = 8, kLoadWarp = 9, kTileThreads = 384;   // (warps 10 and 11 only give up their registers)

// Tensor memory columns: S (and P over it) of tile t, O of tile t.
constexpr uint32_t kColS = 0, kColO = 256, kColTile = 128, kColumns = 512;

template <int DP> struct TileShape {
    static constexpr int kSubs = DP / 64;                     // 64 dims: one swizzled row of 128 bytes
    static constexpr uint32_t kSub = 128 * 128;               // bytes of 128 such rows
    static constexpr uint32_t kOperand = kSubs * kSub;        // one tile of Q, K or V
    static constexpr int kSlots = DP == 64 ? 8 : 4;           // K and V tiles in flight, in turns
    static constexpr uint32_t kStage = 8 * 4096;              // a warp's way out: 32 rows of 32 dims
    static constexpr uint32_t kBytes = 2 * kOperand + kSlots * kOperand + kStage + 1024;
};

struct Barriers {
    uint64_t full[8], empty[8];     // ring of K and V tiles
    uint64_t q_ready[2];            // Q of a row tile is in shared memory
    uint64_t s_full[2];             // S of a row tile is complete
    uint64_t p_half[2], p_ready[2]; // P of a row tile is in tensor memory: its first 64 tokens, all of it
    uint64_t o_full[2];             // the last product of a row tile is complete
    uint32_t tmem;
};

__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tmem_load(float (&v)[32], uint32_t at)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_load16(float (&v)[16], uint32_t at)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Shared-memory operand in the 128-byte swizzle: 8-row groups 1024 bytes apart.  K-major (Q, K: a row is 64
// dims of one token): the leading offset is not used.  MN-major (V: a row is 64 dims, tokens run along
// the product): the leading offset leads to the next 64 dims.
__device__ __forceinline__ uint64_t operand(uint32_t smem, uint32_t leading)
{
    uint64_t d = (smem >> 4) & 0x3fff;
    d |= (uint64_t)((leading >> 4) & 0x3fff) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= 1ull << 46;   // descriptor version of sm_100
    d |= 2ull << 61;   // 128-byte swizzle
    return d;
}
// Instruction word: 32-bit accumulator, A and B of one 16-bit type, M = 128.
template <typename T> __device__ constexpr uint32_t instruction(int n, bool b_mn_major)
{
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return 1u << 4 | type << 7 | type << 10 | (b_mn_major ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (uint32_t)(128 / 16) << 24;
}
__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t word, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                 "r"(word), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t word, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b),
                 "r"(word), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void commit(uint64_t *b)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
// Barrier of `threads` threads; true for all of them where one has something.
__device__ __forceinline__ bool any_of(int barrier, int threads, bool mine)
{
    uint32_t any;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %3, 0;\n barrier.cta.red.or.pred q, %1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
                 : "=r"(any) : "r"(barrier), "r"(threads), "r"((uint32_t)mine) : "memory");
    return any != 0;
}
// (a call: the code is not there eight times)
template <typename T>
__device__ __noinline__ float4 left_out_call(const AttnParams &p, const T *q, int64_t tbl, int head, int from, int to, float base, int d)
{
    return left_out<T>(p, q, tbl, head, from, to, base, d);
}
// What every role has to know about an item.
struct Work {
    AttnItem it;
    int len, limit, tiles;   // tiles of tokens
    bool pair;               // two row tiles share the tokens; else the one row tile has every second tile of tokens
                             // in each half of the CTA, as two parts to be joined
    // Tiles of tokens of half t, and which they are.
    __device__ __forceinline__ int count(int t) const { return pair ? tiles : (tiles + 1 - t) / 2; }
    __device__ __forceinline__ int tile(int t, int j) const { return pair ? j : 2 * j + t; }
    // Place of K (kv 0) or V (1) of token tile i in the order of the loads: K, V alternating, or K K V V.
    __device__ __forceinline__ uint32_t order(int kv, int i) const
    {
        return pair ? 2 * i + kv : i / 2 * 4 + kv * ((i | 1) < tiles ? 2 : 1) + i % 2;
    }
};
template <int FORM> __device__ __forceinline__ Work work_of(const AttnParams &p, const AttnItem &it)
{
    Work w;
    w.it = it;
    w.len = it.seq >= 0 ? own_len(p, it.seq, it.len) : it.len;
    w.limit = min(it.tok1, w.len);
    if (FORM && nobody_there(p, it)) w.limit = min(w.limit, it.tok0);
    w.tiles = w.limit > it.tok0 ? (w.limit - it.tok0 + kTileTokens - 1) / kTileTokens : 0;
    w.pair = it.rows > kTileRows;
    return w;
}

// Q of a row tile: a warp brings its 32 rows, DP / 8 neighbouring lanes a row, 16 bytes each.  Place of the
// lane's k-th piece in shared memory, in the swizzle that the matrix instructions read.
template <int DP> __device__ __forceinline__ uint32_t q_place(int t, int k)
{
    constexpr int kLanes = DP / 8, kRows = 32 / kLanes;
    const int lane = threadIdx.x % 32, row = threadIdx.x / 32 % 4 * 32 + k * kRows + lane / kLanes, c = lane % kLanes;
    return (uint32_t)t * TileShape<DP>::kOperand + c / 8 * TileShape<DP>::kSub + row * 128 + ((c % 8) ^ (row % 8)) * 16;
}
template <typename T, int DP> __device__ __forceinline__ void fetch_q(const AttnParams &p, const Work &w, int t, uint32_t q_at)
{
    constexpr int kLanes = DP / 8, kRows = 32 / kLanes;
    const int lane = threadIdx.x % 32, mine = (w.pair ? t * kTileRows : 0) + threadIdx.x % kSoftmaxThreads, d = 8 * (lane % kLanes);
    const bool live = mine < w.it.rows;
    const RowId id = row_id(p, w.it, w.it.row0 + (live ? mine : 0));
    const int64_t at = live ? id.seq * p.q_stride[0] + id.token * p.q_stride[1] + (w.it.head * p.G + id.g) * p.q_stride[2] : -1;
#pragma unroll 4
    for (int k = 0; k < 32 / kRows; ++k) {
        const int64_t from = __shfl_sync(~0u, at, k * kRows + lane / kLanes);
        const bool there = from >= 0 && d < p.D;   // else zeros
        copy_async(q_at + q_place<DP>(t, k), static_cast<const T *>(p.q) + (there ? from + d : 0), there);
    }
}

}  // namespace

// FORM: another form than plain causal.  A thread turns the logits of its row into what the form says (capped, biased, hidden by the
// row's mask) while they are in registers.  What that takes is added to the chain S, P, O, which bounds an iteration: 8 sequences of 8192 tokens,
// 256 rows of each of 8 heads take 98 us plain, 104 with masks, 158 capped by 30 (few tiles have a far logit; by 2, where all have, 202), 128 biased, 177
// capped by 30 and biased.
template <typename T, int DP, int FORM>
__global__ void __launch_bounds__(kTileThreads, 1) attend_tile_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnParams p)
{
    using G = TileShape<DP>;
    extern __shared__ char raw[];
    __shared__ Barriers bar;
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(raw) + 1023) / 1024 * 1024);
    const uint32_t q_at = smem_u32(smem), ring_at = q_at + 2 * G::kOperand;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const AttnItem first = fetch_item(p.tile_items, blockIdx.x);
    if (threadIdx.x == 0) {
        for (int i = 0; i < G::kSlots; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.empty[i], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&bar.q_ready[t], kSoftmaxThreads / 32);   // a warp arrives once: arrivals of single threads queue up
            mbar_init(&bar.s_full[t], 1);
            mbar_init(&bar.p_half[t], kSoftmaxThreads / 32);
            mbar_init(&bar.p_ready[t], kSoftmaxThreads / 32);
            mbar_init(&bar.o_full[t], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (warp == kLoadWarp && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");   // set up while the work before this call ends
    asm volatile("griddepcontrol.launch_dependents;");
    bool dead = false;
    // tensor memory is there for the warps that use it; the loads of K and V do not wait for it
    auto tensor_memory = [&]() -> uint32_t {
        fence_before();
        asm volatile("bar.sync 1, 288;" ::: "memory");
        fence_after();
        return bar.tmem;
    };

    // 168 registers a thread at launch: the softmax threads, which hold a row of S, take 216, the others keep 72
    // (256 x 216 + 128 x 72 = 384 x 168).
    if (warp >= kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kLoadWarp) {
        // K(0), V(0), K(1), V(1) ... into the ring; a lane loads a box of tokens within one block
        const int page_rows = p.tile_box;
        uint32_t n = 0;
        AttnItem it = first;
        for (bool more = true; more;) {
            const AttnItem next_it = fetch_item(p.tile_items, max(it.next, 0));
            more = it.next >= 0;
            const Work w = work_of<FORM>(p, it);
            it = next_it;
            const int group = w.pair ? 1 : 2;   // tiles of tokens whose K come before their V
            for (int i0 = 0; i0 < w.tiles; i0 += group) {
                int block[2] = {0, 0}, tt[2] = {0, 0}, boxes[2] = {0, 0};
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int t0 = w.it.tok0 + (i0 + g) * kTileTokens;
                    if (g >= group || t0 >= w.limit) continue;
                    boxes[g] = (min(kTileTokens, w.limit - t0) + page_rows - 1) / page_rows;   // pages past the end are not loaded
                    if (lane < boxes[g]) {
                        const int t = t0 + lane * page_rows;
                        block[g] = p.tbl[w.it.tbl + t / p.pool.block_tokens];
                        tt[g] = t % p.pool.block_tokens;
                    }
                }
                for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        if (boxes[g] == 0) continue;
                        const int slot = n % G::kSlots;
                        mbar_wait(&bar.empty[slot], (n / G::kSlots & 1) ^ 1, dead, p.status);
                        ++n;
                        dead = __any_sync(~0u, dead);
                        if (dead) continue;
                        if (lane == 0) mbar_expect(&bar.full[slot], (uint32_t)boxes[g] * page_rows * 128 * G::kSubs);
                        __syncwarp();
                        if (lane < boxes[g]) {
                            const uint32_t to = ring_at + slot * G::kOperand + lane * page_rows * 128;
                            const int lc = 2 * p.layer + kv;
#pragma unroll
                            for (int s = 0; s < G::kSubs; ++s) {
                                if (p.map_layer_major)
                                    load_box(to + s * G::kSub, &map, 64 * s, tt[g], w.it.head, block[g], lc, &bar.full[slot]);
                                else
                                    load_box(to + s * G::kSub, &map, 64 * s, w.it.head, tt[g], lc, block[g], &bar.full[slot]);
                            }
                        }
                    }
            }
        }
    } else if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)), "r"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        const uint32_t tmem = tensor_memory();
        if (lane == 0) {
            constexpr uint32_t kWordS = instruction<T>(kTileTokens, false), kWordO = instruction<T>(DP, true);
            uint32_t n = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
            auto product_s = [&](int t, uint32_t k_slot) {   // S(t) = Q(t) K^T
                const uint32_t q = q_at + t * G::kOperand, k = ring_at + k_slot * G::kOperand;
#pragma unroll
                for (int s = 0; s < DP / 16; ++s) {
                    const uint32_t o = s / 4 * G::kSub + s % 4 * 32;
                    mma_shared(tmem + kColS + t * kColTile, operand(q + o, 16), operand(k + o, 16), kWordS, s > 0);
                }
            };
            auto product_o = [&](int t, uint32_t v_slot, int half, bool add) {   // O(t) += P(t) V, 64 tokens
                const uint32_t v = ring_at + v_slot * G::kOperand;
#pragma unroll
                for (int k = 0; k < kTileTokens / 32; ++k) {
                    const int s = half * (kTileTokens / 32) + k;
                    mma_tensor(tmem + kColO + t * kColTile, tmem + kColS + t * kColTile + 8 * s, operand(v + s * 2048, G::kSub), kWordO, add || k > 0);
                }
            };
            AttnItem it = first;
            for (bool more = true; more;) {
                const AttnItem next_it = fetch_item(p.tile_items, max(it.next, 0));
                more = it.next >= 0;
                const Work w = work_of<FORM>(p, it);
                it = next_it;
                if (w.tiles == 0) continue;
                // the operand at place `at` of the load order has arrived, is no longer needed
                auto arrived = [&](uint32_t at) {
                    const uint32_t slot = (n + at) % G::kSlots;
                    mbar_wait(&bar.full[slot], (n + at) / G::kSlots & 1, dead, p.status);
                    fence_after();
                    return slot;
                };
                for (int t = 0; t < 2; ++t) {
                    if (w.count(t) == 0) continue;
                    mbar_wait(&bar.q_ready[t], q_phase[t], dead, p.status);
                    q_phase[t] ^= 1;
                    const uint32_t k = arrived(w.order(0, w.tile(t, 0)));
                    if (!dead) product_s(t, k);
                    commit(&bar.s_full[t]);
                    if (!w.pair || t == 1) commit(&bar.empty[k]);
                }
                for (int j = 0; j < w.count(0); ++j) {
                    for (int t = 0; t < 2; ++t) {
                        if (j >= w.count(t)) continue;
                        const bool last = j + 1 == w.count(t), release = !w.pair || t == 1;
                        mbar_wait(&bar.p_half[t], p_phase[t], dead, p.status);
                        const uint32_t v = arrived(w.order(1, w.tile(t, j)));
                        if (!dead) product_o(t, v, 0, j > 0);
                        mbar_wait(&bar.p_ready[t], p_phase[t], dead, p.status);
                        p_phase[t] ^= 1;
                        fence_after();
                        if (!dead) product_o(t, v, 1, true);
                        if (release) commit(&bar.empty[v]);
                        if (last) {
                            commit(&bar.o_full[t]);
                        } else {
                            const uint32_t k = arrived(w.order(0, w.tile(t, j + 1)));
                            if (!dead) product_s(t, k);
                            commit(&bar.s_full[t]);
                            if (release) commit(&bar.empty[k]);
                        }
                    }
                }
                n += 2 * w.tiles;
            }
        }
        __syncwarp();
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        bool q_early = false;   // the first item's Q comes while tensor memory is set up
        {
            const Work w = work_of<FORM>(p, first);
            q_early = w.count(warp / 4) > 0;
            if (q_early) fetch_q<T, DP>(p, w, warp / 4, q_at);
        }
        const uint32_t tmem = tensor_memory();
        // softmax of row tile t: one thread a row
        const int t = warp / 4, r = threadIdx.x % kSoftmaxThreads;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + lanes + kColS + t * kColTile, o_at = tmem + lanes + kColO + t * kColTile;
        // what a row's numbers are multiplied by on their way into the exponential (capped and biased ones are in base 2 already)
        const float scale = FORM >= kCapped ? 1.f : fabsf(p.scale_log2);
        const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;   // a negative scale: the signs of Q are turned
        uint32_t s_phase = 0, o_phase = 0, n = 0;
        bool q_there = q_early, q_done = false;   // the item's Q is on its way, has been handed over
        // A warp's 32 rows of 32 numbers leave by way of shared memory: a lane has a row, but eight neighbouring lanes
        // store 128 bytes of one row (lanes storing their own rows touched 32 sectors an instruction: 8000 cycles
        // for a tile of O).  f(row of the warp, number of the first of four columns, the four numbers).
        char *stage = smem + (2 + G::kSlots) * G::kOperand + warp * 4096;
        auto by_rows = [&](const float *v, auto &&f) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                *reinterpret_cast<float4 *>(stage + lane * 128 + ((k ^ (lane % 8)) * 16)) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r4 = 4 * k + lane / 8;
                f(r4, 4 * (lane % 8), *reinterpret_cast<const float4 *>(stage + r4 * 128 + (((lane % 8) ^ (r4 % 8)) * 16)));
            }
            __syncwarp();
        };
        auto finish_q = [&]() {
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (flip) {   // (a lane turns the signs of what it brought itself)
#pragma unroll 1
                for (int k = 0; k < DP / 8; ++k) {
                    uint4 *x = reinterpret_cast<uint4 *>(smem + q_place<DP>(t, k));
                    *x = make_uint4(x->x ^ flip, x->y ^ flip, x->z ^ flip, x->w ^ flip);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.q_ready[t]);
        };
        AttnItem it = first;
        for (bool more = true; more;) {
            const AttnItem next_it = fetch_item(p.tile_items, max(it.next, 0));
            more = it.next >= 0;
            const Work w = work_of<FORM>(p, it);
            it = next_it;
            const uint32_t n0 = n;
            n += 2 * w.tiles;
            const int count = w.count(t), row = (w.pair ? t * kTileRows : 0) + r;
            const bool live = row < w.it.rows, own = w.it.seq >= 0;
            const RowId id = row_id(p, w.it, w.it.row0 + (live ? row : 0));
            float m = -INFINITY, l = 0.f;
            const int n_new = FORM ? newest_of(p, id.seq) : 0;
            const int sees = FORM ? w.limit : own ? min(w.limit, w.len - (p.q_tokens - 1 - id.token)) : w.limit;   // tokens before this one
            const int safe = own ? min(w.limit, FORM ? w.len - n_new : w.len - (p.q_tokens - 1)) : w.limit;        // the same of every row
            const bool there = id.token < n_new;   // FORM: one of the newest
            Bias bias{0.f, 0};
            if (FORM == kSloped) bias = bias_of(p, w.it, id, own ? w.len : own_len(p, id.seq, p.segs[id.seq].len));
            bool wild = false;   // pieces of V were left out
            if (count > 0) {
                if (!q_there) fetch_q<T, DP>(p, w, t, q_at);
                if (!q_there || !q_done) finish_q();
                q_there = q_done = false;
                for (int j = 0; j < count; ++j) {
                    const int t0 = w.it.tok0 + w.tile(t, j) * kTileTokens;
                    const bool masked = t0 + kTileTokens > safe;
                    mbar_wait(&bar.s_full[t], s_phase, dead, p.status);
                    s_phase ^= 1;
                    __syncwarp();
                    fence_after();
                    float v[kTileTokens];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_load(*reinterpret_cast<float(*)[32]>(v + 32 * c), s_at + 32 * c);
                    tmem_load_wait();
                    if constexpr (FORM >= kCapped) {
                        if (FORM == kCapped || p.cap_out != 0.f) {
                            float most = 0.f;
#pragma unroll
                            for (int k = 0; k < kTileTokens; k += 2) most = max3(most, fabsf(v[k]), fabsf(v[k + 1]));
                            // All near: a shorter way to the same bits, so it may be chosen by whatever lies in the tile.  (Two special functions a logit take 2048
                            // cycles a tile of 128 rows, half of the other work.)
                            if (p.cap_unit == 1.f && __all_sync(~0u, !there || __fmul_rn(most, p.cap_in) <= kCapNear)) {
#pragma unroll
                                for (int k = 0; k < kTileTokens; k += 2) {
                                    const float2 z = make_float2(v[k], v[k + 1]), x = capped_near(p, z, mul2(z, z));
                                    v[k] = x.x;
                                    v[k + 1] = x.y;
                                }
                            } else {
#pragma unroll
                                for (int k = 0; k < kTileTokens; k += 2) {
                                    const float2 x = capped(p, make_float2(v[k], v[k + 1]));
                                    v[k] = x.x;
                                    v[k + 1] = x.y;
                                }
                            }
                        }
                    }
                    if constexpr (FORM == kSloped) {
                        // slope * (t0 + k - query): steps of sixteen tokens, and within them
                        const float in = p.cap_out != 0.f ? 1.f : fabsf(p.scale_log2), far = bias.slope * (float)(t0 - bias.query);
                        const float2 in2 = make_float2(in, in);
                        float2 step[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) step[k] = make_float2(bias.slope * (2 * k), bias.slope * (2 * k + 1));
#pragma unroll
                        for (int c = 0; c < kTileTokens; c += 16) {
                            const float at = fmaf(bias.slope, (float)c, far);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float2 x = fma2(make_float2(v[c + 2 * k], v[c + 2 * k + 1]), in2, add2(step[k], make_float2(at, at)));
                                v[c + 2 * k] = x.x;
                                v[c + 2 * k + 1] = x.y;
                            }
                        }
                    }
                    if (FORM && !there) {
#pragma unroll
                        for (int k = 0; k < kTileTokens; ++k) v[k] = -INFINITY;
                    }
                    if (FORM && masked) {
                        const int from = t0 - (w.len - n_new);   // number of tile's first token among the newest
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t seen = own ? newest_seen(p, id.seq, id.token, n_new, from + 32 * c) : ~0u;
                            const int left = w.limit - (t0 + 32 * c);
                            if (left < 32) seen &= left <= 0 ? 0u : (1u << left) - 1;
                            if (FORM == kSloped && own && p.offset && seen != 0) {   // the place of a newest token is not its slot
#pragma unroll
                                for (int k = 0; k < 32; ++k) {
                                    const int j = from + 32 * c + k;
                                    if (j >= 0 && (seen >> k & 1)) v[32 * c + k] = fmaf(bias.slope, (float)(offset_of(p, id.seq, j) - j), v[32 * c + k]);
                                }
                            }
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!(seen >> k & 1)) v[32 * c + k] = -INFINITY;
                        }
                    } else if (masked) {
#pragma unroll
                        for (int k = 0; k < kTileTokens; ++k)
                            if (t0 + k >= sees) v[k] = -INFINITY;
                    }
                    float tops[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) tops[k] = fmaxf(v[2 * k], v[2 * k + 1]);
#pragma unroll
                    for (int k = 8; k < kTileTokens / 2; ++k) tops[k % 8] = max3(tops[k % 8], v[2 * k], v[2 * k + 1]);
                    float top = max3(max3(max3(tops[0], tops[1], tops[2]), tops[3], tops[4]), tops[5], fmaxf(tops[6], tops[7]));
                    top = top == -INFINITY ? top : fmaf(top, scale, -kLift<T>);
                    const bool grew = top > m + kGrowth || (m == -INFINITY && top > m);
                    if (__any_sync(~0u, grew)) {
                        // (FORM: the row's own maximum alone decides on its base, so that its neighbours change no bit of it)
                        const float new_m = !FORM || grew ? fmaxf(m, top) : m, f = new_m == -INFINITY ? 1.f : pow2(m - new_m);
                        l *= f;
                        m = new_m;
                        if (j > 0) {
#pragma unroll 1
                            for (int c = 0; c < DP / 16; ++c) {
                                float x[16];
                                tmem_load16(x, o_at + 16 * c);
                                tmem_load_wait();
#pragma unroll
                                for (int k = 0; k < 16; ++k) x[k] *= f;
                                tmem_store16(o_at + 16 * c, reinterpret_cast<uint32_t(&)[16]>(x));
                            }
                            tmem_store_wait();
                        }
                    }
                    const float base = m == -INFINITY ? 0.f : m;
                    __syncwarp();
                    float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    const float2 scale2 = make_float2(scale, scale), base2 = make_float2(-base, -base);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t packed[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const int i0 = 32 * c + 2 * k;
                            float2 x = fma2(make_float2(v[i0], v[i0 + 1]), scale2, base2);
                            x.x = pow2(x.x);
                            x.y = pow2(x.y);
                            sums[k % 2] = add2(sums[k % 2], x);
                            packed[k] = pack<T>(x.x, x.y);
                        }
                        tmem_store16(s_at + 16 * c, packed);
                        if (c == 1) {
                            if (masked && (t == 0 || !w.pair)) {
                                // rows of V past the end may hold anything; and see left_out
                                const uint32_t x = n0 + w.order(1, w.tile(t, j));
                                mbar_wait(&bar.full[x % G::kSlots], x / G::kSlots & 1, dead, p.status);
                                if (t0 + r >= safe) {
                                    const bool past = t0 + r >= w.limit;
                                    char *row = smem + 2 * G::kOperand + x % G::kSlots * G::kOperand + r * 128;
#pragma unroll 2
                                    for (int i = 0; i < 8 * G::kSubs; ++i) {
                                        uint4 *at = reinterpret_cast<uint4 *>(row + i / 8 * G::kSub + (i + r) % 8 * 16);
                                        if (past || any_not_finite<T>(*at)) {
                                            *at = make_uint4(0, 0, 0, 0);
                                            wild = wild || !past;
                                        }
                                    }
                                }
                                fence_async_smem();
                            }
                            tmem_store_wait();
                            fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&bar.p_half[t]);
                        }
                    }
                    l += sums[0].x + sums[0].y + (sums[1].x + sums[1].y);
                    tmem_store_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar.p_ready[t]);
                }
                // (one row tile: the halves have tiles of tokens, and barriers, of their own)
                if (safe < w.limit) wild = any_of(w.pair ? 2 : 3 + t, w.pair ? 2 * kSoftmaxThreads : kSoftmaxThreads, wild);
                // every product with Q is done: the next item's Q may take its place
                if (more) {
                    const Work next = work_of<FORM>(p, next_it);
                    if (next.count(t) > 0) {
                        fetch_q<T, DP>(p, next, t, q_at);
                        finish_q();
                        q_there = q_done = true;
                    }
                }
                mbar_wait(&bar.o_full[t], o_phase, dead, p.status);
                o_phase ^= 1;
                __syncwarp();
                fence_after();
            }
            const int head = w.it.head * p.G + id.g;
            const int64_t part_row = w.it.part_row + (!w.pair && t == 1 ? w.it.rows : 0);
            const float inv = l == 0.f ? 0.f : 1.f / l;
            // (parts of query tokens that are not there are not read)
            const int64_t to = !live || dead || (FORM && !there && !w.it.direct) ? -1
                               : w.it.direct ? id.seq * p.out_stride[0] + id.token * p.out_stride[1] + head * p.out_stride[2]
                                             : (part_row + row) * p.D;
            // (loops that run once an item stay rolled: fetching their instructions costs more than running them)
#pragma unroll 1
            for (int c = 0; c < DP / 32; ++c) {
                float v[32];
                __syncwarp();
                if (count > 0) {
                    tmem_load(v, o_at + 32 * c);
                    tmem_load_wait();
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = 0.f;
                }
                if (FORM && l == 0.f) {   // a row that saw nothing: its products may be 0 * infinity
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = 0.f;
                }
                if (wild && live) {
                    const T *q = static_cast<const T *>(p.q) + id.seq * p.q_stride[0] + id.token * p.q_stride[1] + head * p.q_stride[2];
#pragma unroll 1
                    for (int j = 0; j < count; ++j) {
                        const int t0 = w.it.tok0 + w.tile(t, j) * kTileTokens, from = max(t0, safe), to = min(t0 + kTileTokens, sees);
                        if (from < to)
#pragma unroll
                            for (int k = 0; k < 32; k += 4)
                                if (32 * c + k < p.D) {
                                    float4 y;
                                    if constexpr (FORM)
                                        y = left_out_formed<T>(p, q, w.it, id, w.len, from, to, m, 32 * c + k);
                                    else
                                        y = left_out_call<T>(p, q, w.it.tbl, w.it.head, from, to, m, 32 * c + k);
                                    v[k] += y.x;
                                    v[k + 1] += y.y;
                                    v[k + 2] += y.z;
                                    v[k + 3] += y.w;
                                }
                    }
                }
                const float f = w.it.direct ? inv : 1.f;
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] *= f;
                by_rows(v, [&](int r4, int col, float4 x) {
                    const int64_t at = __shfl_sync(~0u, to, r4);
                    const int d = 32 * c + col;
                    if (at >= 0 && d < p.D) {
                        if (w.it.direct)
                            *reinterpret_cast<uint2 *>(static_cast<T *>(p.out) + at + d) = make_uint2(pack<T>(x.x, x.y), pack<T>(x.z, x.w));
                        else
                            *reinterpret_cast<float4 *>(p.part_o + at + d) = x;
                    }
                });
            }
            if (live && !dead) {
                if (w.it.direct && p.lse) p.lse[((int64_t)id.seq * p.q_tokens + id.token) * p.G * p.H + head] = (m + log2f(l)) * kLn2;
                if (!w.it.direct || p.with_scores) *reinterpret_cast<float2 *>(p.part_ml + 2 * (part_row + row)) = make_float2(m, l);
            }
        }
    }
    fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(bar.tmem), "r"(kColumns));
    }
}

namespace {

// Shared memory of the weighing kernel: the rows of Q, up to 256, and two tiles of K.
__host__ __device__ constexpr uint32_t weigh_q_sub(int rows) { return (uint32_t)((rows < 256 ? rows + 15 : 256) / 16 * 16) * 128; }   // 64 dims
template <int DP> constexpr uint32_t weigh_bytes(int rows)
{
    return TileShape<DP>::kSubs * weigh_q_sub(rows) + 2 * TileShape<DP>::kOperand + 1024;
}

}  // namespace

// Attention weights of own tokens, summed over the rows of their sequence, for segments that the tile kernel
// attends to: a second pass over K once every row's sum is known.  (Writing the logits and reading them back, as
// is done for few rows, moves 8 bytes a row and token, against 2 bytes a dim for K.)
//
// S^T = K Q^T: a thread has one token and its logits of all rows in tensor memory, so the sum over the
// rows needs no other thread.  Six warps: four compute weights, one issues the products, one the loads of K;
// two tiles of K and two of S^T are on their way.  Two CTAs on an SM up to 128 rows.  12 sequences of 300 to 4096
// tokens, 64 rows each, 8 heads of 128 dims take 27 us as a kernel alone (cold), of which the bytes of K need 9 and the exponentials 3 (16
// a cycle and SM); the tensor pipe is active for 8%, DRAM for 25%.  So latency bounds it: a CTA starts (Q, sums of the rows) for a
// handful of tiles, and ragged lists leave a few CTAs for a second wave.
//
// FORM: logits one by one; a token's bit in the mask, and its place, are looked up for each row, and the row of logits lies in local memory
// (indexed at run time).  Slow: attention with weights of 16 sequences of 2048 tokens, 256 rows of 8 heads, takes 884 us with a tree's mask and
// 121 plain causal, of which 52 and 51 are the attention.
template <typename T, int DP, bool FORM>
__global__ void __launch_bounds__(192) attend_weigh_kernel(const __grid_constant__ CUtensorMap map, const AttnParams p, const int chunks, const int chunk_tiles)
{
    using G = TileShape<DP>;
    extern __shared__ char raw[];
    __shared__ uint64_t k_full[2], k_empty[2], s_full[2], s_empty[2], q_full;
    __shared__ uint32_t tmem_s;
    __shared__ __align__(16) float lse[256];   // negated, base 2
    __shared__ __align__(16) int sees[256];
    __shared__ Bias bias[FORM ? 256 : 1];
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(raw) + 1023) / 1024 * 1024);
    const int R = p.G * p.q_tokens, columns = R > 128 ? 256 : R > 64 ? 128 : 64;   // of one S^T
    const uint32_t q_sub = weigh_q_sub(R), q_at = smem_u32(smem), k_at = q_at + G::kSubs * q_sub;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int chunk = blockIdx.x % chunks, head = blockIdx.x / chunks % p.H, seq = blockIdx.x / chunks / p.H;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], 4);
        }
        mbar_init(&q_full, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(2 * columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    const AttnSeg seg = p.segs[seq];
    asm volatile("griddepcontrol.wait;" ::: "memory");   // sums of the rows, current lengths
    asm volatile("griddepcontrol.launch_dependents;");
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_s;
    const int len = own_len(p, seq, seg.len), begin = chunk * chunk_tiles * kTileTokens;
    const int limit = min(len, begin + chunk_tiles * kTileTokens);
    const int tiles = limit > begin ? (limit - begin + kTileTokens - 1) / kTileTokens : 0;
    bool dead = false;
    uint32_t n = 0;   // tiles so far, over all groups of 256 rows
    if (warp == 5) {
        for (int r0 = 0; r0 < R; r0 += 256)
            for (int j = 0; j < tiles; ++j, ++n) {
                const int t0 = begin + j * kTileTokens, boxes = (min(kTileTokens, limit - t0) + p.tile_box - 1) / p.tile_box, slot = n & 1;
                int block = 0, tt = 0;
                if (lane < boxes) {
                    const int t = t0 + lane * p.tile_box;
                    block = p.tbl[seg.tbl + t / p.pool.block_tokens];
                    tt = t % p.pool.block_tokens;
                }
                mbar_wait(&k_empty[slot], (n >> 1 & 1) ^ 1, dead, p.status);
                dead = __any_sync(~0u, dead);
                if (dead) continue;
                if (lane == 0) mbar_expect(&k_full[slot], (uint32_t)boxes * p.tile_box * 128 * G::kSubs);
                __syncwarp();
                if (lane < boxes) {
#pragma unroll
                    for (int i = 0; i < G::kSubs; ++i) {
                        const uint32_t to = k_at + slot * G::kOperand + i * G::kSub + lane * p.tile_box * 128;
                        if (p.map_layer_major)
                            load_box(to, &map, 64 * i, tt, head, block, 2 * p.layer, &k_full[slot]);
                        else
                            load_box(to, &map, 64 * i, head, tt, 2 * p.layer, block, &k_full[slot]);
                    }
                }
            }
    } else if (warp == 4) {
        if (lane == 0) {
            uint32_t q_phase = 0;
            for (int r0 = 0; r0 < R && tiles > 0; r0 += 256) {
                const uint32_t word = instruction<T>((min(256, R - r0) + 15) / 16 * 16, false);
                mbar_wait(&q_full, q_phase, dead, p.status);
                q_phase ^= 1;
                for (int j = 0; j < tiles; ++j, ++n) {
                    const int b = n & 1;
                    mbar_wait(&k_full[b], n >> 1 & 1, dead, p.status);
                    mbar_wait(&s_empty[b], (n >> 1 & 1) ^ 1, dead, p.status);
                    fence_after();
                    const uint32_t k = k_at + b * G::kOperand;
                    if (!dead) {
#pragma unroll
                        for (int i = 0; i < DP / 16; ++i)
                            mma_shared(tmem + b * columns, operand(k + i / 4 * G::kSub + i % 4 * 32, 16), operand(q_at + i / 4 * q_sub + i % 4 * 32, 16), word, i > 0);
                    }
                    commit(&k_empty[b]);
                    commit(&s_full[b]);
                }
            }
        }
        __syncwarp();
    } else {
        const float scale = fabsf(p.scale_log2);
        const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
        const int64_t out_row = seq * p.scores_out_stride[0] + head * p.scores_out_stride[1];
        const int64_t in_row = seq * p.scores_in_stride[0] + head * p.scores_in_stride[1];
        for (int r0 = 0; r0 < R && tiles > 0; r0 += 256) {
            const int rows = min(256, R - r0), width = (rows + 15) / 16 * 16;
            // Q: DP / 8 neighbouring lanes a row, rows up to a multiple of 16 filled with zeros.  (Every product with the
            // rows before has been waited for.)
            constexpr int kLanes = DP / 8, kRows = 128 / kLanes;
            const int c = threadIdx.x % kLanes;
#pragma unroll 4
            for (int i = threadIdx.x / kLanes; i < width; i += kRows) {
                const int row = r0 + i;
                const bool there = i < rows && 8 * c < p.D;
                const int64_t from = there ? seq * p.q_stride[0] + row / p.G * p.q_stride[1] + (head * p.G + row % p.G) * p.q_stride[2] + 8 * c : 0;
                copy_async(q_at + c / 8 * q_sub + i * 128 + ((c % 8) ^ (i % 8)) * 16, static_cast<const T *>(p.q) + from, there);
            }
            for (int i = threadIdx.x; i < columns; i += 128) {
                const int row = r0 + min(i, rows - 1);
                const float x = p.lse[((int64_t)seq * p.q_tokens + row / p.G) * p.G * p.H + head * p.G + row % p.G];
                lse[i] = i >= rows || x == -INFINITY ? -INFINITY : -x * kLog2e;   // no weight: 2^(z - inf) = 0
                sees[i] = len - (p.q_tokens - 1 - row / p.G);
                if constexpr (FORM) {
                    AttnItem it{};
                    it.seq = seq;
                    it.head = head;
                    bias[i] = bias_of(p, it, {seq, row / p.G, row % p.G}, len);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (flip)   // (a thread turns the signs of what it brought itself)
                for (int i = threadIdx.x / kLanes; i < width; i += kRows) {
                    uint4 *x = reinterpret_cast<uint4 *>(smem + c / 8 * q_sub + i * 128 + ((c % 8) ^ (i % 8)) * 16);
                    *x = make_uint4(x->x ^ flip, x->y ^ flip, x->z ^ flip, x->w ^ flip);
                }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full);
            asm volatile("bar.sync 1, 128;" ::: "memory");   // lse, sees
            for (int j = 0; j < tiles; ++j, ++n) {
                const int b = n & 1, t0 = begin + j * kTileTokens, t = t0 + threadIdx.x;
                mbar_wait(&s_full[b], n >> 1 & 1, dead, p.status);
                __syncwarp();
                fence_after();
                const bool masked = t0 + kTileTokens > len - (p.q_tokens - 1);
                float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                const float2 scale2 = make_float2(scale, scale);
#pragma unroll 1
                for (int col = 0; col < width; col += 32) {
                    float v[32];
                    tmem_load(v, tmem + ((uint32_t)(warp * 32) << 16) + b * columns + col);
                    tmem_load_wait();
                    if constexpr (FORM) {
                        const int n_new = newest_of(p, seq), j = t - (len - n_new);
#pragma unroll 4
                        for (int k = 0; k < 32; ++k) {
                            if (col + k >= rows) break;
                            const int token = (r0 + col + k) / p.G;
                            const Bias b = bias[col + k];
                            // (tokens before the newest: seen by every query token that is there)
                            const bool seen = token < n_new && (j < 0 || (newest_seen(p, seq, token, n_new, j) & 1)) && lse[col + k] != -INFINITY;
                            float x = v[k] * fabsf(p.scale_log2);
                            if (seen && p.cap_out != 0.f) x = capped(p, v[k]);
                            if (p.slopes) x = fmaf(b.slope, (float)((j >= 0 && j < n_new ? len - n_new + offset_of(p, seq, j) : t) - b.query), x);
                            if (seen) sums[0].x += pow2(x + lse[col + k]);
                        }
                        continue;
                    }
                    if (masked || col + 32 > rows) {
                        // Columns past the last row hold anything, or products of zeros, NaN for an infinite K; a token that a row
                        // does not see weighs nothing even where the row's sum is NaN.
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            const float x = pow2(fmaf(v[k], scale, lse[col + k]));
                            if (k % 2)
                                sums[0].y += col + k >= rows || t >= sees[col + k] ? 0.f : x;
                            else
                                sums[0].x += col + k >= rows || t >= sees[col + k] ? 0.f : x;
                        }
                        continue;
                    }
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        const float4 e = *reinterpret_cast<const float4 *>(lse + col + k);
                        float2 x = fma2(make_float2(v[k], v[k + 1]), scale2, make_float2(e.x, e.y));
                        float2 y = fma2(make_float2(v[k + 2], v[k + 3]), scale2, make_float2(e.z, e.w));
                        sums[0] = add2(sums[0], make_float2(pow2(x.x), pow2(x.y)));
                        sums[1] = add2(sums[1], make_float2(pow2(y.x), pow2(y.y)));
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&s_empty[b]);
                if (t < limit && !dead) {
                    const float add = (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
                    const float in = r0 > 0 ? p.scores_out[out_row + t] : p.scores_in ? p.scores_in[in_row + t] : 0.f;
                    p.scores_out[out_row + t] = in + add;
                }
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");   // the next rows' lse, sees and Q take the place of these
        }
        // tokens past the sequence's end have no weight: the row is carried over where it is not in place
        if (p.scores_in != p.scores_out)
            for (int t = max(begin, len) + threadIdx.x; t < min(begin + chunk_tiles * kTileTokens, p.max_len); t += 128)
                p.scores_out[out_row + t] = p.scores_in ? p.scores_in[in_row + t] : 0.f;
    }
    fence_before();
    __syncthreads();
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * columns));
    }
}

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

template <typename T, int DP, int FORM> cudaError_t launch_dims(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(attend_tile_kernel<T, DP, FORM>, (int)TileShape<DP>::kBytes, ready);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.n_tile_ctas);
    cfg.blockDim = dim3(kTileThreads);
    cfg.dynamicSmemBytes = TileShape<DP>::kBytes;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_tile_kernel<T, DP, FORM>, map, p);
}

template <typename T, int DP, bool FORM> cudaError_t launch_weigh(const AttnParams &p, const CUtensorMap &map, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(attend_weigh_kernel<T, DP, FORM>, (int)weigh_bytes<DP>(256), ready);
    if (e != cudaSuccess) return e;
    // two CTAs an SM would hold the sum of all tiles at once (ragged lists make some CTAs more), each at least two
    const int chunk_tiles = (int)std::max<int64_t>(2, (p.own_tiles + 2 * p.sm_count - 1) / (2 * p.sm_count));
    const int chunks = (p.max_len + chunk_tiles * kTileTokens - 1) / (chunk_tiles * kTileTokens);
    const int64_t blocks = (int64_t)p.n_seq * p.H * chunks;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    if (blocks == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(192);
    cfg.dynamicSmemBytes = weigh_bytes<DP>(p.G * p.q_tokens);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_weigh_kernel<T, DP, FORM>, map, p, chunks, chunk_tiles);
}

}  // namespace

// Rows of 64 to 128 dims, blocks of a multiple of 8 tokens (the period of the swizzle).
bool attend_tile_supported(const pdkv_pool_desc &d)
{
    return d.elem_bytes == 2 && d.head_dim >= 64 && d.head_dim <= 128 && d.head_dim % 8 == 0 && d.block_tokens % 8 == 0 && d.num_blocks <= 0x7fffffff;
}
int attend_tile_box(const pdkv_pool_desc &d) { return std::gcd(d.block_tokens, kTileTokens); }

// A map of the pool whose boxes are 64 dims of `box_tokens` tokens of one head.
bool make_attend_map(const pdkv_pool &pool, int box_tokens, void *out)
{
    static_assert(sizeof(CUtensorMap) <= kMapBytes, "a handle's space for the map");
    void *sym = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
        cudaGetLastError();
        return false;
    }
    const pdkv_pool_desc &d = pool.d;
    const PoolView v = pool_view(pool);
    const cuuint64_t H = d.num_kv_heads, B = d.block_tokens, D = d.head_dim, NB = d.num_blocks, LC = 2 * (cuuint64_t)d.num_layers;
    const cuuint32_t rows = (cuuint32_t)box_tokens, ones[5] = {1, 1, 1, 1, 1};
    const bool layer_major = d.layout == PDKV_LAYOUT_LAYER_MAJOR;
    // block-major: (dim, head, token, layer and K/V, block); layer-major: (dim, token, head, block, layer and K/V)
    const cuuint64_t dims_b[5] = {D, H, B, LC, NB}, dims_l[5] = {D, B, H, NB, LC};
    const cuuint64_t strides_b[4] = {(cuuint64_t)v.head_stride, (cuuint64_t)v.tok_stride, (cuuint64_t)v.lc_stride, (cuuint64_t)v.block_stride};
    const cuuint64_t strides_l[4] = {(cuuint64_t)v.tok_stride, (cuuint64_t)v.head_stride, (cuuint64_t)v.block_stride, (cuuint64_t)v.lc_stride};
    const cuuint32_t box_b[5] = {64, 1, rows, 1, 1}, box_l[5] = {64, rows, 1, 1, 1};
    const cuuint64_t *strides = layer_major ? strides_l : strides_b;
    for (int i = 0; i < 4; ++i)
        if (strides[i] >= 1ull << 40) return false;
    return reinterpret_cast<EncodeTiled>(sym)(static_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, pool.base, layer_major ? dims_l : dims_b, strides,
                                              layer_major ? box_l : box_b, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

template <typename T> cudaError_t launch_weigh_type(const AttnParams &p, const CUtensorMap &m, cudaStream_t stream)
{
    if (p.formed) return p.D <= 64 ? launch_weigh<T, 64, true>(p, m, stream) : launch_weigh<T, 128, true>(p, m, stream);
    return p.D <= 64 ? launch_weigh<T, 64, false>(p, m, stream) : launch_weigh<T, 128, false>(p, m, stream);
}
template <typename T> cudaError_t launch_tile_type(const AttnParams &p, const CUtensorMap &m, cudaStream_t stream)
{
    if (p.formed == kSloped) return p.D <= 64 ? launch_dims<T, 64, kSloped>(p, m, stream) : launch_dims<T, 128, kSloped>(p, m, stream);
    if (p.formed == kCapped) return p.D <= 64 ? launch_dims<T, 64, kCapped>(p, m, stream) : launch_dims<T, 128, kCapped>(p, m, stream);
    if (p.formed == kMasked) return p.D <= 64 ? launch_dims<T, 64, kMasked>(p, m, stream) : launch_dims<T, 128, kMasked>(p, m, stream);
    return p.D <= 64 ? launch_dims<T, 64, kPlain>(p, m, stream) : launch_dims<T, 128, kPlain>(p, m, stream);
}

}  // namespace

cudaError_t launch_attend_weigh(const AttnParams &p, const void *map, int dtype, cudaStream_t stream)
{
    const CUtensorMap &m = *static_cast<const CUtensorMap *>(map);
    return dtype == PDKV_DTYPE_BF16 ? launch_weigh_type<__nv_bfloat16>(p, m, stream) : launch_weigh_type<__half>(p, m, stream);
}

cudaError_t launch_attend_tile(const AttnParams &p, const void *map, int dtype, cudaStream_t stream)
{
    const CUtensorMap &m = *static_cast<const CUtensorMap *>(map);
    return dtype == PDKV_DTYPE_BF16 ? launch_tile_type<__nv_bfloat16>(p, m, stream) : launch_tile_type<__half>(p, m, stream);
}

}  // namespace pdkv
