// Eviction: which tokens of a (layer, sequence, KV head) stay, and the move of their rows.
#include <algorithm>
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

namespace {

// Threads of a selecting CTA and keys that each holds in registers: small CTAs, four on an SM, for rows that fit
// one (their rounds are latency, which other CTAs fill); large ones, two on an SM, in clusters for longer rows.
constexpr int kSmallSelect = 256, kSmallKeys = 32, kLargeSelect = 512, kLargeKeys = 32;

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// Barrier over the CTAs of the cluster (all of their threads); a cluster of one is the CTA.
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// To shared memory of CTA `rank` of the cluster, at the place that `p` has in this CTA's.
__device__ __forceinline__ void put_peer(const int *p, uint32_t rank, int a, int b, int c)
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(p), far;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(at), "r"(rank));
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1,%2,%3,%3};" ::"r"(far), "r"(a), "r"(b), "r"(c) : "memory");
}

// c + (key >= value), from the carry of key - value (value > 0): two instructions.
__device__ __forceinline__ void count_reached(uint32_t &c, uint32_t key, uint32_t minus_value)
{
    asm("{.reg .u32 t;\n add.cc.u32 t, %1, %2;\n addc.u32 %0, %0, 0;}" : "+r"(c) : "r"(key), "r"(minus_value));
}
__device__ __forceinline__ void put_peer(const uint32_t *p, uint32_t rank, uint32_t v)
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(p), far;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(at), "r"(rank));
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(far), "r"(v) : "memory");
}

constexpr int kSample = 128;

template <int THREADS> struct alignas(16) SelectShared {
    int count[3][4];                       // of the CTA, by round modulo 3
    alignas(16) int exchange[2][8][4], totals[8][4];   // of every CTA of the cluster, written as vectors of four
    alignas(16) uint32_t sample[kSample];
    uint32_t sorted[kSample];
    uint32_t close[THREADS];               // keys between the bounds, of the CTA
    uint32_t all_close[THREADS == kSmallSelect ? 1 : 8][THREADS];   // and of every CTA
    int n_close, n_all_close[8];
    uint32_t packed[3];
    int warp_over[32], warp_tie[32];
};

// lo <= the want-th largest key < hi: at least `want` keys reach lo, fewer reach hi.
struct Bounds {
    uint32_t lo, hi;
    int reach_lo, reach_hi;
    __device__ __forceinline__ bool done(int want) const { return reach_lo == want || hi - lo == 1; }
    // Three values inside, in order.
    __device__ __forceinline__ void quarters(uint32_t &p1, uint32_t &p2, uint32_t &p3) const
    {
        const uint32_t quarter = max(1u, (hi - lo) / 4);
        p1 = lo + quarter;
        p2 = lo + max(1u, (hi - lo) / 2);
        p3 = hi - quarter;
    }
    __device__ __forceinline__ void narrow(uint32_t p1, uint32_t p2, uint32_t p3, int c1, int c2, int c3, int want)
    {
        if (c3 >= want) {
            lo = p3;
            reach_lo = c3;
        } else {
            hi = p3;
            reach_hi = c3;
            if (c2 >= want) {
                lo = p2;
                reach_lo = c2;
            } else {
                hi = p2;
                reach_hi = c2;
                if (c1 >= want) {
                    lo = p1;
                    reach_lo = c1;
                } else {
                    hi = p1;
                    reach_hi = c1;
                }
            }
        }
    }
};

// Token t of a row's middle part is one of the `want` heaviest: kept[at ..) receives them in order.
// K keys a thread live in registers, read once; K = 0 (rows of more than 8 x 16384 tokens) reads them again in
// every round.
template <int THREADS, int K>
__device__ __forceinline__ void select_row(SelectShared<THREADS> &sh, const float *row, int lo, int hi, int per, int want, int32_t *kept,
                                           uint32_t rank, uint32_t ranks)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    // tokens of this warp: a contiguous run of 32 * per, lane by lane
    const int64_t first = lo + ((int64_t)rank * (THREADS / 32) + warp) * 32 * per + lane;
    const int begin = (int)min(first, (int64_t)hi);
    const uint32_t drawn = threadIdx.x < kSample ? order_key(row[lo + (int)((int64_t)(hi - lo) * threadIdx.x / kSample)]) : 0u;
    uint32_t keys[K > 0 ? K : 1];
    if (K > 0) {
        float x[K > 0 ? K : 1];   // all on their way before the first is looked at
#pragma unroll
        for (int i = 0; i < K; ++i) x[i] = i < per && begin + 32 * i < hi ? row[begin + 32 * i] : NAN;
#pragma unroll
        for (int i = 0; i < K; ++i) keys[i] = order_key(x[i]);
    }
    auto each = [&](auto &&f) {   // every lane of the warp takes part
        if (K > 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) f(keys[i], begin + 32 * i, i < per);
        } else {
            for (int i = 0; i < per; ++i) f(begin + 32 * i < hi ? order_key(row[begin + 32 * i]) : 0u, begin + 32 * i, true);
        }
    };
    if (threadIdx.x < 12) sh.count[threadIdx.x / 4][threadIdx.x % 4] = 0;
    if (threadIdx.x == 0) sh.n_close = 0;
    if (threadIdx.x < 3) sh.packed[threadIdx.x] = 0;
    if (threadIdx.x < kSample) sh.sample[threadIdx.x] = drawn;
    if (ranks > 1)
        cluster_barrier();   // (from here on the CTAs write to one another: all have to have started)
    else
        __syncthreads();

    Bounds at = {0u, ~0u, hi - lo, 0};   // (~0 is no number's key)
    if (at.reach_lo > THREADS && threadIdx.x < kSample) {
        int heavier = 0;
        for (int j = 0; j < kSample; j += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(&sh.sample[j]);
            const int me = threadIdx.x - j;
            heavier += (o.x > drawn || (o.x == drawn && 0 < me)) + (o.y > drawn || (o.y == drawn && 1 < me)) +
                       (o.z > drawn || (o.z == drawn && 2 < me)) + (o.w > drawn || (o.w == drawn && 3 < me));
        }
        sh.sorted[heavier] = drawn;
    }
    __syncthreads();
#pragma unroll 1
    for (int round = 0; !at.done(want) && at.reach_lo - at.reach_hi > THREADS; ++round) {
        uint32_t p1, p2, p3;
        at.quarters(p1, p2, p3);
        if (round == 0) {
            // Where a sample of the row expects the key: two standard deviations to either side
            const float part = (float)want / (float)(hi - lo);
            const int mid = min((int)(part * kSample), kSample - 1), off = 1 + (int)(2.f * sqrtf(kSample * part * (1.f - part)));
            p1 = min(max(sh.sorted[min(mid + off, kSample - 1)], 1u), ~0u - 1u);
            p2 = min(max(sh.sorted[mid], 1u), ~0u - 1u);
            p3 = min(max(sh.sorted[max(mid - off, 0)], 1u), ~0u - 1u);
        }
        int c1 = 0, c2 = 0, c3 = 0;
        if (K > 0) {
            // (a missing key is 0 and reaches nothing).  At most 512 keys a warp: three counts in one number, one
            // reduction -- there are few lanes for those; 1024 keys: two
            uint32_t n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                count_reached(n1, keys[i], 0u - p1);
                count_reached(n2, keys[i], 0u - p2);
                count_reached(n3, keys[i], 0u - p3);
            }
            if (K <= 16) {
                const uint32_t c = __reduce_add_sync(~0u, n1 + (n2 << 10) + (n3 << 20));
                c1 = c & 1023;
                c2 = c >> 10 & 1023;
                c3 = c >> 20;
            } else {
                const uint32_t c = __reduce_add_sync(~0u, n1 + (n2 << 16));
                c1 = c & 0xffff;
                c2 = c >> 16;
                c3 = __reduce_add_sync(~0u, n3);
            }
        } else {
            each([&](uint32_t k, int, bool) {
                c1 += k >= p1;
                c2 += k >= p2;
                c3 += k >= p3;
            });
            c1 = __reduce_add_sync(~0u, c1);
            c2 = __reduce_add_sync(~0u, c2);
            c3 = __reduce_add_sync(~0u, c3);
        }
        int *mine = sh.count[round % 3];
        if (lane < 3) atomicAdd(&mine[lane], lane == 0 ? c1 : lane == 1 ? c2 : c3);
        if (threadIdx.x < 4) sh.count[(round + 1) % 3][threadIdx.x] = 0;   // (read last two rounds ago)
        __syncthreads();
        c1 = mine[0];
        c2 = mine[1];
        c3 = mine[2];
        if (ranks > 1) {
            int(*far)[4] = sh.exchange[round % 2];
            if (threadIdx.x < ranks) put_peer(far[rank], lane, c1, c2, c3);
            cluster_barrier();
            c1 = c2 = c3 = 0;
            for (uint32_t r = 0; r < ranks; ++r) {
                const int4 v = *reinterpret_cast<const int4 *>(far[r]);
                c1 += v.x;
                c2 += v.y;
                c3 += v.z;
            }
        }
        at.narrow(p1, p2, p3, c1, c2, c3, want);
    }
    if (!at.done(want)) {
        // Few keys are left between the bounds: every CTA gets all of them, one a thread (in any order: only their
        // counts are asked for), and goes on by itself.
        int n = 0;
        each([&](uint32_t k, int t, bool there) { n += there && t < hi && k >= at.lo && k < at.hi; });
        int slot = n;   // of the lane's first, among the warp's
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int x = __shfl_up_sync(~0u, slot, d);
            if (lane >= d) slot += x;
        }
        const int warp_n = __shfl_sync(~0u, slot, 31);
        slot -= n;
        if (warp_n > 0) {
            int to = __shfl_sync(~0u, lane == 0 ? atomicAdd(&sh.n_close, warp_n) : 0, 0) + slot;
            each([&](uint32_t k, int t, bool there) {
                if (there && t < hi && k >= at.lo && k < at.hi && to < THREADS) sh.close[to++] = k;
            });
        }
        __syncthreads();
        uint32_t mine = threadIdx.x < sh.n_close ? sh.close[threadIdx.x] : 0u;
        if (ranks > 1) {
            if (threadIdx.x < sh.n_close)
                for (uint32_t r = 0; r < ranks; ++r) put_peer(&sh.all_close[rank][threadIdx.x], r, mine);
            if (threadIdx.x < ranks) put_peer(reinterpret_cast<const uint32_t *>(&sh.n_all_close[rank]), lane, sh.n_close);
            cluster_barrier();
            int i = threadIdx.x;   // of all
            mine = 0;
            for (uint32_t r = 0; r < ranks; ++r) {
                const int n_r = sh.n_all_close[r];
                if (i >= 0 && i < n_r) mine = sh.all_close[r][i];
                i -= n_r;
            }
        }
        const int above = at.reach_hi;
#pragma unroll 1
        for (int round = 0; !at.done(want); ++round) {
            uint32_t p1, p2, p3;
            at.quarters(p1, p2, p3);
            // three counts below 1024 in one number
            const uint32_t c = __reduce_add_sync(~0u, (mine >= p1) + (mine >= p2 ? 1u << 10 : 0u) + (mine >= p3 ? 1u << 20 : 0u));
            if (lane == 0 && c) atomicAdd(&sh.packed[round % 3], c);
            if (threadIdx.x == 0) sh.packed[(round + 1) % 3] = 0;   // (read last two rounds ago)
            __syncthreads();
            const uint32_t sum = sh.packed[round % 3];
            at.narrow(p1, p2, p3, above + (sum & 1023), above + (sum >> 10 & 1023), above + (sum >> 20), want);
        }
    }
    const uint32_t key = at.lo;
    // Either exactly `want` keys reach `key`: all of them stay.  Or `key` is the want-th key itself: of the
    // keys equal to it those of the lowest tokens stay, as many as are left.
    const bool all = at.reach_lo == want;
    int over = 0, tie = 0;
    each([&](uint32_t k, int t, bool there) {
        there = there && t < hi;
        over += there && (all ? k >= key : k > key);
        tie += there && !all && k == key;
    });
    over = __reduce_add_sync(~0u, over);
    tie = __reduce_add_sync(~0u, tie);
    if (lane == 0) {
        sh.warp_over[warp] = over;
        sh.warp_tie[warp] = tie;
    }
    __syncthreads();
    {
        const int o = lane < THREADS / 32 ? sh.warp_over[lane] : 0, e = lane < THREADS / 32 ? sh.warp_tie[lane] : 0;
        over = __reduce_add_sync(~0u, lane < warp ? o : 0);   // from here on: counts before this warp
        tie = __reduce_add_sync(~0u, lane < warp ? e : 0);
        const int all_over = __reduce_add_sync(~0u, o), all_tie = __reduce_add_sync(~0u, e);
        int left = want - all_over;   // of the ties
        if (ranks > 1) {
            if (threadIdx.x < ranks) put_peer(sh.totals[rank], lane, all_over, all_tie, 0);
            cluster_barrier();
            const int o_r = lane < ranks ? sh.totals[lane][0] : 0, e_r = lane < ranks ? sh.totals[lane][1] : 0;
            over += __reduce_add_sync(~0u, lane < rank ? o_r : 0);
            tie += __reduce_add_sync(~0u, lane < rank ? e_r : 0);
            left = want - (int)__reduce_add_sync(~0u, o_r);
        }
        const unsigned below = (1u << lane) - 1;
        if (all) {
            each([&](uint32_t k, int t, bool there) {
                const bool stays = there && t < hi && k >= key;
                const unsigned mask = __ballot_sync(~0u, stays);
                if (stays) kept[over + __popc(mask & below)] = t;
                over += __popc(mask);
            });
        } else {
            each([&](uint32_t k, int t, bool there) {
                there = there && t < hi;
                const bool is_over = there && k > key, is_tie = there && k == key;
                const unsigned over_mask = __ballot_sync(~0u, is_over), tie_mask = __ballot_sync(~0u, is_tie);
                const int x = over + __popc(over_mask & below), e = tie + __popc(tie_mask & below);
                if (is_over || (is_tie && e < left)) kept[x + min(e, left)] = t;
                over += __popc(over_mask);
                tie += __popc(tie_mask);
            });
        }
    }
}

}  // namespace

// One cluster per (layer, sequence, head).  The lightest key that stays is enclosed by counting the keys that reach
// three values a round: first three of a sorted sample, then the quarters of the interval.  Once a CTA's threads can hold
// the keys inside, one each, they are gathered and the rest is counted by barriers; it ends when exactly the
// wanted number of keys reaches the lower bound, or the interval is one key (18 rounds at most whatever the keys: the one of the
// sample, which may cut off a single key, and 17 quarterings of 2^32).
// Then the indices are written in order.  Counting needs two instructions a key and value (a histogram in shared memory
// was 1.5 times slower: scores crowd into few bins); the three counts of a warp go through one integer reduction, CTAs of
// a cluster exchange theirs over distributed shared memory.  Every warp owns a contiguous run of tokens, so the order of
// the indices follows from counts per warp alone.  Bound by the latency of its steps.  16 rows of 100003 tokens, a cluster of 8
// each, take 28 to 30 us: 8000 cycles until the keys are there, 3100 to sort the sample, 2 to 7 rounds over the cluster of
// 3700 to 4900 (the exchange 1500 of them), 8000 to 11000 to gather the keys inside, 4 to 6 rounds within the CTA for 4000, 17000 to
// write the indices.  2048 rows of 16 to 8192 tokens, a CTA each, 35 us.
// (ptxas keeps the kernel to the 64 registers that two CTAs of 512 threads leave, at 108 to 136 bytes of spills.)
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_select_kernel(const EvictParams p)
{
    __shared__ __align__(16) SelectShared<THREADS> sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // set up while the work before this call ends
    asm volatile("griddepcontrol.launch_dependents;");
    const uint32_t rank = THREADS == kSmallSelect ? 0 : cluster_rank(), ranks = THREADS == kSmallSelect ? 1 : cluster_size();
    const int row_id = blockIdx.x / ranks;
    const int head = row_id % p.H, seq = row_id / p.H % p.n_seq, layer = row_id / p.H / p.n_seq;
    const int len = own_len(p, seq);
    int32_t *kept = p.kept + (int64_t)row_id * p.budget;
    const int first = rank * THREADS + threadIdx.x, step = ranks * THREADS;
    const int want = p.budget - p.sink - p.recent;
    for (int j = min(len, p.budget) + first; j < p.budget; j += step) kept[j] = -1;
    if (len <= p.budget || want == 0) {
        const int n = min(len, p.budget), head_part = len <= p.budget ? n : p.sink;
        for (int j = first; j < n; j += step) kept[j] = j < head_part ? j : len - n + j;
        return;
    }
    const int lo = p.sink, hi = len - p.recent;
    for (int j = first; j < p.sink; j += step) kept[j] = j;
    for (int j = first; j < p.recent; j += step) kept[p.budget - p.recent + j] = hi + j;
    const float *row = p.scores + layer * p.scores_stride[0] + seq * p.scores_stride[1] + head * p.scores_stride[2];
    const int per = (int)(((int64_t)hi - lo + step - 1) / step);
    kept += p.sink;
    if (per <= 2)
        select_row<THREADS, 2>(sh, row, lo, hi, per, want, kept, rank, ranks);
    else if (per <= 4)
        select_row<THREADS, 4>(sh, row, lo, hi, per, want, kept, rank, ranks);
    else if (per <= 8)
        select_row<THREADS, 8>(sh, row, lo, hi, per, want, kept, rank, ranks);
    else if (per <= 16)
        select_row<THREADS, 16>(sh, row, lo, hi, per, want, kept, rank, ranks);
    else if (per <= 32)
        select_row<THREADS, 32>(sh, row, lo, hi, per, want, kept, rank, ranks);
    else if (THREADS == kLargeSelect)
        select_row<THREADS, 0>(sh, row, lo, hi, per, want, kept, rank, ranks);
}

namespace {

constexpr int kMoveThreads = 128, kMoveWarps = kMoveThreads / 32;
constexpr int kMoveVecs = 8;      // vectors a lane has in flight

// Vectors of 32 bytes are moved as eight words: one 256-bit access.
struct Vec32 {
    uint32_t w[8];
};
template <typename V> __device__ __forceinline__ V load_vec(const char *p) { return *reinterpret_cast<const V *>(p); }
template <> __device__ __forceinline__ Vec32 load_vec<Vec32>(const char *p)
{
    Vec32 v;
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7])
                 : "l"(p) : "memory");
    return v;
}
template <typename V> __device__ __forceinline__ void store_vec(char *p, const V &v) { *reinterpret_cast<V *>(p) = v; }
template <> __device__ __forceinline__ void store_vec<Vec32>(char *p, const Vec32 &v)
{
    asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]),
                 "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7]), "l"(p) : "memory");
}

// Kept tokens of a row of indices: they stand before the -1s.  32 probes a round.
__device__ __forceinline__ int count_kept(const int32_t *kept, int most, int lane)
{
    int lo = 0, hi = most;   // kept[lo - 1] >= 0, kept[hi] < 0
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, at = lo + step * lane + step - 1;
        const bool there = at < hi && kept[at] >= 0;
        const int n = __popc(__ballot_sync(~0u, there));
        const int new_lo = lo + n * step;
        hi = min(hi, new_lo + step - 1);
        lo = new_lo;
    }
    return lo;
}

}  // namespace

// Moves the kept rows of one (layer, sequence, head, K/V); bound by memory (1.65 GB read and written in 265 us, 6.2 TB/s, with
// blocks of 16 tokens and rows of 256 bytes at random places).  A warp moves `rows`
// consecutive kept rows at a time: lane i looks up where row i lies and goes, the vectors of the
// rows are dealt to the lanes, all of a lane's loads are issued before its first store, and the next
// rows are looked up meanwhile.  Nothing is shared between warps.
//
// Out of place the steps of a row list are dealt to `parts` blocks.  ORDERED (in place, or scores that
// are compacted where they stand): token kept[j] >= j goes to slot j, so the slots that rows [a, b)
// write hold sources of rows < b only.  It is enough that rows are written after all rows up to
// them were read: the parts are the CTAs of one cluster, all of its warps load consecutive rows, and
// a barrier stands between their loads and their stores.  Rows that stay where they are are not touched.
template <typename V, bool ORDERED>
__global__ void __launch_bounds__(kMoveThreads, 4) evict_move_kernel(const EvictParams p, const int parts)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int part = blockIdx.x % parts, x = blockIdx.x / parts, c = x & 1, stream = x >> 1;
    const int head = stream % p.H, seq = stream / p.H % p.n_seq, layer = stream / p.H / p.n_seq;
    const int32_t *kept = p.kept + (int64_t)stream * p.budget;
    const AttnSeg from = p.src_segs[seq], to = p.dst_segs[seq];
    const int vecs = p.row_bytes / (int)sizeof(V);
    const int most = min(p.budget, from.len);
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the indices are written by the kernel before
    const int n_kept = p.seq_len ? count_kept(kept, most, lane) : most;
    const char *src = p.src.base + (2 * (p.layer_begin + layer) + c) * p.src.lc_stride + head * p.src.head_stride;
    char *dst = p.dst.base + (2 * (p.layer_begin + layer) + c) * p.dst.lc_stride + head * p.dst.head_stride;
    float *scores_to = c == 0 && p.kept_scores
                           ? p.kept_scores + layer * p.kept_scores_stride[0] + seq * p.kept_scores_stride[1] + head * p.kept_scores_stride[2]
                           : nullptr;
    const float *scores = p.scores + layer * p.scores_stride[0] + seq * p.scores_stride[1] + head * p.scores_stride[2];
    if (p.new_len && x == seq * p.H * 2 && part == 0 && threadIdx.x == 0) p.new_len[seq] = n_kept;

    // rows of a step; a row of more vectors than a warp takes at once is moved in several pieces
    constexpr int kWarpVecs = 32 * kMoveVecs;
    const int rows = max(1, min(32, kWarpVecs / vecs)), pieces = (vecs + kWarpVecs - 1) / kWarpVecs;
    const int64_t warps = (int64_t)parts * kMoveWarps, runs = (n_kept + rows - 1) / rows;
    const int64_t steps = (runs + warps - 1) / warps * pieces;
    int64_t next_from = -1, next_to = 0;
    float next_score = 0.f;
    int next_j = -1;
    auto look_up = [&](int64_t step) {
        const int64_t j = ((step / pieces * parts + part) * kMoveWarps + warp) * rows + lane;
        next_from = -1;
        next_j = -1;
        if (step >= steps || lane >= rows || j >= n_kept) return;
        const int t = kept[j];
        const int sb = p.src_shift >= 0 ? t >> p.src_shift : t / p.src.block_tokens;
        const int db = p.dst_shift >= 0 ? (int)j >> p.dst_shift : (int)j / p.dst.block_tokens;
        next_to = p.dst_tbl[to.tbl + db] * p.dst.block_stride + ((int)j - db * p.dst.block_tokens) * p.dst.tok_stride;
        if (!(p.in_place && t == j))
            next_from = p.src_tbl[from.tbl + sb] * p.src.block_stride + (t - sb * p.src.block_tokens) * p.src.tok_stride;
        if (scores_to && step % pieces == 0) {
            next_score = scores[t];
            next_j = (int)j;
        }
    };
    look_up(0);
    for (int64_t step = 0; step < steps; ++step) {
        const int64_t from_at = next_from, to_at = next_to;
        const float score = next_score;
        const int score_j = next_j;
        // vector k of the step: lane + 32 i; row k / vecs
        const int first = (int)(step % pieces) * kWarpVecs + lane;
        V v[kMoveVecs];
        int row = pieces > 1 ? 0 : first / vecs, col = pieces > 1 ? first : first % vecs;
#pragma unroll
        for (int i = 0; i < kMoveVecs; ++i) {
            const int64_t at = __shfl_sync(~0u, from_at, row & 31);
            if (row < rows && col < vecs && at >= 0) v[i] = load_vec<V>(src + at + col * (int)sizeof(V));
            col += 32;
            if (pieces == 1)
                while (col >= vecs) {
                    col -= vecs;
                    ++row;
                }
        }
        look_up(step + 1);
        if (ORDERED) cluster_barrier();
        row = pieces > 1 ? 0 : first / vecs, col = pieces > 1 ? first : first % vecs;
#pragma unroll
        for (int i = 0; i < kMoveVecs; ++i) {
            const int64_t at = __shfl_sync(~0u, from_at, row & 31), dat = __shfl_sync(~0u, to_at, row & 31);
            if (row < rows && col < vecs && at >= 0) store_vec<V>(dst + dat + col * (int)sizeof(V), v[i]);
            col += 32;
            if (pieces == 1)
                while (col >= vecs) {
                    col -= vecs;
                    ++row;
                }
        }
        if (score_j >= 0) scores_to[score_j] = score;
    }
    if (scores_to) {
        if (ORDERED) cluster_barrier();
        for (int j = n_kept + part * kMoveThreads + threadIdx.x; j < p.kept_scores_len; j += parts * kMoveThreads) scores_to[j] = 0.f;
    }
}

namespace {

template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), int64_t rows, int cluster, int threads, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * cluster));
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits for the one before it on the device
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;   // (a CTA is a cluster of one)
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename V> cudaError_t launch_move(const EvictParams &p, int sm_count, cudaStream_t stream)
{
    const int64_t streams = 2 * (int64_t)p.n_layers * p.n_seq * p.H;
    const bool ordered = p.in_place || p.kept_scores == p.scores;
    const int vecs = p.row_bytes / (int)sizeof(V), rows = std::max(1, std::min(32, 32 * kMoveVecs / vecs)) * kMoveWarps;
    const int64_t steps = (std::min(p.budget, p.max_len) + rows - 1) / rows;
    // four blocks for every SM if there are that many steps
    int64_t parts = 1;
    const int64_t most = ordered ? 8 : 1 << 16;
    while (parts * 2 <= most && streams * parts < 4 * sm_count && steps >= 2 * parts) parts *= 2;
    if (streams * parts > INT32_MAX) return cudaErrorInvalidConfiguration;
    if (ordered) return launch_clusters(evict_move_kernel<V, true>, streams, (int)parts, kMoveThreads, stream, p, (int)parts);
    return launch_clusters(evict_move_kernel<V, false>, streams * parts, 1, kMoveThreads, stream, p, (int)parts);
}

}  // namespace

cudaError_t launch_evict(const EvictParams &p, int sm_count, cudaStream_t stream)
{
    const int64_t rows = (int64_t)p.n_layers * p.n_seq * p.H;
    cudaError_t e;
    if (p.max_len <= kSmallSelect * kSmallKeys) {
        if (rows > INT32_MAX) return cudaErrorInvalidConfiguration;
        e = launch_clusters(evict_select_kernel<kSmallSelect>, rows, 1, kSmallSelect, stream, p);
    } else {
        // CTAs per row: as many as its keys need registers, or, few rows, as keep every CTA at 2048 keys and more while
        // all clusters run at once (a cluster stays within a group of SMs, so an eighth of them can be left over)
        int cluster = (int)std::min<int64_t>(8, (p.max_len + kLargeSelect * kLargeKeys - 1) / (kLargeSelect * kLargeKeys));
        while (cluster < 8 && rows * (cluster + 1) <= 2 * (sm_count - sm_count / 8) && p.max_len > cluster * 2048) ++cluster;
        if (rows * cluster > INT32_MAX) return cudaErrorInvalidConfiguration;
        e = launch_clusters(evict_select_kernel<kLargeSelect>, rows, cluster, kLargeSelect, stream, p);
    }
    if (e != cudaSuccess) return e;
    switch (p.vec_bytes) {
    case 32: return launch_move<Vec32>(p, sm_count, stream);
    case 16: return launch_move<uint4>(p, sm_count, stream);
    case 8: return launch_move<uint2>(p, sm_count, stream);
    case 4: return launch_move<uint32_t>(p, sm_count, stream);
    case 2: return launch_move<uint16_t>(p, sm_count, stream);
    default: return launch_move<uint8_t>(p, sm_count, stream);
    }
}

}  // namespace pdkv
