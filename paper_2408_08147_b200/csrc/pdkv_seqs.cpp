// Handles of cached sequences and the entry points of the operators that work on them: the host
// checks a batch's tables once, cuts its attention into work items of equal cost and uploads the
// lists; the calls themselves only enqueue kernels.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <limits>
#include <new>
#include <stdexcept>

#include "pdkv_checks.h"
#include "pdkv_seqs.h"

namespace pdkv {

PoolView pool_view(const pdkv_pool &p)
{
    const int64_t row = (int64_t)p.d.head_dim * p.d.elem_bytes, hrow = row * p.d.num_kv_heads;
    PoolView v;
    v.base = p.base;
    v.block_tokens = p.d.block_tokens;
    if (p.d.layout == PDKV_LAYOUT_BLOCK_MAJOR) {
        v.lc_stride = p.d.block_tokens * hrow;
        v.block_stride = 2 * p.d.num_layers * v.lc_stride;
        v.tok_stride = hrow;
        v.head_stride = row;
    } else {
        v.block_stride = p.d.block_tokens * hrow;
        v.lc_stride = p.d.num_blocks * v.block_stride;
        v.tok_stride = row;
        v.head_stride = p.d.block_tokens * row;
    }
    return v;
}

}  // namespace pdkv

namespace {

using pdkv::AttnItem;
using pdkv::AttnSeg;
using pdkv::AttnSeq;
using pdkv::AttnUnit;
using pdkv::aligned;
using pdkv::kMaxTokens;
using pdkv::log2_of;
using pdkv::meet;
using pdkv::ranges_overlap;
using pdkv::Rows;
using pdkv::rows_apart;

constexpr int kMaxRowTile = 64;    // rows of one work item
// Rows from which the tile kernel takes a segment: 40000 tokens of 8 heads of 128 dims, 32 rows 52 to 54 us in the warp kernel and
// 40 rows 82, in the tile kernel 33 to 64 rows 48 to 49.
constexpr int kTileMinRows = 33;

int check_lists(const int64_t *off, const int32_t *tbl, const int32_t *len, int32_t n, int64_t B, int64_t NB)
{
    if (!off || !len) return PDKV_ERR_INVALID_ARG;
    // all offsets before the first id: a caller who knows where the table ends compares it with off[n]
    if (off[0] < 0) return PDKV_ERR_TABLE;
    for (int32_t r = 0; r < n; ++r)
        if (off[r + 1] < off[r]) return PDKV_ERR_TABLE;
    for (int32_t r = 0; r < n; ++r) {
        if (len[r] < 0) return PDKV_ERR_INVALID_ARG;
        if (len[r] > kMaxTokens) return PDKV_ERR_LIMIT;
        const int64_t need = ((int64_t)len[r] + B - 1) / B;
        if (off[r + 1] - off[r] < need) return PDKV_ERR_TABLE;
        if (need && !tbl) return PDKV_ERR_INVALID_ARG;
        for (int64_t j = 0; j < need; ++j)
            if (tbl[off[r] + j] < 0 || tbl[off[r] + j] >= NB) return PDKV_ERR_TABLE;
    }
    return PDKV_OK;
}

// Which kernel takes a segment, and how its rows are cut.  0, the warp kernel: 16 to 64 rows an item.
// 1, the tile kernel: up to 256 rows an item.
struct Shape {
    int kernel, row_tile;
};

// Which of the two is quicker for `rows` rows against `len` own tokens of one head.  The tile kernel multiplies faster
// but takes longer to start and finish an item.  Measured on B200, microseconds of an SM: warp kernel 1.8 an item of
// 64 rows and 2 for each 64 tokens of it; tile kernel 8 an item of up to 256 rows and 2 for each 128 tokens, 256
// with up to 128 rows.  (64 sequences of 12 to 19 tokens, 49 rows, 5 heads: 31 us against 60.)
bool tile_is_faster(int64_t rows, int64_t len)
{
    const double warp = (double)((rows + 63) / 64) * (1.8 + 2.0 * (double)((len + 63) / 64));
    const int64_t full = rows / 256, rest = rows % 256, n128 = (len + 127) / 128, n256 = (len + 255) / 256;
    const double tile = (double)full * (8 + 2.0 * (double)n128) + (rest == 0 ? 0 : 8 + 2.0 * (double)(rest > 128 ? n128 : n256));
    return rows >= kTileMinRows && tile < warp;
}
Shape shape_of(int64_t rows, bool tile)
{
    if (tile) return {1, 256};
    return {0, rows <= 16 ? 16 : rows <= 32 ? 32 : kMaxRowTile};
}

// What starting and finishing an item costs, and what a quantum does: 64 tokens for up to 16 rows in the warp kernel,
// which memory bounds, more rows of long heads by their products; 128 or 256 tokens in the tile kernel.  In halves
// of such a quantum.  Measured: 3 us against 1.5 us (a CTA's share of the memory rate) in the warp kernel, 15000
// cycles against 3700 in the tile kernel.
constexpr int64_t kItemCost[2] = {4, 8};
int64_t quantum_load(int kernel, int32_t rows, int32_t head_dim)
{
    if (kernel == 1 || rows <= 16) return 2;
    if (rows <= 32) return head_dim <= 128 ? 2 : 3;
    return head_dim <= 128 ? 3 : 6;
}

// Tokens of a quantum, its load, how many there are.
struct Unit { int32_t seg, head, row0, rows; int64_t quantum, weight, quanta; };
struct Piece { size_t unit; int64_t from, n; int32_t cta; };

// Deals units to CTAs in order, each CTA up to a load of `most`; units are cut where a CTA is full.  Returns
// false when that takes more than `n_ctas` CTAs.
bool deal(const std::vector<Unit> &units, int64_t cost, int64_t most, int64_t n_ctas, bool cut, std::vector<Piece> *out)
{
    int64_t cta = 0, load = 0;
    for (size_t u = 0; u < units.size(); ++u) {
        const Unit &w = units[u];
        int64_t q = 0;
        while (q < w.quanta) {
            int64_t room = std::max<int64_t>(0, most - load - cost) / w.weight;
            if (load > 0 && (room < 1 || (!cut && room < w.quanta))) {
                ++cta;
                load = 0;
                room = std::max<int64_t>(0, most - cost) / w.weight;
            }
            const int64_t n = std::min(w.quanta - q, room);
            if (cta >= n_ctas || n < 1 || (!cut && n < w.quanta)) return false;
            if (out) out->push_back({u, q, n, (int32_t)cta});
            load += cost + n * w.weight;
            q += n;
        }
    }
    return true;
}

// Smallest load per CTA with which the units fit.
int64_t least_load(const std::vector<Unit> &units, int64_t cost, int64_t n_ctas, bool cut)
{
    int64_t total = 0, longest = 0, heaviest = 1;
    for (const Unit &u : units) {
        total += u.quanta * u.weight + cost;
        longest = std::max(longest, u.quanta * u.weight + cost);
        heaviest = std::max(heaviest, u.weight);
    }
    // (cut, every CTA has room for a quantum; a load of everything always fits)
    int64_t lo = std::max((total + n_ctas - 1) / n_ctas, cut ? cost + heaviest : longest), hi = std::max(lo, total);
    while (lo < hi) {
        const int64_t mid = lo + (hi - lo) / 2;
        if (deal(units, cost, mid, n_ctas, cut, nullptr))
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

std::vector<Unit> units_of(const pdkv_seqs &s, int kernel, const std::vector<int32_t> &n_rows, const std::vector<Shape> &shape)
{
    std::vector<Unit> units;
    for (size_t g = 0; g < s.segs.size(); ++g) {
        const AttnSeg &seg = s.segs[g];
        if (shape[g].kernel != kernel || seg.len == 0 || n_rows[g] == 0) continue;
        for (int32_t r0 = 0; r0 < n_rows[g]; r0 += shape[g].row_tile)
            for (int32_t h = 0; h < s.pool.d.num_kv_heads; ++h) {
                const int32_t rows = std::min<int32_t>(shape[g].row_tile, n_rows[g] - r0);
                const int64_t quantum = kernel == 0 ? 64 : rows <= 128 ? 256 : 128;   // (one row tile: two tiles of tokens at a time)
                units.push_back({(int32_t)g, h, r0, rows, quantum, quantum_load(kernel, rows, s.pool.d.head_dim), (seg.len + quantum - 1) / quantum});
            }
    }
    return units;
}

// SMs for the tile kernel when both kernels have work: they run at the same time, each on SMs of its own (a CTA of
// the tile kernel leaves no shared memory for others), and the slower one should be as quick as possible.
// Measured on B200: 2.2 us a quantum of the tile kernel -- 3.4 us beside a saturated memory -- and 4 us around it; an SM
// of the warp kernel reads 76 GB/s and takes 1.8 us to change items, 6.3 TB/s for all of them, 5 us around it.
int tile_sms(const pdkv_seqs &s, const std::vector<Unit> &warp_units, const std::vector<Unit> &tile_units)
{
    if (warp_units.empty()) return s.sm_count;
    if (tile_units.empty()) return 0;
    double bytes = 0;
    for (const Unit &u : warp_units) bytes += (double)(u.quantum * u.quanta) * 4 * s.pool.d.head_dim;
    int best = 1;
    double best_us = 1e30;
    auto attempt = [&](int n) {
        if (n < 1 || n >= s.sm_count) return;
        const double load = 0.5 * (double)least_load(tile_units, kItemCost[1], n, true);   // quanta
        const double warp_us = 5 + std::max(bytes / 6.3e6, (bytes / 76e3 + 1.8 * (double)warp_units.size()) / (s.sm_count - n));
        const double busy = std::min(1.0, bytes / 6.3e6 / std::max(warp_us, 4 + 2.2 * load));   // share of the time with a saturated memory
        const double us = std::max(warp_us, 4 + (2.2 + 1.2 * busy) * load);
        if (us < best_us) {
            best_us = us;
            best = n;
        }
    };
    for (int n = 4; n < s.sm_count; n += 8) attempt(n);
    const int about = best;
    for (int n = about - 7; n <= about + 7; ++n) attempt(n);
    return best;
}

// Work list of one kernel.  Whole units when that is as quick as cutting them (nothing is to be joined then,
// which saves a kernel: about two quanta more); else CTAs get at least two quanta (one of the tile kernel), so that
// joining stays cheap.
void plan_items(pdkv_seqs &s, int kernel, const std::vector<Unit> &units, std::vector<int32_t> &unit0, int n_ctas_max)
{
    int64_t load = 0;
    for (size_t u = 0; u < units.size(); ++u) {
        load += units[u].quanta * units[u].weight;
        if (unit0[(size_t)units[u].seg] < 0) unit0[(size_t)units[u].seg] = (int32_t)(s.units.size() + u);
    }
    std::vector<AttnItem> &items = s.items[kernel];
    if (units.empty()) return;
    const int64_t cost = kItemCost[kernel], least = kernel == 0 ? 4 : 2;
    const int64_t n_ctas = std::max<int64_t>(1, std::min<int64_t>(n_ctas_max, std::max<int64_t>(units.size(), load / least)));
    std::vector<Piece> pieces;
    const int64_t cut = least_load(units, cost, n_ctas, true), whole = least_load(units, cost, n_ctas, false);
    const bool keep_whole = whole <= cut + 4;
    deal(units, cost, keep_whole ? whole : cut, n_ctas, !keep_whole, &pieces);
    const size_t first_unit = s.units.size();
    s.units.resize(first_unit + units.size());
    for (const Piece &x : pieces) {
        const Unit &w = units[x.unit];
        const AttnSeg &seg = s.segs[(size_t)w.seg];
        const int parts = kernel == 1 && w.rows <= 128 ? 2 : 1;   // the tile kernel leaves one for each half of a CTA
        AttnUnit &unit = s.units[first_unit + x.unit];
        if (x.from == 0) unit = {s.part_rows, 0, w.rows};
        unit.n_parts += parts;
        AttnItem it{};
        it.part_row = s.part_rows;
        it.tbl = seg.tbl;
        it.seq = seg.seq;
        it.member_begin = seg.member_begin;
        it.len = seg.len;
        it.head = w.head;
        it.row0 = w.row0;
        it.rows = w.rows;
        it.tok0 = (int32_t)(x.from * w.quantum);
        it.tok1 = (int32_t)std::min<int64_t>(seg.len, (x.from + x.n) * w.quantum);
        s.part_rows += parts * w.rows;
        pdkv_attend_item li{};
        li.prefix = w.seg >= s.n_seq ? w.seg - s.n_seq : -1;
        li.seq = w.seg < s.n_seq ? w.seg : -1;
        li.head = w.head;
        li.row_begin = w.row0;
        li.row_end = w.row0 + w.rows;
        li.tok_begin = it.tok0;
        li.tok_end = it.tok1;
        li.kernel = kernel;
        li.cta = x.cta;
        s.listing.push_back(li);
        items.push_back(it);
        s.item_cta[kernel].push_back(x.cta);
    }
    s.n_ctas[kernel] = pieces.back().cta + 1;
}

// The list as the kernels read it: the first item of CTA c at place c, the CTA's further ones behind all
// first ones, each item leading to the next.  A CTA starts on its first item after one load.
std::vector<AttnItem> chain_items(const std::vector<AttnItem> &items, const std::vector<int32_t> &cta, int32_t n_ctas)
{
    std::vector<AttnItem> out((size_t)n_ctas);
    size_t last = 0;
    for (size_t i = 0; i < items.size(); ++i) {
        size_t at = (size_t)cta[i];
        if (i > 0 && cta[i] == cta[i - 1]) {
            at = out.size();
            out.push_back(AttnItem{});
            out[last].next = (int32_t)at;
        }
        out[at] = items[i];
        out[at].next = -1;
        last = at;
    }
    return out;
}

}  // namespace

extern "C" {

int pdkv_seqs_create(const pdkv_pool *pool, const pdkv_seqs_desc *d, void *workspace, size_t workspace_bytes,
                     size_t *needed_bytes, void *stream, pdkv_seqs **out)
{
    if (out) *out = nullptr;
    if (needed_bytes) *needed_bytes = 0;
    if (!out || !pool || !d) return PDKV_ERR_INVALID_ARG;
    if (d->n_seq < 0 || d->n_prefix < 0 || d->num_q_heads < 0) return PDKV_ERR_INVALID_ARG;
    if (workspace && !aligned(workspace, 16)) return PDKV_ERR_INVALID_ARG;
    const pdkv_pool_desc &g = pool->d;
    const bool attention = d->num_q_heads > 0;
    if (attention) {
        if (d->q_tokens < 1 || (d->dtype != PDKV_DTYPE_BF16 && d->dtype != PDKV_DTYPE_FP16)) return PDKV_ERR_INVALID_ARG;
        if (d->num_q_heads % g.num_kv_heads || g.elem_bytes != 2 || g.head_dim % 8 || g.head_dim > 256) return PDKV_ERR_GEOMETRY;
        // rows of one sequence and head, and rows behind one prefix, are counted in 32 bits
        const int64_t rows = (int64_t)d->q_tokens * d->num_q_heads, most = (int64_t)1 << 30;
        if (rows > most / std::max(1, d->n_seq)) return PDKV_ERR_INVALID_ARG;
    }
    const int64_t B = g.block_tokens;
    try {
        if (d->n_seq > 0) {
            const int rc = check_lists(d->tbl_off, d->tbl, d->seq_len, d->n_seq, B, g.num_blocks);
            if (rc != PDKV_OK) return rc;
        }
        if (d->n_prefix > 0) {
            const int rc = check_lists(d->prefix_tbl_off, d->prefix_tbl, d->prefix_len, d->n_prefix, B, g.num_blocks);
            if (rc != PDKV_OK) return rc;
            if (!d->seq_prefix && d->n_seq > 0) return PDKV_ERR_INVALID_ARG;
            for (int32_t r = 0; r < d->n_seq; ++r)
                if (d->seq_prefix[r] < -1 || d->seq_prefix[r] >= d->n_prefix) return PDKV_ERR_INVALID_ARG;
        }
        pdkv_seqs *s = new pdkv_seqs;
        struct Holder {
            pdkv_seqs *s;
            ~Holder() { if (s) pdkv_seqs_destroy(s); }
        } hold{s};
        s->pool = *pool;
        s->device = pool->device;
        s->n_seq = d->n_seq;
        s->n_prefix = d->n_prefix;
        s->len.assign(d->seq_len, d->seq_len + d->n_seq);
        for (int32_t n : s->len) s->max_len = std::max(s->max_len, n);
        s->Hq = d->num_q_heads;
        s->G = attention ? d->num_q_heads / g.num_kv_heads : 0;
        s->q_tokens = attention ? d->q_tokens : 0;
        s->dtype = d->dtype;

        if (!pdkv::tunables().dry_run) {
            const cudaError_t e = cudaDeviceGetAttribute(&s->sm_count, cudaDevAttrMultiProcessorCount, s->device);
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "cudaDeviceGetAttribute");
        }

        // tables, own tokens first, only the entries that hold tokens
        std::vector<int32_t> tbl;
        std::vector<uint8_t> seen((size_t)g.num_blocks, 0);
        auto add = [&](const int64_t *off, const int32_t *ids, int32_t r, int32_t len, int32_t seq) {
            AttnSeg seg{};
            seg.tbl = (int64_t)tbl.size();
            seg.len = len;
            seg.seq = seq;
            const int64_t need = ((int64_t)len + B - 1) / B;
            for (int64_t j = 0; j < need; ++j) {
                const int32_t id = ids[off[r] + j];
                tbl.push_back(id);
                if (seen[(size_t)id]) s->unique_blocks = false;
                seen[(size_t)id] = 1;
            }
            s->segs.push_back(seg);
        };
        for (int32_t r = 0; r < d->n_seq; ++r) {
            add(d->tbl_off, d->tbl, r, d->seq_len[r], r);
            if (d->n_prefix > 0 && d->seq_prefix[r] >= 0) s->segs.back().before = d->prefix_len[d->seq_prefix[r]];
        }
        for (int32_t p = 0; p < d->n_prefix; ++p) add(d->prefix_tbl_off, d->prefix_tbl, p, d->prefix_len[p], -1);

        std::vector<int32_t> members;
        if (attention) {
            const int64_t R = (int64_t)s->G * s->q_tokens;
            std::vector<int32_t> n_rows(s->segs.size(), 0), row0((size_t)s->n_seq, 0);
            for (int32_t r = 0; r < s->n_seq; ++r) n_rows[(size_t)r] = (int32_t)R;
            for (int32_t p = 0; p < s->n_prefix; ++p) {
                AttnSeg &seg = s->segs[(size_t)(s->n_seq + p)];
                seg.member_begin = (int32_t)members.size();
                for (int32_t r = 0; r < s->n_seq; ++r)
                    if (d->seq_prefix[r] == p) {
                        row0[(size_t)r] = n_rows[(size_t)(s->n_seq + p)];
                        n_rows[(size_t)(s->n_seq + p)] += (int32_t)R;
                        members.push_back(r);
                    }
            }
            bool tile_ok = pdkv::attend_tile_supported(g);
            if (!pdkv::tunables().dry_run) {
                tile_ok = tile_ok && pdkv::make_attend_map(*pool, pdkv::attend_tile_box(g), s->map[1]);
                s->use_map = pdkv::attend_map_supported(g) && pdkv::make_attend_map(*pool, pdkv::attend_map_box(g), s->map[0]);
            }
            std::vector<Shape> shape;
            // one kernel for all own tokens (their scores are found in one way), by their average
            int64_t own = 0;
            for (int32_t n : s->len) own += n;
            s->own_tiles = tile_ok && s->n_seq > 0 && tile_is_faster(R, own / s->n_seq);
            for (size_t i = 0; i < s->segs.size(); ++i)
                // (a prefix of many rows always goes to the tile kernel, which runs beside the own tokens: 71 sequences
                // behind 49 tokens 19 us, 31 with the prefix among the own tokens)
                shape.push_back(shape_of(n_rows[i], (int32_t)i < s->n_seq ? s->own_tiles : tile_ok && n_rows[i] >= kTileMinRows));
            // unit of (row tile 0, head 0) of every segment
            std::vector<int32_t> unit0(s->segs.size(), -1);
            const std::vector<Unit> warp_units = units_of(*s, 0, n_rows, shape), tile_units = units_of(*s, 1, n_rows, shape);
            const int sms = tile_sms(*s, warp_units, tile_units);
            plan_items(*s, 1, tile_units, unit0, sms);
            plan_items(*s, 0, warp_units, unit0, pdkv::attend_ctas_per_sm(g.head_dim) * std::max(1, s->sm_count - s->n_ctas[1]));
            s->seqs.resize((size_t)s->n_seq);
            for (int32_t r = 0; r < s->n_seq; ++r) {
                AttnSeq &q = s->seqs[(size_t)r];
                q.len = s->len[(size_t)r];
                q.own_unit = unit0[(size_t)r];
                q.own_tile = shape[(size_t)r].row_tile;
                const int32_t p = d->n_prefix > 0 ? d->seq_prefix[r] : -1;
                q.prefix_unit = p >= 0 ? unit0[(size_t)(s->n_seq + p)] : -1;
                q.prefix_tile = p >= 0 ? shape[(size_t)(s->n_seq + p)].row_tile : 1;
                q.prefix_row0 = row0[(size_t)r];
                q.logit_stride = (q.len + 3) / 4 * 4;
                q.logits = s->logit_floats;
                if (!s->own_tiles) s->logit_floats += (int64_t)q.logit_stride * R * g.num_kv_heads;
                q.direct = q.own_unit >= 0 && q.prefix_unit < 0;
                if (q.direct) {   // every (row tile, head) in one part?
                    const int64_t tiles = (R + q.own_tile - 1) / q.own_tile;
                    for (int64_t u = 0; u < tiles * g.num_kv_heads; ++u)
                        if (s->units[(size_t)(q.own_unit + u)].n_parts != 1) q.direct = 0;
                }
                if (!q.direct) s->join = true;
            }
            for (const AttnUnit &u : s->units) s->most_parts = std::max(s->most_parts, u.n_parts);
            for (std::vector<AttnItem> &list : s->items)
                for (AttnItem &it : list) it.direct = it.seq >= 0 && s->seqs[(size_t)it.seq].direct;
        }

        // device arrays: one block, each list 16-byte aligned
        size_t bytes = 0;
        auto place = [&](size_t n) {
            const size_t o = bytes;
            bytes += (n + 15) / 16 * 16;
            return o;
        };
        const size_t o_status = place(16), o_tbl = place(tbl.size() * 4), o_members = place(members.size() * 4),
                     o_segs = place(s->segs.size() * sizeof(AttnSeg)), o_units = place(s->units.size() * sizeof(AttnUnit)),
                     o_seqs = place(s->seqs.size() * sizeof(AttnSeq)),
                     o_items[2] = {place(s->items[0].size() * sizeof(AttnItem)), place(s->items[1].size() * sizeof(AttnItem))};
        static_assert(sizeof(AttnItem) == 64, "an item is fetched as four vectors");
        if (needed_bytes) *needed_bytes = bytes;
        if (workspace && workspace_bytes < bytes) return PDKV_ERR_BUFFER_TOO_SMALL;
        if (!pdkv::tunables().dry_run) {
            std::vector<char> image(bytes, 0);
            auto put = [&](size_t o, const void *p, size_t n) { if (n) memcpy(image.data() + o, p, n); };
            put(o_tbl, tbl.data(), tbl.size() * 4);
            put(o_members, members.data(), members.size() * 4);
            for (int k = 0; k < 2; ++k) {
                const std::vector<AttnItem> list = chain_items(s->items[k], s->item_cta[k], s->n_ctas[k]);
                put(o_items[k], list.data(), list.size() * sizeof(AttnItem));
            }
            put(o_segs, s->segs.data(), s->segs.size() * sizeof(AttnSeg));
            put(o_units, s->units.data(), s->units.size() * sizeof(AttnUnit));
            put(o_seqs, s->seqs.data(), s->seqs.size() * sizeof(AttnSeq));
            s->dev_bytes = bytes;
            pdkv::DeviceGuard guard(s->device);
            if (guard.err != cudaSuccess) return pdkv::report_cuda_error(guard.err, "cudaSetDevice");
            if (workspace) {
                s->dev_mem = workspace;
                s->owns_dev_mem = false;
            } else {
                cudaError_t e = cudaMalloc(&s->dev_mem, bytes);
                if (e != cudaSuccess) {
                    s->dev_mem = nullptr;
                    return pdkv::report_cuda_error(e, "cudaMalloc");
                }
            }
            cudaStream_t st = static_cast<cudaStream_t>(stream);
            cudaError_t e = cudaMemcpyAsync(s->dev_mem, image.data(), bytes, cudaMemcpyHostToDevice, st);
            if (e == cudaSuccess) e = cudaStreamSynchronize(st);
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "cudaMemcpyAsync");
            char *b = static_cast<char *>(s->dev_mem);
            s->d_status = reinterpret_cast<unsigned long long *>(b + o_status);
            s->d_tbl = reinterpret_cast<const int32_t *>(b + o_tbl);
            s->d_members = reinterpret_cast<const int32_t *>(b + o_members);
            for (int k = 0; k < 2; ++k) s->d_items[k] = reinterpret_cast<const AttnItem *>(b + o_items[k]);
            s->d_segs = reinterpret_cast<const AttnSeg *>(b + o_segs);
            s->d_units = reinterpret_cast<const AttnUnit *>(b + o_units);
            s->d_seqs = reinterpret_cast<const AttnSeq *>(b + o_seqs);
        }
        hold.s = nullptr;
        *out = s;
        return PDKV_OK;
    } catch (const std::bad_alloc &) {
        return PDKV_ERR_NOMEM;
    } catch (const std::length_error &) {
        return PDKV_ERR_NOMEM;
    }
}

int pdkv_seqs_destroy(pdkv_seqs *s)
{
    if (!s) return PDKV_OK;
    int rc = PDKV_OK;
    if (s->dev_mem && s->owns_dev_mem) {
        pdkv::DeviceGuard guard(s->device);
        cudaError_t e = cudaFree(s->dev_mem);
        if (e != cudaSuccess) rc = pdkv::report_cuda_error(e, "cudaFree");
    }
    delete s;
    return rc;
}

int pdkv_seqs_status(const pdkv_seqs *s, void *stream)
{
    if (!s || !s->dev_mem) return PDKV_ERR_INVALID_ARG;
    pdkv::DeviceGuard guard(s->device);
    if (guard.err != cudaSuccess) return pdkv::report_cuda_error(guard.err, "cudaSetDevice");
    unsigned long long v = 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemcpyAsync(&v, s->d_status, sizeof v, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return pdkv::report_cuda_error(e, "cudaMemcpyAsync");
    if (v == 0) return PDKV_OK;
    // reported once: it says nothing about the calls that follow
    e = cudaMemsetAsync(s->d_status, 0, sizeof v, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return pdkv::report_cuda_error(e, "cudaMemsetAsync");
    return v == pdkv::kStatusLength ? PDKV_ERR_TABLE : PDKV_ERR_DEVICE_BOUNDS;
}

int pdkv_seqs_items(const pdkv_seqs *s, const pdkv_attend_item **items, int64_t *n_items)
{
    if (!s || !items || !n_items) return PDKV_ERR_INVALID_ARG;
    *items = s->listing.data();
    *n_items = (int64_t)s->listing.size();
    return PDKV_OK;
}

}  // extern "C"

namespace {

struct ScratchLayout {
    size_t o = 0, ml = 0, logits = 0, lse = 0, bytes = 0;
};

ScratchLayout scratch_layout(const pdkv_seqs *s, bool with_scores)
{
    ScratchLayout l;
    auto place = [&](size_t n) {
        const size_t o = l.bytes;
        l.bytes += (n + 255) / 256 * 256;
        return o;
    };
    l.o = place(s->join ? (size_t)s->part_rows * (size_t)s->pool.d.head_dim * 4 : 0);
    l.ml = place((s->join || with_scores) ? (size_t)s->part_rows * 8 : 0);
    l.logits = place(with_scores ? (size_t)s->logit_floats * 4 : 0);
    l.lse = place(with_scores && s->own_tiles ? (size_t)s->n_seq * s->q_tokens * s->Hq * 4 : 0);
    return l;
}

}  // namespace

extern "C" {

int pdkv_attend_scratch(const pdkv_seqs *s, int with_scores, size_t *bytes)
{
    if (!s || !bytes || s->Hq == 0) return PDKV_ERR_INVALID_ARG;
    *bytes = scratch_layout(s, with_scores != 0).bytes;
    return PDKV_OK;
}

}  // extern "C"

namespace {

// `f`: another form than plain causal, or null.
int attend_call(const pdkv_seqs *s, int layer, const pdkv_attend_args *a, const pdkv_attend_form *f, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!s || !a || s->Hq == 0 || layer < 0 || layer >= s->pool.d.num_layers) return PDKV_ERR_INVALID_ARG;
    const float scale_log2 = (float)((double)a->scale * 1.4426950408889634);
    if (!std::isfinite(scale_log2)) return PDKV_ERR_INVALID_ARG;
    double cap_in = 0, cap_out = 0;
    if (f) {
        if (!(f->cap >= 0.f) || !std::isfinite(f->cap)) return PDKV_ERR_INVALID_ARG;
        cap_out = f->cap * 1.4426950408889634;
        if (f->cap > 0.f) cap_in = 2 * 1.4426950408889634 * std::fabs(a->scale) / f->cap;
        if (!std::isfinite((float)cap_in) || !std::isfinite((float)(2 * cap_out)) || (f->cap > 0.f && (float)cap_out == 0.f)) return PDKV_ERR_INVALID_ARG;
        if (!aligned(f->slopes, 4) || !aligned(f->mask, 4) || !aligned(f->n_new, 4) || !aligned(f->offset, 4)) return PDKV_ERR_INVALID_ARG;
        if (f->mask && (f->mask_stride[0] < 0 || f->mask_stride[1] < 0)) return PDKV_ERR_INVALID_ARG;
        if (f->offset && f->offset_stride < 0) return PDKV_ERR_INVALID_ARG;
    }
    try {
        const int64_t rows[3] = {s->n_seq, s->q_tokens, s->Hq};
        const int64_t D = s->pool.d.head_dim;
        if (s->n_seq > 0) {
            if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16)) return PDKV_ERR_INVALID_ARG;
            for (int i = 0; i < 3; ++i)
                if (rows[i] > 1 && (a->q_stride[i] % 8 || a->out_stride[i] % 8 || a->q_stride[i] < 0)) return PDKV_ERR_INVALID_ARG;
            if (!rows_apart(D, a->out_stride, rows, 3)) return PDKV_ERR_INVALID_ARG;
        }
        if (a->lse && !aligned(a->lse, 4)) return PDKV_ERR_INVALID_ARG;
        if (a->seq_len && !aligned(a->seq_len, 4)) return PDKV_ERR_INVALID_ARG;
        const bool scores = a->scores_out != nullptr;
        if (!scores && a->scores_in) return PDKV_ERR_INVALID_ARG;
        if (scores) {
            if (!aligned(a->scores_out, 4) || !aligned(a->scores_in, 4)) return PDKV_ERR_INVALID_ARG;
            const int64_t n[2] = {s->n_seq, s->pool.d.num_kv_heads};
            if (!rows_apart(s->max_len, a->scores_out_stride, n, 2)) return PDKV_ERR_INVALID_ARG;
            if (a->scores_in) {
                const bool same = a->scores_in == a->scores_out;
                for (int i = 0; i < 2; ++i)
                    if (n[i] > 1 && (a->scores_in_stride[i] < 0 || (same && a->scores_in_stride[i] != a->scores_out_stride[i])))
                        return PDKV_ERR_INVALID_ARG;
            }
        }
        const ScratchLayout l = scratch_layout(s, scores);
        if (l.bytes && (!scratch || !aligned(scratch, 32))) return PDKV_ERR_INVALID_ARG;
        if (s->n_seq > 0) {
            // what the call writes lies apart from what it reads and from one another
            const int64_t heads[2] = {s->n_seq, s->pool.d.num_kv_heads};
            const Rows written[4] = {Rows(a->out, D, 2, a->out_stride, rows, 3), Rows(a->lse, 4 * rows[0] * rows[1] * rows[2]),
                                     Rows(a->scores_out, s->max_len, 4, a->scores_out_stride, heads, 2), Rows(scratch, (int64_t)std::min(scratch_bytes, l.bytes))};
            const Rows read[5] = {Rows(a->q, D, 2, a->q_stride, rows, 3), Rows(s->pool.base, (int64_t)pdkv_pool_bytes(&s->pool.d)),
                                  Rows(a->seq_len, 4 * rows[0]), Rows(s->dev_mem, (int64_t)s->dev_bytes),
                                  Rows(a->scores_in, s->max_len, 4, a->scores_in_stride, heads, 2)};
            for (int i = 0; i < 4; ++i) {
                for (int j = 0; j < i; ++j)
                    if (meet(written[i], written[j])) return PDKV_ERR_INVALID_ARG;
                for (int j = 0; j < 5; ++j)
                    if (!(i == 2 && j == 4 && a->scores_in == a->scores_out) && meet(written[i], read[j])) return PDKV_ERR_INVALID_ARG;
            }
            if (f) {
                const int64_t words = ((int64_t)s->q_tokens + 31) / 32;
                const Rows more[4] = {Rows(f->slopes, 4 * rows[2]), Rows(f->mask, words, 4, f->mask_stride, rows, 2), Rows(f->n_new, 4 * rows[0]),
                                      Rows(f->offset, s->q_tokens, 4, &f->offset_stride, rows, 1)};
                for (const Rows &w : written)
                    for (const Rows &r : more)
                        if (meet(w, r)) return PDKV_ERR_INVALID_ARG;
            }
        }
        if (scratch_bytes < l.bytes) return PDKV_ERR_BUFFER_TOO_SMALL;
        if (!s->dev_mem) return PDKV_ERR_INVALID_ARG;   // host-only handle
        if (s->n_seq == 0) return PDKV_OK;
        // blocks of the joining and weighing kernels: refused before anything is enqueued
        if ((double)s->n_seq * s->pool.d.num_kv_heads * ((double)s->G * s->q_tokens + 1 + (scores ? s->max_len / 128.0 + 1 : 0)) > 2e9)
            return PDKV_ERR_LIMIT;

        pdkv::AttnParams p{};
        p.pool = pdkv::pool_view(s->pool);
        p.tbl = s->d_tbl;
        p.segs = s->d_segs;
        p.units = s->d_units;
        p.seqs = s->d_seqs;
        p.members = s->d_members;
        p.items = s->d_items[0];
        p.n_ctas = s->n_ctas[0];
        p.tile_items = s->d_items[1];
        p.n_tile_ctas = s->n_ctas[1];
        p.use_map = s->use_map;
        p.map_box = pdkv::attend_map_box(s->pool.d);
        p.tile_box = pdkv::attend_tile_box(s->pool.d);
        p.map_layer_major = s->pool.d.layout == PDKV_LAYOUT_LAYER_MAJOR;
        p.status = s->d_status;
        p.n_seq = s->n_seq;
        p.H = s->pool.d.num_kv_heads;
        p.G = s->G;
        p.D = s->pool.d.head_dim;
        p.q_tokens = s->q_tokens;
        p.q = a->q;
        p.out = a->out;
        for (int i = 0; i < 3; ++i) {
            p.q_stride[i] = rows[i] > 1 ? a->q_stride[i] : 0;
            p.out_stride[i] = rows[i] > 1 ? a->out_stride[i] : 0;
        }
        p.lse = a->lse;
        p.scale_log2 = scale_log2;
        // The kernels hide tokens as logits of -infinity, which a scale of zero would turn into NaN: the smallest number
        // instead, by which no finite logit comes near 1.
        if (p.scale_log2 == 0.f) p.scale_log2 = std::copysign(std::numeric_limits<float>::denorm_min(), a->scale);
        p.seq_len = a->seq_len;
        if (f) {
            p.formed = f->slopes ? 3 : f->cap > 0.f ? 2 : 1;
            // (a factor of zero as above: the logits' infinities stay what they are)
            p.cap_in = (float)cap_in == 0.f && f->cap > 0.f ? std::numeric_limits<float>::denorm_min() : (float)cap_in;
            p.cap_out = (float)cap_out;
            // The powers of cap_in are in the terms, a product a logit less, where neither they nor z^2 leave the range of 32 bits (the last
            // term, of which a few bits are enough, is the first to do so).
            const double square = (double)p.cap_in * p.cap_in, last = pdkv::kCapTerms[4] * std::fabs(p.scale_log2) * square * square * square * square;
            const bool folded = cap_in > 1.0 / (1 << 14) && cap_in < 1 << 14 && last > 1e-40 && last < 1e36;
            p.cap_unit = folded ? 1.f : p.cap_in;
            double unit = std::fabs(p.scale_log2);
            for (int i = 0; i < 5; ++i, unit *= folded ? square : 1.0) p.cap_terms[i] = (float)(pdkv::kCapTerms[i] * unit);
            p.slopes = f->slopes;
            p.mask = f->mask;
            p.n_new = f->n_new;
            p.offset = f->offset;
            if (f->mask)
                for (int i = 0; i < 2; ++i) p.mask_stride[i] = rows[i] > 1 ? f->mask_stride[i] : 0;
            p.offset_stride = f->offset && rows[0] > 1 ? f->offset_stride : 0;
        }
        char *w = static_cast<char *>(scratch);
        p.part_o = reinterpret_cast<float *>(w + l.o);
        p.part_ml = reinterpret_cast<float *>(w + l.ml);
        if (scores) {
            p.with_scores = 1;
            if (s->own_tiles) {
                if (!p.lse) p.lse = reinterpret_cast<float *>(w + l.lse);
                for (int32_t n : s->len) p.own_tiles += (int64_t)((n + 127) / 128) * p.H;
                p.sm_count = s->sm_count;
            } else
                p.logits = reinterpret_cast<float *>(w + l.logits);
            p.scores_in = a->scores_in;
            p.scores_out = a->scores_out;
            for (int i = 0; i < 2; ++i) {
                p.scores_in_stride[i] = a->scores_in_stride[i];
                p.scores_out_stride[i] = a->scores_out_stride[i];
            }
        }
        p.max_len = s->max_len;
        p.layer = layer;
        p.block_shift = log2_of(s->pool.d.block_tokens);
        pdkv::DeviceGuard guard(s->device);
        if (guard.err != cudaSuccess) return pdkv::report_cuda_error(guard.err, "cudaSetDevice");
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        if (p.n_tile_ctas > 0) {
            const cudaError_t e = pdkv::launch_attend_tile(p, s->map[1], s->dtype, st);
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "attention tile kernel launch");
        }
        if (p.n_ctas > 0) {
            const cudaError_t e = pdkv::launch_attend(p, s->map[0], s->dtype, st);
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "attention kernel launch");
        }
        if (s->join || p.logits) {
            const cudaError_t e = pdkv::launch_attend_join(p, s->dtype, s->join, s->most_parts, st);
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "join kernel launch");
        }
        if (scores && s->own_tiles) {
            const cudaError_t e = pdkv::launch_attend_weigh(p, s->map[1], s->dtype, st);
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "weighing kernel launch");
        }
        return PDKV_OK;
    } catch (const std::bad_alloc &) {
        return PDKV_ERR_NOMEM;
    } catch (const std::length_error &) {
        return PDKV_ERR_NOMEM;
    }
}

}  // namespace

extern "C" {

int pdkv_attend(const pdkv_seqs *s, int layer, const pdkv_attend_args *a, void *scratch, size_t scratch_bytes, void *stream)
{
    return attend_call(s, layer, a, nullptr, scratch, scratch_bytes, stream);
}

int pdkv_attend_formed(const pdkv_seqs *s, int layer, const pdkv_attend_args *a, const pdkv_attend_form *f, void *scratch, size_t scratch_bytes,
                       void *stream)
{
    if (!f) return PDKV_ERR_INVALID_ARG;
    return attend_call(s, layer, a, f, scratch, scratch_bytes, stream);
}

int pdkv_evict(const pdkv_seqs *s, const pdkv_seqs *t, int layer_begin, int layer_end, const pdkv_evict_args *a, void *stream)
{
    if (!s || !t || !a || layer_begin < 0 || layer_begin > layer_end || layer_end > s->pool.d.num_layers) return PDKV_ERR_INVALID_ARG;
    if (a->sink < 0 || a->recent < 0 || a->budget < 1 || (int64_t)a->sink + a->recent > a->budget) return PDKV_ERR_INVALID_ARG;
    if (s->n_seq != t->n_seq) return PDKV_ERR_INVALID_ARG;
    const pdkv_pool_desc &x = s->pool.d, &y = t->pool.d;
    if (x.num_layers != y.num_layers || x.num_kv_heads != y.num_kv_heads || x.head_dim != y.head_dim || x.elem_bytes != y.elem_bytes)
        return PDKV_ERR_GEOMETRY;
    if (s->device != t->device) return PDKV_ERR_INVALID_ARG;
    if (!t->unique_blocks) return PDKV_ERR_TABLE;
    if (s != t) {
        if (ranges_overlap(s->pool.base, pdkv_pool_bytes(&x), t->pool.base, pdkv_pool_bytes(&y))) return PDKV_ERR_INVALID_ARG;
        for (int32_t r = 0; r < s->n_seq; ++r)
            if (t->len[(size_t)r] < std::min(s->len[(size_t)r], a->budget)) return PDKV_ERR_TABLE;
    }
    try {
        const int64_t layers = layer_end - layer_begin;
        const int64_t n[3] = {layers, s->n_seq, x.num_kv_heads};
        const int64_t top = std::min(s->max_len, a->budget);
        if (s->n_seq > 0 && layers > 0) {
            if (!a->kept || (!a->scores && s->max_len > 0)) return PDKV_ERR_INVALID_ARG;
            if (!aligned(a->scores, 4) || !aligned(a->kept, 4) || !aligned(a->kept_scores, 4) || !aligned(a->seq_len, 4) || !aligned(a->new_len, 4))
                return PDKV_ERR_INVALID_ARG;
            for (int i = 0; i < 3; ++i)
                if (n[i] > 1 && a->scores_stride[i] < 0) return PDKV_ERR_INVALID_ARG;
            const bool same = a->kept_scores && a->kept_scores == a->scores;
            if (a->kept_scores) {
                if (a->kept_scores_len < top || !rows_apart(a->kept_scores_len, a->kept_scores_stride, n, 3)) return PDKV_ERR_INVALID_ARG;
                for (int i = 0; i < 3; ++i)
                    if (same && n[i] > 1 && a->scores_stride[i] != a->kept_scores_stride[i]) return PDKV_ERR_INVALID_ARG;
            }
            // what the call writes lies apart from what it reads and from one another
            const Rows written[3] = {Rows(a->kept, 4 * layers * s->n_seq * x.num_kv_heads * a->budget), Rows(a->kept_scores, a->kept_scores_len, 4, a->kept_scores_stride, n, 3),
                                     Rows(a->new_len, 4 * (int64_t)s->n_seq)};
            const Rows read[6] = {Rows(a->scores, s->max_len, 4, a->scores_stride, n, 3), Rows(a->seq_len, 4 * (int64_t)s->n_seq),
                                  Rows(s->pool.base, (int64_t)pdkv_pool_bytes(&x)), Rows(t->pool.base, (int64_t)pdkv_pool_bytes(&y)),
                                  Rows(s->dev_mem, (int64_t)s->dev_bytes), Rows(t->dev_mem, (int64_t)t->dev_bytes)};
            for (int i = 0; i < 3; ++i) {
                for (int j = 0; j < i; ++j)
                    if (meet(written[i], written[j])) return PDKV_ERR_INVALID_ARG;
                for (int j = 0; j < 6; ++j) {
                    if ((i == 1 && j == 0 && same) || (i == 2 && j == 1 && a->new_len == a->seq_len)) continue;   // updated where they stand
                    if (meet(written[i], read[j])) return PDKV_ERR_INVALID_ARG;
                }
            }
            for (int j = 0; j < 2; ++j)   // (the moved rows)
                if (meet(read[j], read[3])) return PDKV_ERR_INVALID_ARG;
        }
        // the kernels count tokens and entries of a row in 32 bits
        if (a->budget > kMaxTokens || (a->kept_scores && a->kept_scores_len > kMaxTokens)) return PDKV_ERR_LIMIT;
        if (!s->dev_mem || !t->dev_mem) return PDKV_ERR_INVALID_ARG;   // host-only handle
        if (s->n_seq == 0 || layers == 0) return PDKV_OK;
        if ((double)layers * s->n_seq * x.num_kv_heads * 16 > 2e9) return PDKV_ERR_LIMIT;   // blocks of a kernel
        if (s->max_len > 0 || a->kept || a->new_len) {
            if (!a->kept) return PDKV_ERR_INVALID_ARG;
            pdkv::EvictParams p{};
            p.src = pdkv::pool_view(s->pool);
            p.dst = pdkv::pool_view(t->pool);
            p.src_tbl = s->d_tbl;
            p.dst_tbl = t->d_tbl;
            p.src_segs = s->d_segs;
            p.dst_segs = t->d_segs;
            p.n_seq = s->n_seq;
            p.H = x.num_kv_heads;
            p.row_bytes = x.head_dim * x.elem_bytes;
            p.layer_begin = layer_begin;
            p.n_layers = (int32_t)layers;
            p.in_place = s == t;
            p.budget = a->budget;
            p.sink = a->sink;
            p.recent = a->recent;
            p.seq_len = a->seq_len;
            p.scores = a->scores;
            p.kept = a->kept;
            p.kept_scores = a->kept_scores;
            p.kept_scores_len = a->kept_scores_len;
            p.new_len = a->new_len;
            for (int i = 0; i < 3; ++i) {
                p.scores_stride[i] = n[i] > 1 ? a->scores_stride[i] : 0;
                p.kept_scores_stride[i] = n[i] > 1 ? a->kept_scores_stride[i] : 0;
            }
            p.max_len = s->max_len;
            p.vec_bytes = aligned(p.src.base, 32) && aligned(p.dst.base, 32) ? 32 : 16;
            while (p.vec_bytes > 1 && p.row_bytes % p.vec_bytes) p.vec_bytes /= 2;
            p.src_shift = log2_of(x.block_tokens);
            p.dst_shift = log2_of(y.block_tokens);
            pdkv::DeviceGuard guard(s->device);
            if (guard.err != cudaSuccess) return pdkv::report_cuda_error(guard.err, "cudaSetDevice");
            const cudaError_t e = pdkv::launch_evict(p, s->sm_count, static_cast<cudaStream_t>(stream));
            if (e != cudaSuccess) return pdkv::report_cuda_error(e, "eviction kernel launch");
        }
        return PDKV_OK;
    } catch (const std::bad_alloc &) {
        return PDKV_ERR_NOMEM;
    } catch (const std::length_error &) {
        return PDKV_ERR_NOMEM;
    }
}

}  // extern "C"
