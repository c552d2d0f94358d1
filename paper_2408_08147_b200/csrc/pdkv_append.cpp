// Entry points of the calls that put tokens into a filled pool and settle drafted ones: checks on the host, then one launch.
#include <cmath>
#include <new>
#include <stdexcept>

#include "pdkv_append.h"
#include "pdkv_checks.h"

using pdkv::aligned;
using pdkv::log2_of;
using pdkv::meet;
using pdkv::Rows;
using pdkv::rows_apart;
using pdkv::touches;

namespace {

bool rows_meet(const Rows &a, const Rows &b) { return !apart_in_token(a, b) && meet(a, b); }

}  // namespace

extern "C" {

int pdkv_rotary_turns(const double *radians, int n, uint64_t *turns)
{
    if (n < 0 || (n > 0 && (!radians || !turns))) return PDKV_ERR_INVALID_ARG;
    constexpr long double kTurn = 6.283185307179586476925286766559005768L;
    for (int i = 0; i < n; ++i)
        if (!std::isfinite(radians[i])) return PDKV_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        long double t = (long double)radians[i] / kTurn;
        t -= std::floor(t);
        // (a fraction that rounds up to a whole turn is none)
        const long double x = std::floor(t * 18446744073709551616.0L + 0.5L);
        turns[i] = x >= 18446744073709551616.0L ? 0 : (uint64_t)x;
    }
    return PDKV_OK;
}

int pdkv_append(const pdkv_seqs *s, int layer, const pdkv_append_args *a, void *stream)
{
    if (!s || !a || layer < 0 || layer >= s->pool.d.num_layers) return PDKV_ERR_INVALID_ARG;
    const pdkv_pool_desc &g = s->pool.d;
    if (s->dtype != PDKV_DTYPE_BF16 && s->dtype != PDKV_DTYPE_FP16) return PDKV_ERR_INVALID_ARG;
    if (g.elem_bytes != 2 || g.head_dim % 8 || g.head_dim > 256 || !aligned(s->pool.base, 16)) return PDKV_ERR_GEOMETRY;
    if (a->rows < 0 || (a->q && s->Hq == 0) || (a->q == nullptr) != (a->q_out == nullptr)) return PDKV_ERR_INVALID_ARG;
    if (a->row_begin && a->n_new) return PDKV_ERR_INVALID_ARG;
    if (!a->row_begin && (s->n_seq ? a->rows % s->n_seq : a->rows) != 0) return PDKV_ERR_INVALID_ARG;
    if ((a->q_norm || a->k_norm) && !(a->norm_eps >= 0.f && std::isfinite(a->norm_eps))) return PDKV_ERR_INVALID_ARG;
    const pdkv_rotary &r = a->rotary;
    if (r.dims < 0 || r.dims % 2 || r.dims > g.head_dim) return PDKV_ERR_INVALID_ARG;
    if (r.dims > 0 && (!r.turns || !aligned(r.turns, 8) || r.n_axes < 1 || !std::isfinite(r.scale) || (r.adjacent != 0 && r.adjacent != 1) ||
                       (r.n_axes > 1 && (!a->position || !r.axis || a->position_stride < a->rows))))
        return PDKV_ERR_INVALID_ARG;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->q_out, 16) || !aligned(a->q_norm, 16) || !aligned(a->k_norm, 16) ||
        !aligned(a->row_begin, 4) || !aligned(a->n_new, 4) || !aligned(a->seq_len, 4) || !aligned(a->position, 4))
        return PDKV_ERR_INVALID_ARG;
    try {
        const int64_t D = g.head_dim, H = g.num_kv_heads, Hq = a->q ? s->Hq : 0, n_seq = a->row_begin ? 1 : s->n_seq;
        const int64_t per = n_seq > 0 ? a->rows / n_seq : 0;
        const int64_t nq[3] = {n_seq, per, Hq}, nk[3] = {n_seq, per, H};
        if (a->rows > 0) {
            if (!a->k || !a->v) return PDKV_ERR_INVALID_ARG;
            const int64_t *stride[4] = {a->q_stride, a->q_out_stride, a->k_stride, a->v_stride};
            for (int x = Hq > 0 ? 0 : 2; x < 4; ++x)
                for (int i = 0; i < 3; ++i)
                    if ((x < 2 ? nq : nk)[i] > 1 && (stride[x][i] % 8 || stride[x][i] < 0)) return PDKV_ERR_INVALID_ARG;
            // what the call writes (queries, the pool) lies apart from what it reads and from one another
            const Rows pool(s->pool.base, (int64_t)pdkv_pool_bytes(&g)), k(a->k, D, 2, a->k_stride, nk, 3), v(a->v, D, 2, a->v_stride, nk, 3);
            const Rows q(a->q, D, 2, a->q_stride, nq, 3), q_out(a->q_out, D, 2, a->q_out_stride, nq, 3);
            const Rows small[9] = {Rows(a->row_begin, 4 * ((int64_t)s->n_seq + 1)), Rows(a->n_new, 4 * (int64_t)s->n_seq), Rows(a->seq_len, 4 * (int64_t)s->n_seq),
                                   Rows(r.dims > 0 ? a->position : nullptr, 4 * ((r.n_axes - 1) * a->position_stride + a->rows)), Rows(a->q_norm, 4 * D), Rows(a->k_norm, 4 * D),
                                   Rows(r.dims > 0 ? r.turns : nullptr, 4 * (int64_t)r.dims), Rows(r.dims > 0 && r.n_axes > 1 ? r.axis : nullptr, r.dims / 2),
                                   Rows(s->dev_mem, (int64_t)s->dev_bytes)};
            if (touches(pool, k) || touches(pool, v) || touches(pool, q) || touches(pool, q_out)) return PDKV_ERR_INVALID_ARG;
            if (Hq > 0) {
                if (!rows_apart(D, a->q_out_stride, nq, 3)) return PDKV_ERR_INVALID_ARG;
                bool same = a->q == a->q_out;   // where they stand
                for (int i = 0; i < 3; ++i) same = same && (nq[i] <= 1 || a->q_stride[i] == a->q_out_stride[i]);
                if (rows_meet(q_out, k) || rows_meet(q_out, v) || (!same && rows_meet(q_out, q))) return PDKV_ERR_INVALID_ARG;
            }
            for (const Rows &x : small)
                if (touches(pool, x) || touches(x, q_out)) return PDKV_ERR_INVALID_ARG;
        }
        // (well inside what a launch takes)
        if ((double)a->rows * ((double)Hq + 2.0 * (double)H) / 4 > 2e9) return PDKV_ERR_LIMIT;
        if (!s->dev_mem) return PDKV_ERR_INVALID_ARG;   // host-only handle
        if (s->n_seq == 0 || a->rows == 0) return PDKV_OK;
        pdkv::AppendParams p{};
        p.pool = pdkv::pool_view(s->pool);
        p.tbl = s->d_tbl;
        p.segs = s->d_segs;
        p.layer = layer;
        p.n_seq = s->n_seq;
        p.Hq = (int32_t)Hq;
        p.H = (int32_t)H;
        p.D = (int32_t)D;
        p.rows = a->rows;
        p.per = (int32_t)per;
        p.row_begin = a->row_begin;
        p.n_new = a->n_new;
        p.seq_len = a->seq_len;
        p.q = a->q;
        p.k = a->k;
        p.v = a->v;
        p.q_out = a->q_out;
        for (int i = 0; i < 3; ++i) {
            p.q_stride[i] = nq[i] > 1 ? a->q_stride[i] : 0;
            p.q_out_stride[i] = nq[i] > 1 ? a->q_out_stride[i] : 0;
            p.k_stride[i] = nk[i] > 1 ? a->k_stride[i] : 0;
            p.v_stride[i] = nk[i] > 1 ? a->v_stride[i] : 0;
        }
        p.q_norm = a->q_norm;
        p.k_norm = a->k_norm;
        p.eps = a->norm_eps;
        p.rotated = r.dims;
        p.adjacent = r.adjacent;
        p.axes = r.n_axes;
        p.turns = r.turns;
        p.axis = r.n_axes > 1 ? r.axis : nullptr;
        p.rotary_scale = r.scale;
        p.position = a->position;
        p.position_stride = a->position_stride;
        p.block_shift = log2_of(g.block_tokens);
        p.status = s->d_status;
        pdkv::DeviceGuard guard(s->device);
        if (guard.err != cudaSuccess) return pdkv::report_cuda_error(guard.err, "cudaSetDevice");
        const cudaError_t e = pdkv::launch_append(p, s->dtype, s->sm_count, static_cast<cudaStream_t>(stream));
        return e == cudaSuccess ? PDKV_OK : pdkv::report_cuda_error(e, "append kernel launch");
    } catch (const std::bad_alloc &) {
        return PDKV_ERR_NOMEM;
    } catch (const std::length_error &) {
        return PDKV_ERR_NOMEM;
    }
}

int pdkv_accept(const pdkv_seqs *s, int layer_begin, int layer_end, const pdkv_accept_args *a, void *stream)
{
    if (!s || !a || layer_begin < 0 || layer_begin >= layer_end || layer_end > s->pool.d.num_layers) return PDKV_ERR_INVALID_ARG;
    if (a->path_len < 0 || a->new_tokens < 0 || a->path_stride < 0 || (a->path_len > 0 && !a->path && s->n_seq > 0)) return PDKV_ERR_INVALID_ARG;
    if (!aligned(a->path, 4) || !aligned(a->n_new, 4) || !aligned(a->seq_len, 4) || !aligned(a->new_len, 4)) return PDKV_ERR_INVALID_ARG;
    try {
        const pdkv_pool_desc &g = s->pool.d;
        const int64_t n = s->n_seq;
        const Rows pool(n > 0 ? s->pool.base : nullptr, (int64_t)pdkv_pool_bytes(&g)), new_len(a->new_len, 4 * n);
        const Rows read[4] = {Rows(a->path_len > 0 ? a->path : nullptr, a->path_len, 4, &a->path_stride, &n, 1), Rows(a->n_new, 4 * n), Rows(a->seq_len, 4 * n),
                              Rows(s->dev_mem, (int64_t)s->dev_bytes)};
        for (int i = 0; i < 4; ++i) {
            if (touches(pool, read[i])) return PDKV_ERR_INVALID_ARG;
            if (!(i == 2 && a->new_len == a->seq_len) && touches(new_len, read[i])) return PDKV_ERR_INVALID_ARG;
        }
        if (touches(pool, new_len)) return PDKV_ERR_INVALID_ARG;
        int32_t vec = 16, row_bytes = g.head_dim * g.elem_bytes;
        while (vec > 1 && (row_bytes % vec || !aligned(s->pool.base, (size_t)vec))) vec /= 2;
        // (blocks along one axis of a launch)
        if ((int64_t)(row_bytes / vec) * g.num_kv_heads * 2 * (layer_end - layer_begin) > (int64_t)65535 * 128) return PDKV_ERR_LIMIT;
        if (!s->dev_mem) return PDKV_ERR_INVALID_ARG;   // host-only handle
        if (n == 0) return PDKV_OK;
        pdkv::AcceptParams p{};
        p.pool = pdkv::pool_view(s->pool);
        p.tbl = s->d_tbl;
        p.segs = s->d_segs;
        p.n_seq = s->n_seq;
        p.H = g.num_kv_heads;
        p.row_bytes = row_bytes;
        p.lc_begin = 2 * layer_begin;
        p.n_lc = 2 * (layer_end - layer_begin);
        p.path = a->path;
        p.path_stride = a->path_stride;
        p.path_len = a->path_len;
        p.new_tokens = a->new_tokens;
        p.n_new = a->n_new;
        p.seq_len = a->seq_len;
        p.new_len = a->new_len;
        p.vec_bytes = vec;
        p.block_shift = log2_of(g.block_tokens);
        p.status = s->d_status;
        pdkv::DeviceGuard guard(s->device);
        if (guard.err != cudaSuccess) return pdkv::report_cuda_error(guard.err, "cudaSetDevice");
        const cudaError_t e = pdkv::launch_accept(p, static_cast<cudaStream_t>(stream));
        return e == cudaSuccess ? PDKV_OK : pdkv::report_cuda_error(e, "accept kernel launch");
    } catch (const std::bad_alloc &) {
        return PDKV_ERR_NOMEM;
    } catch (const std::length_error &) {
        return PDKV_ERR_NOMEM;
    }
}

}  // extern "C"
