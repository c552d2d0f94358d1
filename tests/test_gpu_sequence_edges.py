"""Corners of attention, accumulated weights and eviction on the GPU."""
import numpy as np
import pytest
import torch

from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200.sequences import CacheSession, Sequences
from paper_2408_08147_b200.workloads import BLOCK_MAJOR, LAYER_MAJOR, Geometry
from test_gpu_sequences import Evict, Setup, check, check_scores, logit_error

pytestmark = pytest.mark.gpu


def not_given_away(make):
    """The memory of the tensors that `make` gives up is not handed out while the stream that uses it is busy."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)    # half a second
    mine = make(side)
    lost = [(t.data_ptr(), t.numel() * t.element_size()) for t in mine]
    assert all(n > 0 for _, n in lost)
    del mine
    fresh = [torch.empty(n, dtype=torch.uint8, device="cuda") for _, n in lost for _ in range(50)]
    busy = not side.query()
    again = [a for a, n in lost if any(t.data_ptr() < a + n and a < t.data_ptr() + t.numel() for t in fresh)]
    side.synchronize()
    assert busy and not again


def test_outputs_of_attention_on_another_stream():
    s = Setup([300, 40], G=4, D=64)
    with s.session() as c:
        c.attend(s.layer, s.q_t)
        torch.cuda.synchronize()
        not_given_away(lambda side: c.attend(s.layer, s.q_t, stream=side.cuda_stream))


def test_outputs_of_a_session_with_a_stream_of_its_own():
    s = Setup([300, 40], G=4, D=64)
    side = torch.cuda.Stream()
    with s.session(stream=side.cuda_stream) as c:
        c.attend(s.layer, s.q_t)
        torch.cuda.synchronize()

        def make(other):
            side.wait_stream(other)
            out = c.attend(s.layer, s.q_t)
            other.wait_stream(side)
            return out

        not_given_away(make)


@pytest.mark.parametrize("with_scores", [False, True])
def test_scratch_used_on_another_stream(with_scores):
    """The session's scratch, allocated on the current stream and used on another one."""
    s = Setup([3000, 40], H=1, G=4, D=64)
    scores = torch.zeros(2, 1, 3000, device="cuda") if with_scores else None
    out, lse = torch.empty_like(s.q_t), torch.empty(s.q_t.shape[:3], device="cuda")
    with s.session() as c:
        def make(side):
            c.attend(s.layer, s.q_t, out_t=out, lse_t=lse, scores_t=scores, stream=side.cuda_stream)
            scratch = [t for t in c._scratch if t is not None]
            c._scratch = [None, None]
            return scratch

        c.attend(s.layer, s.q_t, out_t=out, lse_t=lse, scores_t=scores)
        torch.cuda.synchronize()
        not_given_away(make)


def test_outputs_of_eviction_on_another_stream():
    e = Evict([100, 50], 30)
    src_t, dst_t = e.tensors()
    scores = torch.from_numpy(e.scores).cuda()
    with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(e.dst, dst_t, e.dst_seqs) as b:
        a.evict(b, scores, 30)
        torch.cuda.synchronize()
        not_given_away(lambda side: a.evict(b, scores, 30, stream=side.cuda_stream))


@pytest.mark.parametrize("G", [2, 40])                  # warp kernel, tile kernel
@pytest.mark.parametrize("below", [11.0, 14.0, 17.0, 18.5])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_many_light_tokens_beside_a_heavy_one(dtype, below, G):
    """A heavy token without a value before 40000 tokens that lie `below` nats under it and have a value of one.  Many
    sequences share the blocks, so that no list is cut: all tokens meet the heavy one's base."""
    n, D, n_seq = 40000, 64, 320
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    geom = Geometry(LAYER_MAJOR, 1, 1, D, 2, 64, n // 64)
    pool = torch.zeros(geom.shape(), dtype=dt, device="cuda")     # [layer][K/V][block][head][token][dim]
    pool[0, 0, :, 0, :, 0] = -2 * below                           # q 4, scale 1/8: logits of -below (exact in both types)
    pool[0, 1] = 1.0
    pool[0, :, 0, 0, 5] = 0.0
    q = torch.zeros(n_seq, 1, G, D, dtype=dt, device="cuda")
    q[..., 0] = 4.0
    light = (n - 1) * np.exp(-below)
    want = light / (1 + light)
    seqs = Sequences([n] * n_seq, n // 64 * np.arange(n_seq + 1), np.tile(np.arange(n // 64), n_seq))
    with CacheSession(geom, pool, seqs, num_q_heads=G, dtype=dt) as c:
        items = c.items()
        assert set(items["kernel"]) == {1 if G == 40 else 0} and items["tok_end"].max() > 20000
        out, _ = c.attend(0, q)
    # A light weight is rounded once, by half a step, and fp16 loses 2^-32 of the heaviest weight at most; logits are exact but
    # for 4 roundings of 18.5 nats (2^-24 each) and the exponential (2^-22); sums of n terms in 32 bits (the tensor cores cut: 2^-23
    # of the sum each, in steps of 16 tokens); the result is rounded once more.
    half = torch.finfo(dt).eps / 2
    tol = 1.01 * want * (2 * half + 4 * 18.5 * 2.0 ** -23 + 2.0 ** -22 + 2 * (n / 16 + 64) * 2.0 ** -23) + n * 2.0 ** -32 + 2.0 ** -25
    off = (out.double() - want).abs().max().item()
    assert off <= tol


def cached_row(s, r, token, kv, head):
    """A row of K or V in the pool of a Setup."""
    b, tt = int(s.seqs.tbl[s.seqs.tbl_off[r] + token // s.block]), token % s.block
    return s.pool_t[b, s.layer, kv, tt, head] if s.layout == BLOCK_MAJOR else s.pool_t[s.layer, kv, b, head, tt]


def kernel_of_own_tokens(c):
    items = c.items()
    kernels = set(items["kernel"][items["seq"] >= 0].tolist())
    assert len(kernels) == 1
    return kernels.pop()


def check_where_finite(s, out_t, want):
    """Infinite and NaN where the definition is, close to it elsewhere (the tolerance of test_attention with one more rounding of the result;
    magnitudes and the largest value are those of the dims that are finite)."""
    out, _, _, e = want
    got = out_t.double().cpu().numpy()
    fin = np.isfinite(out)
    assert (np.isfinite(got) == fin).all() and (np.isnan(got) == np.isnan(out)).all()
    assert (got[np.isinf(out)] == out[np.isinf(out)]).all()
    half = torch.finfo(s.dtype).eps / 2
    rel = 2 * logit_error(e, s.D) + half + (e["n"] + 64) * 2.0 ** -23
    pool = s.pool_t.double()
    v_max = pool[torch.isfinite(pool)].abs().max().item()
    with np.errstate(invalid="ignore"):
        tol = 1.01 * (rel[..., None] * e["mag"] + 2 * half * np.abs(out)) + (e["n"][..., None] * 2.0 ** -32 * v_max + 2.0 ** -25 if s.dtype == torch.float16 else 0)
    assert (np.abs(got[fin] - out[fin]) <= tol[fin]).all()


HIDDEN = [   # kernel, then the shape
    (0, dict(lens=[90, 33, 2], G=2, Q=4, D=64)),
    (0, dict(lens=[90, 33], G=2, Q=4, D=80, block=7)),
    (0, dict(lens=[90, 33], G=4, Q=8, D=128, block=24, dtype="fp16")),
    (0, dict(lens=[90, 33], G=3, Q=40, D=192, layout=LAYER_MAJOR)),
    (0, dict(lens=[90, 260], G=16, Q=4, D=256, layout=LAYER_MAJOR)),
    (0, dict(lens=[3000], H=1, G=2, Q=4, D=128, block=32)),
    (1, dict(lens=[700, 500], G=12, Q=4, D=64, layout=LAYER_MAJOR)),
    (1, dict(lens=[700, 500], G=50, Q=4, D=128, dtype="fp16")),
    (1, dict(lens=[700, 300], H=1, G=1, Q=200, D=96)),
    (1, dict(lens=[400, 290], H=2, G=2, Q=140, D=72, block=8, prefix_len=[70], member=[0, -1])),
]


@pytest.mark.parametrize("scale", [1, -1])
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("kernel,kw", HIDDEN, ids=[str(i) for i in range(len(HIDDEN))])
def test_values_that_a_query_does_not_see(kernel, kw, value, scale):
    """The newest tokens have infinite and NaN values: queries before them are not touched, queries that see them are."""
    s = Setup(q_scale=0.5, **kw)
    for r, n in enumerate(s.lens):
        for back, d in ((1, 0), (2, 5), (3, 9), (s.Q - 1, 30), (s.Q // 2, 60)):
            if back <= n:
                row = cached_row(s, r, n - back, 1, back % s.H)
                row[d], row[d + 1] = value, -value
    scores = torch.zeros(len(s.lens), s.H, max(s.lens), device="cuda")
    scale *= s.D ** -0.5
    with s.session() as c:
        assert kernel_of_own_tokens(c) == kernel
        with np.errstate(invalid="ignore"):
            want = s.expect(scale=scale)
        assert not np.isfinite(want[0][:, -1]).all() and np.isfinite(want[0][:, 0]).all()
        check_where_finite(s, c.attend(s.layer, s.q_t, scale=scale)[0], want)
        check_where_finite(s, c.attend(s.layer, s.q_t, scale=scale, scores_t=scores)[0], want)
        c.status()
    assert torch.isfinite(scores).all()


@pytest.mark.parametrize("G,Q", [(2, 2), (12, 3), (33, 1), (50, 6)])
def test_weights_of_a_key_that_no_row_heeds(G, Q):
    """A key of infinite length whose logits are all -infinity has no weight, however many rows fill a block of the kernel."""
    s = Setup([700, 260], H=1, G=G, Q=Q, D=64, block=32)
    s.q_t[..., 0] = -s.q_t[..., 0].abs() - 0.1
    cached_row(s, 0, 300, 0, 0)[0] = float("inf")
    before = np.random.default_rng(2).random((2, 1, 700)).astype(np.float32)
    scores = torch.from_numpy(before).cuda()
    with s.session() as c:
        assert kernel_of_own_tokens(c) == (G * Q > 32)
        out, lse = c.attend(s.layer, s.q_t, scores_t=scores)
        c.status()
    want = s.expect()
    check(s, out, lse, want)
    check_scores(s, before.astype(np.float64), scores, want, s.lens)
    assert scores[0, 0, 300].item() == before[0, 0, 300]


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-37])
@pytest.mark.parametrize("G", [2, 40])                  # warp kernel, tile kernel
def test_scale_of_zero_and_large_products(G, scale):
    """Products of 1e36: with a scale of zero all tokens weigh the same; a small scale is not taken for zero."""
    s = Setup([700], H=1, G=G, D=64)
    s.q_t[..., 0] = 2.0 ** 60
    for t in range(700):
        cached_row(s, 0, t, 0, 0)[0] = 2.0 ** 60 * (-1) ** t * (1 + t % 3)
    scores = torch.zeros(1, 1, 700, device="cuda")
    with s.session() as c:
        assert kernel_of_own_tokens(c) == (G == 40)
        out, lse = c.attend(s.layer, s.q_t, scale=scale, scores_t=scores)
    want = s.expect(scale=scale)
    check(s, out, lse, want)
    check_scores(s, np.zeros((1, 1, 700)), scores, want, s.lens)


def test_an_error_is_reported_once():
    """A kernel's report, as a write to the handle's status word (the first of its workspace)."""
    s = Setup([90, 33], G=2, D=64)
    workspace = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    with s.session(workspace_t=workspace) as c:
        c.status()
        workspace[0] = 1
        with pytest.raises(B.PdkvError) as e:
            c.status()
        assert e.value.status == B.PDKV_ERR_DEVICE_BOUNDS
        check(s, *c.attend(s.layer, s.q_t), s.expect())
        c.status()


# ---------------------------------------------------------------------------
# paths that only some shapes take
# ---------------------------------------------------------------------------

LARGE = [   # own tokens in the tile kernel: one row tile, two, several items of 256 rows, heads of 72 to 128 dims
    dict(lens=[700, 500], G=12, Q=4, D=64),
    dict(lens=[700, 333], G=50, Q=4, D=128, layout=LAYER_MAJOR, dtype="fp16"),
    dict(lens=[700, 130], H=1, G=8, Q=40, D=64),                          # 320 rows: 256 and 64
    dict(lens=[700, 290], H=1, G=7, Q=43, D=128, block=24),               # 301 rows: the last group is no multiple of 16
    dict(lens=[600, 400], H=1, G=5, Q=110, D=72, block=8, layout=LAYER_MAJOR),   # 550 rows: three groups
    dict(lens=[900, 260, 700], H=2, G=20, Q=2, D=96, prefix_len=[300], member=[0, -1, 0]),
]
FEW = [     # own tokens in the warp kernel
    dict(lens=[90, 33], G=4, D=64),
    dict(lens=[90, 200], G=4, Q=6, D=128, block=24, dtype="fp16"),
    dict(lens=[300, 190], H=1, G=10, Q=9, D=256),                         # 90 rows: items behind the first row tile
    dict(lens=[130, 60], H=2, G=7, Q=20, D=80, block=7),                  # 140 rows, a block size without boxes
    dict(lens=[500, 60], H=1, G=20, Q=10, D=192, layout=LAYER_MAJOR, dtype="fp16", prefix_len=[150], member=[0, 0]),
]
ALL = [(1, kw) for kw in LARGE] + [(0, kw) for kw in FEW]
ids = [f"tile{i}" for i in range(len(LARGE))] + [f"warp{i}" for i in range(len(FEW))]


def scores_like(s, width=None, seed=1):
    host = np.random.default_rng(seed).random((len(s.lens), s.H, width or max(s.caps))).astype(np.float32)
    return host.astype(np.float64), torch.from_numpy(host).cuda()


@pytest.mark.parametrize("scale", [None, -0.2, 0.0])
@pytest.mark.parametrize("kernel,kw", ALL, ids=ids)
def test_scores_and_scales(kernel, kw, scale):
    s = Setup(**kw)
    before, scores = scores_like(s)
    want = s.expect(scale=scale)
    with s.session() as c:
        assert kernel_of_own_tokens(c) == kernel
        check(s, *c.attend(s.layer, s.q_t, scale=scale), want)
        check(s, *c.attend(s.layer, s.q_t, scale=scale, scores_t=scores), want)
        c.status()
    check_scores(s, before, scores, want, s.lens)


@pytest.mark.parametrize("kernel,kw", ALL, ids=ids)
def test_current_lengths_of_all_kinds(kernel, kw):
    """Lengths from the device below the handle's, down to none and to fewer than query tokens; NaN behind them in the pool."""
    full = kw["lens"]
    for lens in ([n - 1 - 127 * i for i, n in enumerate(full)], [n // 3 for n in full], [0] + full[1:], [kw.get("Q", 1) - 1] * len(full), [1] * len(full)):
        lens = [max(0, n) for n in lens]
        s = Setup(**{**kw, "lens": lens, "caps": full})
        lens_t = torch.tensor([n if n else -3 for n in lens], dtype=torch.int32, device="cuda")
        before, scores = scores_like(s)
        other = torch.full_like(scores, 7.0)
        want = s.expect()
        with s.session() as c:
            assert kernel_of_own_tokens(c) == kernel
            check(s, *c.attend(s.layer, s.q_t, seq_len_t=lens_t), want)
            c.attend(s.layer, s.q_t, seq_len_t=lens_t, scores_t=other, scores_in_t=scores)
            check(s, *c.attend(s.layer, s.q_t, seq_len_t=lens_t, scores_t=scores), want)
            c.status()
        check_scores(s, before, scores, want, s.lens)
        assert torch.equal(other, scores)


@pytest.mark.parametrize("kernel,kw", ALL, ids=ids)
def test_strides_of_all_kinds(kernel, kw):
    """q, out and scores as views in other orders, of wider buffers."""
    s = Setup(**kw)
    n, Q, Hq, D = s.q_t.shape
    q = torch.zeros(Q, n, Hq + 5, D + 8, dtype=s.dtype, device="cuda").permute(1, 0, 2, 3)[:, :, 2:2 + Hq, :D]
    q.copy_(s.q_t)
    out = torch.full((Hq, n, Q, D + 16), 9.0, dtype=s.dtype, device="cuda")
    view = out.permute(1, 2, 0, 3)[..., 8:8 + D]
    before, dense = scores_like(s, max(s.caps) + 5)
    both = torch.full((2, s.H, n, max(s.caps) + 5), 7.0, device="cuda")
    both[0] = dense.transpose(0, 1)
    want = s.expect()
    with s.session() as c:
        _, lse = c.attend(s.layer, q, out_t=view, scores_in_t=both[0].transpose(0, 1), scores_t=both[1].transpose(0, 1))
        c.status()
    check(s, view, lse, want)
    assert (out[..., :8] == 9).all() and (out[..., 8 + D:] == 9).all()
    got = both[1].transpose(0, 1)
    assert (got[..., -5:] == 7).all() and torch.equal(both[0].transpose(0, 1), dense)
    check_scores(s, before[..., :-5], got[..., :-5], want, s.lens)


@pytest.mark.parametrize("one_q", [False, True])
@pytest.mark.parametrize("kernel,kw", ALL, ids=ids)
def test_scores_without_an_input(kernel, kw, one_q):
    """scores_in NULL stands for zeros: tokens past a sequence's end get them, entries behind the longest sequence are left.  And q
    with strides of zero: one query for all."""
    s = Setup(**kw)
    if one_q:
        s.q_t = s.q_t[:1, :1, :1].expand_as(s.q_t)
    width = max(s.lens) + 3
    scores = torch.full((len(s.lens), s.H, width), 7.0, device="cuda")
    want = s.expect(q_t=s.q_t)
    with s.session() as c:
        out, lse = torch.empty(s.q_t.shape, dtype=s.dtype, device="cuda"), torch.empty(s.q_t.shape[:3], device="cuda")
        scratch = torch.empty(c.scratch_bytes(True), dtype=torch.uint8, device="cuda")
        a = B.pdkv_attend_args(q=s.q_t.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), scale=s.D ** -0.5, scores_out=scores.data_ptr())
        a.q_stride[:], a.out_stride[:], a.scores_out_stride[:] = s.q_t.stride()[:3], out.stride()[:3], scores.stride()[:2]
        torch.cuda.synchronize()
        B.pdkv_attend(c.handle, s.layer, a, scratch.data_ptr(), scratch.numel(), torch.cuda.current_stream().cuda_stream)
        c.status()
    check(s, out, lse, want)
    assert (scores[..., -3:] == 7).all()
    check_scores(s, np.zeros((len(s.lens), s.H, width - 3)), scores[..., :-3], want, s.lens)


def test_lse_is_optional():
    for kernel, kw in ALL[::3]:
        s = Setup(**kw)
        before, scores = scores_like(s)
        with s.session() as c:
            want = c.attend(s.layer, s.q_t)[0]
            out = torch.empty_like(want)
            scratch = torch.empty(c.scratch_bytes(True), dtype=torch.uint8, device="cuda")
            a = B.pdkv_attend_args(q=s.q_t.data_ptr(), out=out.data_ptr(), scale=s.D ** -0.5, scores_in=scores.data_ptr(), scores_out=scores.data_ptr())
            a.q_stride[:], a.out_stride[:] = s.q_t.stride()[:3], out.stride()[:3]
            a.scores_in_stride[:], a.scores_out_stride[:] = scores.stride()[:2], scores.stride()[:2]
            torch.cuda.synchronize()
            B.pdkv_attend(c.handle, s.layer, a, scratch.data_ptr(), scratch.numel(), torch.cuda.current_stream().cuda_stream)
            c.status()
        assert torch.equal(out, want)
        check_scores(s, before, scores, s.expect(), s.lens)


@pytest.mark.parametrize("kernel,kw", ALL, ids=ids)
def test_the_same_bits_from_a_graph_beside_another(kernel, kw):
    """Two recorded calls with a scratch each, replayed at once on two streams, again and again."""
    s = Setup(**kw)
    with s.session() as c:
        q = [s.q_t, (s.q_t * 0.5)]
        zero = torch.zeros(len(s.lens), s.H, max(s.caps), device="cuda")
        sc = [zero.clone() for _ in q]
        want = [c.attend(s.layer, x, scores_t=y)[0].clone() for x, y in zip(q, sc)]
        want_sc = [x.clone() for x in sc]
        out = [torch.empty_like(x) for x in want]
        lse = [torch.empty(s.q_t.shape[:3], device="cuda") for _ in q]
        scratch = [torch.empty(c.scratch_bytes(True), dtype=torch.uint8, device="cuda") for _ in q]
        streams, graphs = [torch.cuda.Stream() for _ in q], []
        torch.cuda.synchronize()
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[i]):
                for _ in range(5):
                    c.attend(s.layer, q[i], out_t=out[i], lse_t=lse[i], scores_t=sc[i], scores_in_t=zero, scratch_t=scratch[i])
            graphs.append(g)
        for _ in range(5):
            for x in out + sc:
                x.zero_()
            torch.cuda.synchronize()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out + sc, want + want_sc))
        c.status()


def test_on_the_streams_of_an_sm_partition():
    """Attention and eviction on few SMs and on the others."""
    part = B.pdkv_sm_partition_create(0, 8)
    try:
        for which in (0, 1):
            stream = torch.cuda.ExternalStream(B.pdkv_sm_partition_stream(part, which))
            for kernel, kw in ALL[::4]:
                s = Setup(**kw)
                before, scores = scores_like(s)
                out, lse = torch.empty_like(s.q_t), torch.empty(s.q_t.shape[:3], device="cuda")
                with s.session() as c:
                    c.attend(s.layer, s.q_t, out_t=out, lse_t=lse)
                    scratch = torch.empty(c.scratch_bytes(True), dtype=torch.uint8, device="cuda")
                    torch.cuda.synchronize()
                    c.attend(s.layer, s.q_t, out_t=out, lse_t=lse, scores_t=scores, scratch_t=scratch, stream=stream.cuda_stream)
                    c.status(stream.cuda_stream)
                want = s.expect()
                check(s, out, lse, want)
                check_scores(s, before, scores, want, s.lens)
            for kw in (dict(lens=[300, 50], budget=64), dict(lens=[20000, 9000], budget=2049, H=1, layers=1)):
                e = Evict(**kw)
                src_t, dst_t = e.tensors()
                want_kept, want_sc, want_pool = e.expect(0, 0, (0, e.layers))
                scores = torch.from_numpy(e.scores).cuda()
                kept, sc = torch.zeros(want_kept.shape, dtype=torch.int32, device="cuda"), torch.zeros(want_sc.shape, device="cuda")
                n = torch.zeros(len(e.lens), dtype=torch.int32, device="cuda")
                with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(e.dst, dst_t, e.dst_seqs) as b:
                    torch.cuda.synchronize()
                    a.evict(b, scores, e.budget, kept_t=kept, kept_scores_t=sc, new_len_t=n, stream=stream.cuda_stream)
                    torch.cuda.synchronize()
                assert (kept.cpu().numpy() == want_kept).all() and (sc.cpu().numpy() == want_sc).all()
                assert (e.back(dst_t, want_pool) == want_pool).all()
    finally:
        B.pdkv_sm_partition_destroy(part)


@pytest.mark.parametrize("longest", [300, 9000])
def test_evictions_of_lengths_from_the_device(longest):
    """Into another pool and in place; lengths of none, one, the budget and above it, below the handle's."""
    caps = [longest, 40, 64, 90, 200, 33]
    for lens in ([longest - 7, 0, 1, 30, 31, 29], [5, 40, 64, 90, 200, 33], [longest, 0, 0, 0, 0, 0]):
        for in_place in (False, True):
            e = Evict(lens, 30, caps=caps, H=2, D=8, layers=2)
            src_t, dst_t = e.tensors()
            want_kept, want_sc, want_pool = e.expect(1, 2, (0, 2), in_place)
            lens_t = torch.tensor([n if n else -9 for n in lens], dtype=torch.int32, device="cuda")
            with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(e.dst, dst_t, e.dst_seqs) as b:
                kept, sc, n = a.evict(a if in_place else b, torch.from_numpy(e.scores).cuda(), 30, sink=1, recent=2, seq_len_t=lens_t)
            assert (kept.cpu().numpy() == want_kept).all() and (sc.cpu().numpy() == want_sc).all()
            assert n.tolist() == [min(x, 30) for x in lens]
            assert (e.back(src_t if in_place else dst_t, want_pool) == want_pool).all()


def test_sequences_without_a_token():
    """Handles whose sequences hold none: zeros, -infinity, -1 and lengths of zero."""
    s = Setup([0, 0], G=2, D=64, prefix_len=[0], member=[0, -1])
    with s.session() as c:
        out, lse = c.attend(s.layer, s.q_t, scores_t=torch.zeros(2, s.H, 4, device="cuda"))
        assert (out == 0).all() and torch.isneginf(lse).all()
        kept, sc, n = c.evict(c, torch.zeros(2, 2, s.H, 0, device="cuda"), 5)
        assert (kept == -1).all() and (sc == 0).all() and n.tolist() == [0, 0]
        c.status()


def test_the_default_stream_from_another_current_one():
    s = Setup([90, 33], G=2, D=64)
    with s.session() as c:
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            out, lse = c.attend(s.layer, s.q_t, stream=0)
            torch.cuda.default_stream().synchronize()
        check(s, out, lse, s.expect())


@pytest.mark.parametrize("kw", [
    dict(lens=[300, 41], G=8, D=64),
    dict(lens=[300, 41], G=4, Q=2, D=128, layout=LAYER_MAJOR, block=128),
    dict(lens=[700, 41], G=1, D=256, dtype="fp16"),
    dict(lens=[300, 41], G=7, D=80, block=7),
    dict(lens=[900, 300], G=3, D=128, dtype="fp16", prefix_len=[200], member=[0, -1]),
    dict(lens=[5000], H=1, G=6, D=96),
], ids=str)
def test_weights_of_few_rows_keep_their_bits(kw):
    """Up to 8 rows of a KV head: the weights go into the product with V as two 16-bit numbers, so that a weight is off by half a step of half
    a step, and the result by little more than its own rounding (half a step)."""
    s = Setup(q_scale=0.7, **kw)
    out, _, _, e = s.expect()
    with s.session() as c:
        assert kernel_of_own_tokens(c) == 0 and (c.items()["row_end"] - c.items()["row_begin"]).max() <= 8
        got = c.attend(s.layer, s.q_t)[0].double().cpu().numpy()
    half = torch.finfo(s.dtype).eps / 2
    rel = 2 * logit_error(e, s.D) + half * half + (e["n"] + 64) * 2.0 ** -23
    tol = 1.01 * (rel[..., None] * e["mag"] + half * np.abs(out)) + (e["n"][..., None] * 2.0 ** -32 * e["v"][..., None] + 2.0 ** -25 if s.dtype == torch.float16 else 0)
    over = (np.abs(got - out) / tol).max()
    assert over <= 1


@pytest.mark.parametrize("kernel,kw", [(0, dict(lens=[90, 33], G=2, Q=4, D=64)), (0, dict(lens=[90, 33], G=7, Q=3, D=80, block=7)),
                                       (1, dict(lens=[700, 260], G=12, Q=4, D=64)), (1, dict(lens=[700, 260], H=1, G=3, Q=100, D=128, block=32))], ids=str)
def test_weights_of_queries_that_are_nan(kernel, kw):
    """A query of NaN gives NaN to the tokens it sees, and nothing to those behind it."""
    s = Setup(**kw)
    before, scores = scores_like(s)
    want = s.expect()
    for r, i, hq, dims in ((0, 0, 0, slice(None)), (len(s.lens) - 1, 1, s.H * s.G - 1, 3)):
        s.q_t[r, i, hq, dims] = float("nan")
        want[0][r, i, hq] = want[1][r, i, hq] = np.nan
        want[2][r][hq // s.G, i * s.G + hq % s.G, :s.lens[r] - (s.Q - 1 - i)] = np.nan
    with s.session() as c:
        assert kernel_of_own_tokens(c) == kernel
        out, lse = c.attend(s.layer, s.q_t, scores_t=scores)
        c.status()
    assert (torch.isnan(out).cpu().numpy() == np.isnan(want[0])).all() and (torch.isnan(lse).cpu().numpy() == np.isnan(want[1])).all()
    assert torch.isnan(out).any() and not torch.isnan(out).all()
    got = scores.double().cpu().numpy()
    for r, n in enumerate(s.lens):
        add = want[2][r].sum(1)
        assert (np.isnan(got[r, :, :n]) == np.isnan(add)).all()
        assert np.isnan(add).any() and not np.isnan(add).all()
        # (the errors of test_scores are far below this)
        fin = ~np.isnan(add)
        assert (np.abs(got[r, :, :n][fin] - before[r, :, :n][fin] - add[fin]) <= 1e-4 * (1 + add[fin])).all()
