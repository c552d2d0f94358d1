"""Attention, accumulated weights and eviction on the GPU against 64-bit definitions."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200.sequences import CacheSession, Sequences
from paper_2408_08147_b200.workloads import BLOCK_MAJOR, LAYER_MAJOR, Geometry

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


class Setup:
    """A pool whose unused slots hold NaN, sequences in it, queries."""

    def __init__(self, lens, *, H=2, G=2, D=64, block=16, layout=BLOCK_MAJOR, dtype="bf16", Q=1, prefix_len=(), member=None,
                 layers=2, layer=1, seed=0, q_scale=2.0, spare=3, caps=None):
        rng = np.random.default_rng(seed)
        self.H, self.G, self.D, self.block, self.layout, self.Q, self.layer, self.layers = H, G, D, block, layout, Q, layer, layers
        self.dtype = DT[dtype]
        self.lens = [int(x) for x in lens]
        self.caps = self.lens if caps is None else caps
        self.prefix_len = list(prefix_len)
        counts = [-(-n // block) for n in self.prefix_len + self.caps]
        off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        blocks = int(off[-1]) + spare
        perm = rng.permutation(blocks)[:off[-1]].astype(np.int32)
        P = len(self.prefix_len)
        self.seqs = Sequences(self.caps, off[P:] - off[P], perm[off[P]:], self.prefix_len or None, off[:P + 1] if P else None,
                              perm[:off[P]] if P else None, member if P else None)
        self.geom = Geometry(layout, layers, H, D, 2, block, blocks)
        pool = np.full(self.geom.shape(), np.nan)
        self.fill(pool, rng, [(self.seqs.tbl[self.seqs.tbl_off[r]:], n) for r, n in enumerate(self.lens)])
        if P:
            self.fill(pool, rng, [(perm[off[i]:], n) for i, n in enumerate(self.prefix_len)])
        self.pool_t = torch.from_numpy(pool).to(self.dtype).cuda()
        q = rng.standard_normal((len(self.lens), Q, H * G, D)) * q_scale
        self.q_t = torch.from_numpy(q).to(self.dtype).cuda()

    def fill(self, pool, rng, lists):
        for tbl, n in lists:
            for t in range(n):
                x = rng.standard_normal((self.layers, 2, self.H, self.D))
                if self.layout == BLOCK_MAJOR:
                    pool[tbl[t // self.block], :, :, t % self.block] = x
                else:
                    pool[:, :, tbl[t // self.block], :, t % self.block] = x

    def session(self, **kw):
        return CacheSession(self.geom, self.pool_t, self.seqs, num_q_heads=self.H * self.G, q_tokens=self.Q, dtype=self.dtype, **kw)

    def expect(self, lens=None, scale=None, q_t=None):
        q = (self.q_t if q_t is None else q_t).double().cpu().numpy()
        return O.attend(self.pool_t.double().cpu().numpy(), self.layout, self.block, self.layer, self.seqs,
                        self.lens if lens is None else lens, q, self.H, self.D ** -0.5 if scale is None else scale)


def logit_error(e, D):
    """Bound on the absolute error of a logit.  The product of two 16-bit numbers is exact in 32 bits; D of them
    are added in 32 bits, each addition (the tensor cores cut instead of rounding) off by at most 2^-23 of the
    sum of magnitudes; scaling, the base-2 factor and its use round three times more (2^-24 each, on |z|), and
    the exponential is off by 2 units in the last place (2^-22 of the weight)."""
    return e["dot"] * D * 2.0 ** -23 + e["z"] * 4 * 2.0 ** -24 + 2.0 ** -22


def check(s, out_t, lse_t, want, q_lens=None):
    out, lse, _, e = want
    got, got_lse = out_t.double().cpu().numpy(), lse_t.double().cpu().numpy()
    d = logit_error(e, s.D)
    half = torch.finfo(s.dtype).eps / 2
    # weights: relative error of numerator and sum by the logits (2d), rounding of the weight for the product with
    # V (half a step), sums of n terms in 32 bits (n 2^-23); the result is rounded once more.  fp16 weights under
    # 2^-14 of the largest have an absolute error of 2^-25 each, the result likewise.
    rel = 2 * d + half + (e["n"] + 64) * 2.0 ** -23
    tol = 1.01 * (rel[..., None] * e["mag"] + half * np.abs(out))
    if s.dtype == torch.float16:
        tol += (e["n"] * 2.0 ** -25 * e["v"])[..., None] + 2.0 ** -25
    assert not np.isnan(got).any()
    bad = np.abs(got - out) > tol
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - out).max(), tol[bad][:3])
    empty = np.isneginf(lse)
    assert (np.isneginf(got_lse) == empty).all()
    assert (got[empty] == 0).all()
    lt = d + (e["n"] + 64) * 2.0 ** -23 + 4 * 2.0 ** -24 * np.where(empty, 0, np.abs(lse))
    off = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, lse))
    assert (off <= lt).all(), (off - lt).max()


def check_scores(s, before, got_t, want, lens):
    _, _, weights, e = want
    got = got_t.double().cpu().numpy()
    d = logit_error(e, s.D)
    for r, n in enumerate(lens):
        per_row = (2 * d[r] + (e["n"][r] + 64) * 2.0 ** -23).reshape(s.Q, s.H, s.G).transpose(1, 0, 2).reshape(s.H, s.Q * s.G)
        add = weights[r].sum(1)
        tol = 1.01 * (weights[r] * per_row[:, :, None]).sum(1) + (s.Q * s.G + 1) * 2.0 ** -23 * (add + np.abs(before[r, :, :n]))
        assert (np.abs(got[r, :, :n] - before[r, :, :n] - add) <= tol).all(), r
        assert (got[r, :, n:] == before[r, :, n:]).all()


CASES = [
    dict(lens=[1]),
    dict(lens=[300], H=4, G=2),
    dict(lens=[0, 1, 15, 16, 17, 63, 64, 65, 129], G=4),
    dict(lens=[700, 3], H=1, G=1, D=128, layout=LAYER_MAJOR, block=128),
    dict(lens=[200, 31], G=8, D=128, dtype="fp16", block=24),
    dict(lens=[200, 31], G=7, D=80, block=7, layout=LAYER_MAJOR),
    dict(lens=[90, 257], G=3, D=96, dtype="fp16", layout=LAYER_MAJOR, block=100),
    dict(lens=[90, 257], G=2, D=256, block=32),
    dict(lens=[70, 40], G=2, D=8, block=16),
    dict(lens=[70, 40], G=2, D=248, block=1, dtype="fp16"),
    dict(lens=[130, 5, 0, 3], G=5, Q=4),
    dict(lens=[130, 60], G=16, Q=1, H=1, D=128),
    dict(lens=[130, 60], G=12, Q=2, H=1, D=128),
    dict(lens=[130, 60], G=13, Q=3, H=1, D=128, dtype="fp16"),
    dict(lens=[130, 260], G=8, Q=16, H=2),
    dict(lens=[2500], H=1, G=4, D=128, block=64),
    dict(lens=[20, 40, 60], prefix_len=[100], member=[0, 0, 0], G=4, D=128),
    dict(lens=[20, 0, 60, 9], prefix_len=[33, 200, 0], member=[1, 0, -1, 2], G=4, Q=2, layout=LAYER_MAJOR),
    dict(lens=[5] * 40, prefix_len=[260], member=[0] * 40, H=1, G=4, D=128, dtype="fp16"),
    dict(lens=[5] * 17, prefix_len=[129, 64], member=[i % 2 for i in range(17)], H=1, G=8, D=64, block=32, layout=LAYER_MAJOR),
    dict(lens=[3] * 70, prefix_len=[515], member=[0] * 70, H=1, G=4, D=128, block=128, layout=LAYER_MAJOR),
    dict(lens=[0] * 9, prefix_len=[70], member=[0] * 9, H=2, G=8, D=128),
    dict(lens=[2] * 20, prefix_len=[385, 1, 128], member=[i % 3 for i in range(20)], H=2, G=8, D=80, block=8),
    dict(lens=[9] * 33, prefix_len=[700], member=[0] * 33, H=1, G=8, D=96, block=256, layout=LAYER_MAJOR, dtype="fp16"),
    dict(lens=[9] * 33, prefix_len=[257], member=[0] * 33, H=3, G=2, D=72, block=64, q_scale=12.0),
    dict(lens=[1, 500, 40, 0], H=2, G=6, Q=30, D=128, block=32),
    dict(lens=[700], H=1, G=4, Q=64, D=64, block=128, layout=LAYER_MAJOR, dtype="fp16"),
    dict(lens=[3000, 2990], H=1, G=8, Q=8, D=128, block=64, prefix_len=[1500], member=[0, 0]),
    dict(lens=[40, 150], H=2, G=50, D=64, block=24),
    # several items for every CTA
    dict(lens=[33, 0, 7, 64, 65, 31, 96, 1] * 24, H=8, G=1, D=64, layers=1, layer=0),
    dict(lens=[70, 300, 5, 129] * 20, H=4, G=4, D=128, block=8, layout=LAYER_MAJOR, layers=1, layer=0, dtype="fp16", prefix_len=[40], member=[0, -1] * 40),
    dict(lens=[70, 300, 5, 129] * 20, H=4, G=3, Q=4, D=80, block=12, layers=1, layer=0),
]


@pytest.mark.parametrize("kw", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention(kw):
    s = Setup(**kw)
    with s.session() as c:
        check(s, *c.attend(s.layer, s.q_t), s.expect())
        c.status()


@pytest.mark.parametrize("kw", CASES, ids=[str(i) for i in range(len(CASES))])
def test_scores(kw):
    s = Setup(**kw)
    width = max(s.lens) + 3
    before = np.random.default_rng(1).random((len(s.lens), s.H, width)).astype(np.float32)
    scores = torch.from_numpy(before).cuda()
    want = s.expect()
    with s.session() as c:
        out, lse = c.attend(s.layer, s.q_t, scores_t=scores)
        check(s, out, lse, want)
        check_scores(s, before.astype(np.float64), scores, want, s.lens)
        other = torch.full_like(scores, 7.0)
        c.attend(s.layer, s.q_t, scores_t=other, scores_in_t=torch.from_numpy(before).cuda())
        assert torch.equal(other[..., :-3], scores[..., :-3]) and (other[..., -3:] == 7.0).all()


@pytest.mark.parametrize("kw", [
    dict(lens=[20000], H=1, G=3, D=96),
    dict(lens=[9000, 700], H=1, G=2, Q=3, D=256, prefix_len=[8000], member=[0, -1]),
    dict(lens=[12000, 3], H=1, G=40, D=64, prefix_len=[5000], member=[-1, 0]),
    dict(lens=[15000, 2], H=1, G=20, Q=4, D=128),
], ids=str)
def test_rows_in_many_parts(kw):
    """Few heads and long lists: a row is cut into one part for each of the machine's CTAs."""
    s = Setup(layers=1, layer=0, **kw)
    scores = torch.zeros(len(s.lens), s.H, max(s.lens), device="cuda")
    want = s.expect()
    with s.session() as c:
        items = c.items()
        assert max(np.unique(np.stack([items["seq"], items["prefix"], items["row_begin"]]), axis=1, return_counts=True)[1]) > 16
        check(s, *c.attend(0, s.q_t), want)
        check(s, *c.attend(0, s.q_t, scores_t=scores), want)
        c.status()
    check_scores(s, np.zeros(scores.shape), scores, want, s.lens)


def test_current_lengths_from_the_device():
    """Lengths under the handle's; negative and too large ones are clamped; slots past them hold NaN."""
    s = Setup([3, 0, 90, 33, 200], caps=[40, 50, 128, 33, 200], G=4, Q=2, prefix_len=[50], member=[-1, -1, 0, 0, -1])
    lens_t = torch.tensor([3, -5, 90, 1000, 200], dtype=torch.int32, device="cuda")
    scores = torch.zeros(5, s.H, 200, device="cuda")
    with s.session() as c:
        out, lse = c.attend(s.layer, s.q_t, seq_len_t=lens_t, scores_t=scores)
        want = s.expect()
        check(s, out, lse, want)
        check_scores(s, np.zeros(scores.shape), scores, want, s.lens)


def test_strides_and_other_orders():
    s = Setup([40, 7, 100], G=2, Q=3, D=64)
    n, Q, Hq, D = s.q_t.shape
    wide = torch.zeros(Q, n, Hq + 5, D + 8, dtype=s.dtype, device="cuda")
    q = wide.permute(1, 0, 2, 3)[:, :, 2:2 + Hq, :D]
    q.copy_(s.q_t)
    out = torch.full((Hq, n, Q, D + 16), 9.0, dtype=s.dtype, device="cuda")
    view = out.permute(1, 2, 0, 3)[..., 8:8 + D]
    sc = torch.zeros(s.H, n, 131, device="cuda")
    with s.session() as c:
        _, lse = c.attend(s.layer, q, out_t=view, scores_t=sc.transpose(0, 1))
        want = s.expect()
        check(s, view, lse, want)
        check_scores(s, np.zeros((n, s.H, 131)), sc.transpose(0, 1), want, s.lens)
    assert (out[..., :8] == 9).all() and (out[..., 8 + D:] == 9).all()


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.5])
@pytest.mark.parametrize("G", [2, 60])
def test_scale(scale, G):
    s = Setup([150, 40], G=G, D=64)
    with s.session() as c:
        check(s, *c.attend(s.layer, s.q_t, scale=scale), s.expect(scale=scale))


def test_logits_of_minus_infinity_and_large_ones():
    s = Setup([80, 80, 80], H=1, G=2, D=64, dtype="fp16", block=16)
    pool = s.pool_t.clone()
    tb = s.seqs.tbl.reshape(3, 5)
    pool[tb[0].tolist(), s.layer, 0] = 0.0
    pool[tb[0].tolist(), s.layer, 0, :, :, 0] = -float("inf")     # every logit of sequence 0: -inf
    pool[tb[1][0], s.layer, 0, 3, 0, 0] = -float("inf")           # one of sequence 1
    s.q_t.abs_()
    pool[tb[2].tolist(), s.layer, 0] *= 300.0                     # logits in the thousands
    s.pool_t.copy_(pool)
    with s.session() as c:
        out, lse = c.attend(s.layer, s.q_t)
        check(s, out, lse, s.expect())
    assert torch.isneginf(lse[0]).all() and (out[0] == 0).all()


def test_nan_in_a_cached_token_stays_in_its_rows():
    s = Setup([60, 60], H=2, G=2, D=64)
    s.pool_t[s.seqs.tbl[1], s.layer, 0, 2, 1] = float("nan")      # a key of sequence 0, KV head 1
    with s.session() as c:
        out, lse = c.attend(s.layer, s.q_t)
    assert torch.isnan(out[0, 0, 2:]).all() and torch.isnan(lse[0, 0, 2:]).all()
    assert not torch.isnan(out[0, 0, :2]).any() and not torch.isnan(out[1]).any()


def test_same_bits_every_time_and_on_other_streams():
    s = Setup([900, 33, 400], H=2, G=4, D=128, prefix_len=[300], member=[0, 0, -1])
    with s.session() as c:
        sc = torch.zeros(3, 2, 900, device="cuda")
        first = c.attend(s.layer, s.q_t, scores_t=sc)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            sc2 = torch.zeros(3, 2, 900, device="cuda")
            again = c.attend(s.layer, s.q_t, scores_t=sc2)
        side.synchronize()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and torch.equal(sc, sc2)


def test_two_calls_at_once_with_a_scratch_each():
    s = Setup([900, 33, 400], H=2, G=4, D=128)
    with s.session() as c:
        want = c.attend(s.layer, s.q_t)[0].clone()
        q2 = s.q_t.flip(0).contiguous()
        want2 = c.attend(s.layer, q2)[0].clone()
        torch.cuda.synchronize()
        st = [torch.cuda.Stream() for _ in range(2)]
        scr = [torch.empty(c.scratch_bytes(), dtype=torch.uint8, device="cuda") for _ in range(2)]
        out = [torch.zeros_like(want) for _ in range(2)]
        lse = [torch.zeros(want.shape[:3], device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for i, q in enumerate((s.q_t, q2)):
                c.attend(s.layer, q, out_t=out[i], lse_t=lse[i], scratch_t=scr[i], stream=st[i].cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want) and torch.equal(out[1], want2)


def test_recorded_steps_follow_lengths_and_queries():
    s = Setup([90, 33, 200], caps=[90, 33, 200], G=4, D=128, prefix_len=[70], member=[0, 0, -1])
    lens_t = torch.tensor([1, 1, 1], dtype=torch.int32, device="cuda")
    q, sc = s.q_t.clone(), torch.zeros(3, s.H, 200, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    with s.session() as c:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            c.attend(s.layer, q, out_t=out, lse_t=lse, seq_len_t=lens_t, scores_t=sc)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.attend(s.layer, q, out_t=out, lse_t=lse, seq_len_t=lens_t, scores_t=sc)
        for lens in ([5, 33, 64], [90, 1, 200]):
            lens_t.copy_(torch.tensor(lens, dtype=torch.int32))
            q.copy_(s.q_t * 0.5)
            sc.zero_()
            g.replay()
            torch.cuda.synchronize()
            want = s.expect(lens, q_t=q)
            check(s, out, lse, want)
            check_scores(s, np.zeros(sc.shape), sc, want, lens)


@pytest.mark.parametrize("G", [2, 40])
def test_calls_follow_the_work_before_them(G):
    """Queries and lengths written by the operation just before a call, again and again and in a recorded sequence
    (a copy, a kernel of torch, a call of the library): a call never starts on them too early."""
    s = Setup([300, 33, 200], G=G, D=64, prefix_len=[70], member=[0, 0, -1])
    n = len(s.lens)
    with s.session() as c:
        qs = [s.q_t * f for f in (1.0, 0.5, 0.25)]
        want = [c.attend(s.layer, q)[0].clone() for q in qs]
        short = c.attend(s.layer, qs[1], seq_len_t=torch.tensor([7, 1, 9], dtype=torch.int32, device="cuda"))[0].clone()
        q, out, lse = torch.empty_like(s.q_t), torch.empty_like(s.q_t), torch.empty(s.q_t.shape[:3], device="cuda")
        lens, few = torch.empty(n, dtype=torch.int32, device="cuda"), torch.tensor([7, 1, 9], dtype=torch.int32, device="cuda")
        full = torch.tensor(s.lens, dtype=torch.int32, device="cuda")
        got = torch.empty(4, *out.shape, dtype=out.dtype, device="cuda")

        def steps():
            for i, x in enumerate(qs):
                torch.mul(s.q_t, (1.0, 0.5, 0.25)[i], out=q)
                lens.copy_(full)
                c.attend(s.layer, q, out_t=out, lse_t=lse, seq_len_t=lens)
                got[i].copy_(out)
            lens.copy_(few)
            c.attend(s.layer, qs[1], out_t=got[3], lse_t=lse, seq_len_t=lens)

        for _ in range(30):
            got.zero_()
            steps()
            assert all(torch.equal(got[i], want[i]) for i in range(3)) and torch.equal(got[3], short)
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            steps()
        for _ in range(5):
            got.zero_()
            g.replay()
            assert all(torch.equal(got[i], want[i]) for i in range(3)) and torch.equal(got[3], short)


def test_offsets_past_32_bits():
    """A pool of 5 GiB whose last blocks hold the tokens (both layouts)."""
    for layout in (BLOCK_MAJOR, LAYER_MAJOR):
        H, D, block, blocks = 8, 128, 128, 10300
        geom = Geometry(layout, 1, H, D, 2, block, blocks)
        pool = torch.empty(geom.shape(), dtype=torch.bfloat16, device="cuda")
        tbl = np.array([blocks - 1, blocks - 2, 0, blocks - 5], np.int32)
        view = pool if layout == BLOCK_MAJOR else pool.permute(2, 0, 1, 4, 3, 5)     # [block, layer, kv, token, head, dim]
        g = torch.Generator(device="cuda").manual_seed(3)
        for b in tbl:
            view[int(b)] = torch.randn(1, 2, block, H, D, device="cuda", generator=g).bfloat16()
        n = 500
        with CacheSession(geom, pool, Sequences([n], np.array([0, 4]), tbl), num_q_heads=16) as c:
            q = torch.randn(1, 1, 16, D, device="cuda", generator=g).bfloat16()
            out, lse = c.attend(0, q)
            k, v = (torch.cat([view[int(b), 0, kv] for b in tbl])[:n].double() for kv in (0, 1))
            z = torch.einsum("hd,thd->ht", q[0, 0].double(), k.repeat_interleave(2, 1)) * D ** -0.5
            want = torch.einsum("ht,thd->hd", torch.softmax(z, -1), v.repeat_interleave(2, 1))
            # weights and result rounded once each (half a step), everything else is far smaller
            mag = torch.einsum("ht,thd->hd", torch.softmax(z, -1), v.abs().repeat_interleave(2, 1))
            assert ((out[0, 0].double() - want).abs() <= 1.05 * 2.0 ** -8 * (mag + want.abs())).all()
            sc = torch.rand(1, 1, H, n, device="cuda", generator=g)
            c.evict(c, sc, 300)
            idx = torch.sort(torch.sort(sc[0, 0], descending=True, stable=True)[1][:, :300])[0]
            for kv, rows in ((0, k), (1, v)):
                got = torch.cat([view[int(b), 0, kv] for b in tbl])[:300].double()
                for h in range(H):
                    assert torch.equal(got[:, h], rows[idx[h], h])
        del pool, view
        torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------

class Evict:
    def __init__(self, lens, budget, *, H=2, D=16, E=2, layers=3, src=(BLOCK_MAJOR, 16), dst=(LAYER_MAJOR, 32), seed=0, caps=None):
        rng = np.random.default_rng(seed)
        self.lens, self.budget, self.H, self.layers = [int(x) for x in lens], budget, H, layers
        self.caps = self.lens if caps is None else caps
        self.np_t = {1: np.uint8, 2: np.uint16, 4: np.uint32, 8: np.uint64}[E]

        def side(layout, block, need):
            counts = [-(-n // block) for n in need]
            off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
            blocks = int(off[-1]) + 2
            tbl = rng.permutation(blocks)[:off[-1]].astype(np.int32)
            geom = Geometry(layout, layers, H, D, E, block, blocks)
            return geom, Sequences(need, off, tbl), rng.integers(0, 2 ** (8 * E) - 1, size=geom.shape(), dtype=self.np_t, endpoint=True)

        self.src, self.src_seqs, self.src_pool = side(*src, self.caps)
        self.dst, self.dst_seqs, self.dst_pool = side(*dst, [min(n, budget) for n in self.caps])
        self.width = max(self.caps + [1]) + 2
        self.scores = rng.standard_normal((layers, len(lens), H, self.width)).astype(np.float32)

    def tensors(self):
        return [torch.from_numpy(x.view(np.uint8).copy()).cuda() for x in (self.src_pool, self.dst_pool)]

    def back(self, t, like):
        return t.cpu().numpy().view(self.np_t).reshape(like.shape)

    def expect(self, sink, recent, layers, in_place=False):
        pool = (self.src_pool if in_place else self.dst_pool).copy()
        geom, seqs = (self.src, self.src_seqs) if in_place else (self.dst, self.dst_seqs)
        kept = np.full((layers[1] - layers[0], len(self.lens), self.H, self.budget), -1, np.int64)
        sc = np.zeros(kept.shape, np.float32)
        for l in range(*layers):
            for r, n in enumerate(self.lens):
                for h in range(self.H):
                    ids = O.select(self.scores[l - layers[0], r, h, :n], self.budget, sink, recent)
                    kept[l - layers[0], r, h, :len(ids)] = ids
                    sc[l - layers[0], r, h, :len(ids)] = self.scores[l - layers[0], r, h, ids]
                    O.move(self.src_pool, self.src.layout, self.src.block_tokens, self.src_seqs.tbl[self.src_seqs.tbl_off[r]:],
                           pool, geom.layout, geom.block_tokens, seqs.tbl[seqs.tbl_off[r]:], l, h, ids)
        return kept, sc, pool


EVICT = [
    dict(lens=[40, 7, 100], budget=20, sink=2, recent=5),
    dict(lens=[40, 7, 0, 1, 20, 21], budget=20),
    dict(lens=[300, 257, 256], budget=1, dst=(LAYER_MAJOR, 1)),
    dict(lens=[300], budget=299, sink=100, recent=199),
    dict(lens=[300, 50], budget=64, sink=64),
    dict(lens=[300, 50], budget=64, recent=64),
    dict(lens=[700, 1500], budget=500, sink=4, recent=100, H=1, src=(LAYER_MAJOR, 128), dst=(BLOCK_MAJOR, 7)),
    dict(lens=[90, 33], budget=30, E=1, D=5, src=(LAYER_MAJOR, 7)),
    dict(lens=[90, 33], budget=30, E=4, D=3),
    dict(lens=[90, 33], budget=30, E=8, D=80, src=(BLOCK_MAJOR, 1), dst=(BLOCK_MAJOR, 16)),
    dict(lens=[90, 33], budget=30, E=2, D=128, H=5),
    dict(lens=[5000, 9000], budget=2049, recent=7, H=1, layers=1),
    dict(lens=[140001], budget=70000, sink=1, recent=3, H=1, layers=1, D=4, src=(LAYER_MAJOR, 128), dst=(LAYER_MAJOR, 64)),
    dict(lens=[20, 50], budget=40, H=1, layers=2, D=9000, E=2),
    dict(lens=[40001], budget=12345, sink=1, recent=3, H=1, layers=1, D=8, src=(LAYER_MAJOR, 128), dst=(LAYER_MAJOR, 64)),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kw", EVICT, ids=[str(i) for i in range(len(EVICT))])
def test_eviction(kw, in_place):
    kw = dict(kw)
    sink, recent = kw.pop("sink", 0), kw.pop("recent", 0)
    e = Evict(**kw)
    src_t, dst_t = e.tensors()
    want_kept, want_sc, want_pool = e.expect(sink, recent, (0, e.layers), in_place)
    scores = torch.from_numpy(e.scores).cuda()
    with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(e.dst, dst_t, e.dst_seqs) as b:
        kept, sc, n = a.evict(a if in_place else b, scores, e.budget, sink=sink, recent=recent)
    assert (kept.cpu().numpy() == want_kept).all()
    assert (sc.cpu().numpy() == want_sc).all()
    assert n.tolist() == [min(x, e.budget) for x in e.lens]
    assert (e.back(src_t if in_place else dst_t, want_pool) == want_pool).all()
    if not in_place:
        assert (e.back(src_t, e.src_pool) == e.src_pool).all()
    assert (scores.cpu().numpy() == e.scores).all()


def test_equal_zero_infinite_and_nan_scores():
    e = Evict([60, 61, 62, 63, 300], 20, layers=1, H=1)
    s = e.scores[0, :, 0]
    s[0] = 1.0                                                    # all equal: the first ones
    s[1, ::2], s[1, 1::2] = 0.0, -0.0                             # -0 ties with +0
    s[2] = np.nan
    s[2, 40:50] = -np.inf                                         # above NaN
    s[3] = -1.0
    s[3, 5], s[3, 50], s[3, 7] = np.inf, np.inf, np.nan
    s[4, :300] = np.repeat(np.arange(75, dtype=np.float32) % 7, 4)      # many ties across warps
    src_t, dst_t = e.tensors()
    want = e.expect(0, 0, (0, 1))
    with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(e.dst, dst_t, e.dst_seqs) as b:
        kept, _, _ = a.evict(b, torch.from_numpy(e.scores).cuda(), 20)
    assert (kept.cpu().numpy() == want[0]).all()


def _rows_to_select_from(n, rng):
    """Scores that a sample, or the halving of an interval, is misled by."""
    comb = rng.random(n).astype(np.float32)
    comb[(n * np.arange(128)) // 128] = 5.0                       # evenly spaced: what a sample may see
    tied = rng.integers(0, 3, n).astype(np.float32)
    rare = np.full(n, -np.inf, np.float32)
    rare[rng.integers(0, n, 40)] = rng.standard_normal(40)
    rare[rng.integers(0, n, 40)] = np.nan
    tiny = (rng.random(n) * 1e-42).astype(np.float32)             # subnormal
    return [np.exp(3 * rng.standard_normal(n)).astype(np.float32), np.sort(rng.standard_normal(n)).astype(np.float32)[::-1], comb,
            tied, rare, tiny, np.where(rng.random(n) < 0.5, np.float32(1), np.float32(1 + 2.0**-23)).astype(np.float32)]


@pytest.mark.parametrize("longest", [300, 1500, 8192, 8193, 20000, 131073])
def test_selection_by_rows_and_budgets(longest):
    """Rows in registers of one CTA and of clusters, rows that are read again and again, shorter rows beside them."""
    rng = np.random.default_rng(longest)
    rows = [_rows_to_select_from(n, rng) for n in (longest, longest - longest // 3, 290)]
    lens = [len(r[0]) for r in rows]
    e = Evict(lens, 1, layers=7, H=1, D=8)
    scores = np.zeros((7, 3, 1, longest), np.float32)
    for r, kinds in enumerate(rows):
        for k in range(7):
            scores[k, r, 0, :lens[r]] = kinds[k]
    src_t, _ = e.tensors()
    dev = torch.from_numpy(scores).cuda()
    for budget, sink, recent in ((1, 0, 0), (64, 4, 16), (289, 0, 1), (longest // 2, 3, 100), (longest - 1, 0, 0)):
        d = Evict(lens, budget, layers=7, H=1, D=8)
        _, dst_t = d.tensors()
        with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(d.dst, dst_t, d.dst_seqs) as b:
            kept, _, n = a.evict(b, dev, budget, sink=sink, recent=recent)
        kept = kept.cpu().numpy()
        for k in range(7):
            for r in range(3):
                want = O.select(scores[k, r, 0, :lens[r]], budget, sink, recent)
                assert (kept[k, r, 0, :len(want)] == want).all() and (kept[k, r, 0, len(want):] == -1).all(), (k, r, budget)


def test_compaction_in_place_with_its_scores_and_device_lengths():
    """One buffer of scores and one of lengths, both updated in place; a range of layers."""
    e = Evict([100, 12, 0, 64], 30, caps=[160, 40, 20, 64])
    e.scores = e.scores[1:3].copy()
    src_t, _ = e.tensors()
    want_kept, want_sc, want_pool = e.expect(3, 4, (1, 3), in_place=True)
    scores = torch.from_numpy(e.scores).cuda()
    lens = torch.tensor([100, 12, -7, 64], dtype=torch.int32, device="cuda")
    with CacheSession(e.src, src_t, e.src_seqs) as a:
        kept, sc, n = a.evict(a, scores, 30, sink=3, recent=4, layers=(1, 3), kept_scores_t=scores, seq_len_t=lens, new_len_t=lens)
    assert (kept.cpu().numpy() == want_kept).all() and n.tolist() == [30, 12, 0, 30]
    assert (sc[..., :30].cpu().numpy() == want_sc).all() and (sc[..., 30:] == 0).all()
    assert (e.back(src_t, want_pool) == want_pool).all()


def test_eviction_is_recorded_and_replayed():
    e = Evict([100, 50], 30)
    src_t, dst_t = e.tensors()
    scores = torch.zeros(e.scores.shape, device="cuda")
    with CacheSession(e.src, src_t, e.src_seqs) as a, CacheSession(e.dst, dst_t, e.dst_seqs) as b:
        kept, sc, n = a.evict(b, scores, 30)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            a.evict(b, scores, 30, kept_t=kept, kept_scores_t=sc, new_len_t=n)
        scores.copy_(torch.from_numpy(e.scores))
        g.replay()
        torch.cuda.synchronize()
    want = e.expect(0, 0, (0, 3))
    assert (kept.cpu().numpy() == want[0]).all() and (e.back(dst_t, want[2]) == want[2]).all()


def test_decode_evict_decode():
    """As they are used: attend and weigh for some steps, compact in place, attend over what is left."""
    s = Setup([150, 90], H=2, G=2, D=64, layers=1, layer=0)
    scores = torch.zeros(2, 2, 150, device="cuda")
    lens_t = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    total = np.zeros((2, 2, 150))
    with s.session() as c:
        for n in ([148, 88], [149, 89], [150, 90]):
            lens_t.copy_(torch.tensor(n, dtype=torch.int32))
            out, lse = c.attend(0, s.q_t, scores_t=scores, seq_len_t=lens_t)
            want = s.expect(n)
            check(s, out, lse, want)
            for r in range(2):
                total[r, :, :n[r]] += want[2][r].sum(1)
        assert np.abs(scores.double().cpu().numpy() - total).max() < 1e-4
        before = s.pool_t.clone()
        host = scores.cpu().numpy()
        kept, _, _ = c.evict(c, scores[None], 64, sink=2, recent=16, kept_scores_t=scores[None], new_len_t=lens_t, seq_len_t=lens_t)
        assert lens_t.tolist() == [64, 64]
        ids = kept.cpu().numpy()[0]
        for r in range(2):
            for h in range(2):
                assert (ids[r, h] == O.select(host[r, h, :s.lens[r]], 64, 2, 16)).all()
        out, lse = c.attend(0, s.q_t, scores_t=scores, seq_len_t=lens_t)
        # the same attention, computed over the kept tokens of the pool as it was
        full = before.double().cpu().numpy()
        q = s.q_t.double().cpu().numpy()
        for r in range(2):
            tbl = s.seqs.tbl[s.seqs.tbl_off[r]:]
            for h in range(2):
                k, v = (O.token_rows(full, s.layout, s.block, 0, kv, h, tbl, s.lens[r])[ids[r, h]] for kv in (0, 1))
                for g in range(2):
                    z = k @ q[r, 0, 2 * h + g] * 64 ** -0.5
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    got = out[r, 0, 2 * h + g].double().cpu().numpy()
                    # weights and result are rounded once each: half a step of bf16, 2^-8
                    assert (np.abs(got - w @ v) <= 1.05 * 2.0 ** -8 * (w @ np.abs(v) + np.abs(w @ v))).all()
