"""Attention in other forms than plain causal (masks among the newest tokens, capped and biased scores) on the GPU against 64-bit definitions."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200.sequences import Rotary, pack_mask
from paper_2408_08147_b200.workloads import BLOCK_MAJOR, LAYER_MAJOR
from test_gpu_sequence_edges import cached_row, kernel_of_own_tokens
from test_gpu_sequences import Setup, check, check_scores

pytestmark = pytest.mark.gpu


def tree(rng, Q, m):
    """Ancestors of each of m nodes, and depths."""
    see, depth = np.zeros((Q, Q), bool), np.zeros(Q, np.int32)
    for i in range(m):
        if i:
            parent = int(rng.integers(max(0, i - 5), i))
            see[i], depth[i] = see[parent], depth[parent] + 1
        see[i, i] = True
    return see, depth


def mask_of(kind, rng, Q, news):
    n, at = len(news), np.arange(Q)
    see, depth = np.zeros((n, Q, Q), bool), np.tile(at.astype(np.int32), (n, 1))
    for r, m in enumerate(news):
        if kind == "tree":
            see[r], depth[r] = tree(rng, Q, m)
        elif kind == "documents":
            doc = np.cumsum(rng.random(Q) < 0.2)
            see[r] = (doc[:, None] == doc[None]) & (at[:, None] >= at[None])
        elif kind == "prefix":
            see[r] = (at[:, None] >= at[None]) | (at[None] < Q // 3)
        else:                              # any: rows that see none of the newest, tokens that nobody sees
            see[r] = rng.random((Q, Q)) < 0.4
            see[r, Q // 2] = False
            see[r, :, Q // 3] = False
    return see, depth


class Form:
    def __init__(self, s, kind="causal", cap=0.0, slopes=False, ragged=False, offset=False, seed=7):
        rng = np.random.default_rng(seed)
        n, Q = len(s.lens), s.Q
        self.s, self.cap = s, cap
        self.news = [int(x) for x in rng.integers(0, Q + 1, n)] if ragged else [Q] * n
        self.see, depth = mask_of(kind, rng, Q, self.news) if kind != "causal" else (None, np.tile(rng.integers(0, 9, Q).astype(np.int32), (n, 1)))
        self.offset = depth if offset else None
        self.slopes = (2.0 ** -rng.uniform(1, 8, s.H * s.G)).astype(np.float32) if slopes else None
        self.kw = dict(cap=cap or None, slopes_t=None if self.slopes is None else torch.from_numpy(self.slopes).cuda(),
                       mask_t=None if self.see is None else pack_mask(torch.from_numpy(self.see).cuda()),
                       n_new_t=torch.tensor(self.news, dtype=torch.int32, device="cuda") if ragged else None,
                       offset_t=None if self.offset is None else torch.from_numpy(self.offset).cuda())

    def expect(self, lens=None, scale=None, q_t=None):
        s = self.s
        q = (s.q_t if q_t is None else q_t).double().cpu().numpy()
        out, lse, w, e = O.attend_formed(s.pool_t.double().cpu().numpy(), s.layout, s.block, s.layer, s.seqs, s.lens if lens is None else lens, q, s.H,
                                         s.D ** -0.5 if scale is None else scale, self.cap, self.slopes, self.see, self.news, self.offset)
        # A capped logit, out (1 - 2 / (1 + 2^y)): the exponential is off by 2^-22 of itself, which moves the quotient by a quarter of that;
        # the sum, reciprocal and last step round by 2^-24, 2^-23 and 2^-24: below 2^-21 of the cap.  A bias is a product and three sums, its factor
        # and the distance rounded too: 6 * 2^-24.  `check` counts 4 * 2^-24 of what stands under "z".
        e["z"] = e["z"] + (self.cap * 2.0 ** -21 + e["bias"] * 6 * 2.0 ** -24) / (4 * 2.0 ** -24)
        return out, lse, w, e


CASES = [
    dict(lens=[1], Q=1, form=dict(cap=20.0)),
    dict(lens=[300], H=4, G=2, form=dict(cap=5.0)),
    dict(lens=[0, 1, 15, 16, 17, 63, 64, 65, 129], G=4, form=dict(cap=5.0, slopes=True)),
    dict(lens=[300, 41], G=3, Q=2, form=dict(slopes=True)),
    dict(lens=[300, 41], G=3, Q=2, form=dict(slopes=True, offset=True)),
    dict(lens=[700, 3, 40], H=1, G=1, D=128, layout=LAYER_MAJOR, block=128, Q=7, form=dict(kind="tree")),
    dict(lens=[200, 31], G=2, D=128, dtype="fp16", block=24, Q=8, form=dict(kind="tree", ragged=True)),
    dict(lens=[200, 31, 90], G=7, D=80, block=7, layout=LAYER_MAJOR, Q=5, form=dict(kind="any", ragged=True)),
    dict(lens=[90, 257], G=3, D=96, dtype="fp16", layout=LAYER_MAJOR, block=100, Q=6, form=dict(kind="documents", cap=3.0)),
    dict(lens=[90, 57], G=1, D=200, Q=12, form=dict(kind="prefix", cap=30.0, slopes=True, ragged=True)),
    dict(lens=[90, 57], G=2, D=256, Q=33, form=dict(kind="tree", slopes=True, offset=True, ragged=True)),
    dict(lens=[3, 0, 20, 9], G=2, D=64, Q=9, form=dict(kind="any", ragged=True)),                               # shorter than their newest tokens
    dict(lens=[3, 0, 20, 9], G=2, D=64, Q=9, form=dict(ragged=True)),
    dict(lens=[40, 13, 70], G=2, D=64, Q=4, prefix_len=[70, 33], member=[0, 1, 0], form=dict(kind="tree", ragged=True, slopes=True, offset=True)),
    dict(lens=[40, 13, 70], G=4, D=128, Q=16, prefix_len=[300], member=[0, -1, 0], form=dict(kind="any", ragged=True, cap=10.0, slopes=True)),
    dict(lens=[5, 6, 7, 8], G=8, D=128, Q=6, prefix_len=[200], member=[0] * 4, dtype="fp16", form=dict(kind="tree", ragged=True)),
    dict(lens=[3, 0, 40], G=3, D=40, Q=6, prefix_len=[50], member=[0, 0, 0], form=dict(kind="any", slopes=True, cap=9.0)),            # the same behind a prefix
    dict(lens=[70, 33], G=2, D=8, Q=3, form=dict(kind="tree", cap=4.0)),
    # the tile kernel: one and two row tiles, masks that cross its tiles of 128 tokens
    dict(lens=[1200], H=1, G=4, D=128, Q=16, block=16, form=dict(kind="tree"), kernel=1),
    dict(lens=[1200, 700], H=1, G=4, D=128, Q=64, block=128, layout=LAYER_MAJOR, form=dict(kind="tree", ragged=True, slopes=True, offset=True), kernel=1),
    dict(lens=[1100], H=2, G=1, D=64, Q=200, block=16, dtype="fp16", form=dict(kind="documents", cap=8.0), kernel=1),
    dict(lens=[900, 801], H=1, G=2, D=96, Q=100, block=24, form=dict(kind="any", ragged=True, cap=20.0, slopes=True), kernel=1),
    dict(lens=[900, 40], H=1, G=1, D=128, Q=300, block=8, form=dict(kind="prefix", slopes=True), kernel=1),      # (one sequence shorter than its newest tokens)
    dict(lens=[640, 513], H=1, G=5, D=80, Q=30, block=64, prefix_len=[400], member=[0, 0], form=dict(kind="any", ragged=True, cap=6.0, slopes=True, offset=True), kernel=1),
    dict(lens=[1300], H=1, G=2, D=128, Q=128, form=dict(ragged=True), kernel=1),
]
ids = lambda c: "-".join(f"{k}{v}" for k, v in c.items()).replace(" ", "").replace("'", "")  # noqa: E731


def setup(c, **more):
    c = dict(c)
    form, kernel = c.pop("form"), c.pop("kernel", None)
    s = Setup(**{**c, **more})
    return s, Form(s, **form), kernel


@pytest.mark.parametrize("c", CASES, ids=ids)
def test_forms(c):
    s, f, kernel = setup(c)
    with s.session() as x:
        if kernel is not None:
            assert kernel_of_own_tokens(x) == kernel
        got = x.attend(s.layer, s.q_t, **f.kw)
        x.status()
    check(s, *got, f.expect())


@pytest.mark.parametrize("c", CASES, ids=ids)
def test_weights_of_forms(c):
    s, f, _ = setup(c)
    width = max(s.lens) + 5
    scores = torch.rand(len(s.lens), s.H, width, device="cuda")
    before = scores.double().cpu().numpy()
    with s.session() as x:
        got = x.attend(s.layer, s.q_t, scores_t=scores, **f.kw)
        x.status()
    want = f.expect()
    check(s, *got, want)
    check_scores(s, before, scores, want, s.lens)


KERNELS = [dict(lens=[150, 90], G=2, D=64, Q=5), dict(lens=[700, 600], H=1, G=4, D=128, Q=40, block=64)]
# the prefix in the tile kernel, own tokens in the other one beside it
BOTH = dict(lens=[150, 90, 33], G=4, D=128, Q=5, prefix_len=[700], member=[0, 0, 0], layout=LAYER_MAJOR)


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
def test_nothing_special_is_plain_causal(c):
    s = Setup(**c)
    full = np.tril(np.ones((s.Q, s.Q), bool))
    want = s.expect()
    with s.session() as x:
        for kw in (dict(mask_t=pack_mask(torch.from_numpy(full).cuda()).expand(len(s.lens), -1, -1)),       # one mask for all
                   dict(n_new_t=torch.full((len(s.lens),), s.Q, dtype=torch.int32, device="cuda")),
                   dict(slopes_t=torch.zeros(s.H * s.G, device="cuda"))):
            check(s, *x.attend(s.layer, s.q_t, **kw), want)


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales_of_capped_logits(c, scale):
    s = Setup(**c)
    f = Form(s, kind="tree", cap=12.0, slopes=True, ragged=True)
    with s.session() as x:
        check(s, *x.attend(s.layer, s.q_t, scale=scale, **f.kw), f.expect(scale=scale))


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
def test_queries_and_values_that_are_not_there(c):
    """NaN in query tokens that are not there, infinities in the pool among the newest tokens: only rows that see them notice."""
    s = Setup(**c)
    f = Form(s, kind="tree", ragged=True, seed=3)
    f.news[0] = s.Q // 2
    f.see[0] = tree(np.random.default_rng(1), s.Q, f.news[0])[0]
    f.kw.update(mask_t=pack_mask(torch.from_numpy(f.see).cuda()), n_new_t=torch.tensor(f.news, dtype=torch.int32, device="cuda"))
    s.q_t[0, f.news[0]:] = float("nan")
    scores = torch.zeros(2, s.H, max(s.lens), device="cuda")
    first = s.lens[0] - f.news[0]
    cached_row(s, 0, first + 2, 1, 0)[3] = float("inf")            # the value of node 2, which its descendants see
    cached_row(s, 0, first + f.news[0] - 1, 0, 0)[5] = float("nan")   # the key of the last node, which only itself sees
    with s.session() as x:
        out, lse = x.attend(s.layer, s.q_t, scores_t=scores, **f.kw)
        x.status()
    assert (out[0, f.news[0]:] == 0).all() and torch.isneginf(lse[0, f.news[0]:]).all()
    last = f.news[0] - 1
    sees2, seesl = f.see[0, :, 2], f.see[0, :, last]
    assert seesl[:last].sum() == 0
    for i in range(last):
        heads = out[0, i, :s.G]
        assert torch.isfinite(heads[:, 4:]).all() and torch.isfinite(heads[:, :3]).all(), i
        assert torch.isinf(heads[:, 3]).all() if sees2[i] else torch.isfinite(heads[:, 3]).all(), i
        assert torch.isfinite(lse[0, i]).all()
    assert torch.isnan(out[0, last, :s.G]).all()
    # the last node's row has no finite sum, so its weights are NaN; tokens that it does not see (other branches) still have finite ones
    unseen = torch.from_numpy(np.concatenate([np.zeros(first, bool), ~f.see[0, last, :f.news[0]]]))
    assert torch.isfinite(scores[0, 0, :s.lens[0]].cpu()[unseen]).all()
    if s.H > 1:
        assert torch.isfinite(scores[0, 1, :s.lens[0]]).all()


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
def test_a_row_that_sees_nothing_beside_infinite_values(c):
    """Query tokens that are not there see none of the tokens that all others see: 0 times infinity in their products."""
    s = Setup(**c)
    f = Form(s, kind="any", ragged=True)
    f.news[:] = [2, s.Q]
    f.kw["n_new_t"] = torch.tensor(f.news, dtype=torch.int32, device="cuda")
    for kv in (1, 0):
        cached_row(s, 0, 1, kv, 0)[:4] = float("inf")
    with s.session() as x:
        out, lse = x.attend(s.layer, s.q_t, **f.kw)
    assert (out[0, 2:] == 0).all() and torch.isneginf(lse[0, 2:]).all()
    want = f.expect()
    assert np.isfinite(want[0][1]).all()
    got = out[1].double().cpu().numpy()
    assert np.isfinite(got).all()


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
def test_lengths_from_the_device(c):
    s = Setup(**c)
    f = Form(s, kind="tree", cap=9.0, slopes=True, ragged=True, offset=True)
    for lens in ([s.lens[0] - 37, 33], [3, s.lens[1]], [0, s.Q]):
        t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        with s.session() as x:
            check(s, *x.attend(s.layer, s.q_t, seq_len_t=t, **f.kw), f.expect(lens=lens))


def test_a_step_of_speculative_decoding():
    """append a tree, attend to it, accept a path, append behind it and attend again: as if the accepted tokens had been cached at once."""
    Q, lens = 12, [100, 61, 33]
    s = Setup([n + Q for n in lens], G=4, D=128, Q=Q, layout=LAYER_MAJOR, block=16)
    rng = np.random.default_rng(4)
    values = lambda *shape: torch.from_numpy(rng.standard_normal(shape) * 1.5).to(s.dtype).cuda()  # noqa: E731
    see, depth = mask_of("tree", rng, Q, [Q] * 3)
    paths = []
    for r in range(3):
        leaf = int(rng.integers(1, Q))
        paths.append(np.flatnonzero(see[r, leaf]).tolist())
    path_t = torch.tensor([p + [-1] * (Q - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    rotary = Rotary(128, base=500000.0)
    w = torch.rand(128, device="cuda") + 0.5
    k, v, q = values(3, Q, s.H, 128), values(3, Q, s.H, 128), values(3, Q, s.H * s.G, 128)
    k2, v2, q2 = values(3, Q, s.H, 128), values(3, Q, s.H, 128), values(3, Q, s.H * s.G, 128)
    layer, dev = s.layer, "cuda"
    lens_t = torch.tensor(s.lens, dtype=torch.int32, device=dev)
    positions = torch.from_numpy((np.array(lens)[:, None] + depth).reshape(-1).astype(np.int32)).to(dev)
    start = s.pool_t.clone()
    with s.session() as x:
        turned = x.append(layer, k, v, q, rotary=rotary, position_t=positions, q_norm_t=w, k_norm_t=w, seq_len_t=lens_t)
        out, _ = x.attend(layer, turned, mask_t=pack_mask(torch.from_numpy(see).to(dev)), seq_len_t=lens_t)
        new_len = x.accept(path_t, seq_len_t=lens_t)
        assert new_len.tolist() == [n + len(p) for n, p in zip(lens, paths)]
        # the next step: one token behind each accepted path
        one = torch.ones(3, dtype=torch.int32, device=dev)
        turned2 = x.append(layer, k2, v2, q2, rotary=rotary, q_norm_t=w, k_norm_t=w, seq_len_t=new_len + 1, n_new_t=one)
        out2, _ = x.attend(layer, turned2, seq_len_t=new_len + 1, n_new_t=one)
        torch.cuda.synchronize()
        # the accepted tokens alone, in order, then the same token
        s.pool_t.copy_(start)
        for r, p in enumerate(paths):
            m = len(p)
            idx = torch.tensor(p, device=dev)
            pad = lambda t: torch.cat([t[r, idx], t[r, :Q - m]])[None].expand(3, -1, -1, -1).contiguous()  # noqa: E731
            mine = torch.zeros(3, dtype=torch.int32, device=dev)
            mine[r] = m
            plain = x.append(layer, pad(k), pad(v), pad(q), rotary=rotary, q_norm_t=w, k_norm_t=w, seq_len_t=new_len, n_new_t=mine)
            ref, _ = x.attend(layer, plain, seq_len_t=new_len, n_new_t=mine)
            assert torch.equal(plain[r, :m], turned[r, idx])
            # the same sums in another order: each side rounds weights and result by half a step, 2^-8, of the largest value at most
            assert (ref[r, :m].float() - out[r, idx].float()).abs().max() <= 4 * 2.0 ** -8 * s.pool_t.float().nan_to_num().abs().max()
        turned3 = x.append(layer, k2, v2, q2, rotary=rotary, q_norm_t=w, k_norm_t=w, seq_len_t=new_len + 1, n_new_t=one)
        out3, _ = x.attend(layer, turned3, seq_len_t=new_len + 1, n_new_t=one)
        assert torch.equal(turned3[:, 0], turned2[:, 0]) and torch.equal(out3, out2)


@pytest.mark.parametrize("c", KERNELS + [BOTH], ids=["warp", "tile", "both"])
def test_recorded_and_replayed_beside_another_graph(c):
    s = Setup(**c)
    forms = [Form(s, kind="tree", ragged=True, cap=9.0, seed=1), Form(s, kind="any", ragged=True, slopes=True, seed=2)]
    with s.session() as x:
        alone = [tuple(t.clone() for t in x.attend(s.layer, s.q_t, **f.kw)) for f in forms]
        graphs, outs = [], []
        for f in forms:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                outs.append(x.attend(s.layer, s.q_t, **f.kw))
            graphs.append(g)
        for _ in range(3):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, alone):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("c", KERNELS + [BOTH], ids=["warp", "tile", "both"])
def test_work_before_the_call_is_waited_for(c):
    s = Setup(**c)
    f = Form(s, kind="tree", ragged=True, cap=9.0, slopes=True, offset=True)
    side = torch.cuda.Stream()
    with s.session() as x:
        want = x.attend(s.layer, s.q_t, **f.kw)
        torch.cuda.synchronize()
        late = {k: torch.zeros_like(t) for k, t in f.kw.items() if torch.is_tensor(t)}
        q = torch.zeros_like(s.q_t)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(900_000_000)
            for k, t in late.items():
                t.copy_(f.kw[k])
            q.copy_(s.q_t)
        got = x.attend(s.layer, q, stream=side.cuda_stream, **{**f.kw, **late})
        side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("c", [
    dict(lens=[300, 230], G=2, D=64, Q=9, block=16, form=dict(kind="any", cap=20.0)),
    dict(lens=[900, 770], H=1, G=4, D=128, Q=100, block=32, form=dict(kind="any", cap=20.0)),
    dict(lens=[900, 770], H=1, G=2, D=128, Q=140, block=32, form=dict(kind="any", cap=20.0, slopes=True)),
], ids=["warp", "tile", "tile-sloped"])
def test_bits_do_not_depend_on_what_is_not_seen(c):
    """Keys behind a sequence's end, of a token that nobody sees, and queries that are not there: whatever they hold."""
    s, f, _ = setup(c)
    f.news[:] = [s.Q - 3, s.Q]
    f.kw["n_new_t"] = torch.tensor(f.news, dtype=torch.int32, device="cuda")
    nobody = s.Q // 3
    with s.session() as x:
        want = None
        for value in (float("nan"), 0.0, 1000.0, -3.0, float("inf")):
            s.q_t[0, s.Q - 3:] = value
            for r, n in enumerate(s.lens):
                first = n - f.news[r]
                f.see[r, :, nobody] = False
                for kv in (0, 1):
                    cached_row(s, r, first + nobody, kv, 0)[:] = value
                    for t in range(n, -(-n // s.block) * s.block):
                        cached_row(s, r, t, kv, 0)[:] = value
            got = x.attend(s.layer, s.q_t, **f.kw)
            if want is None:
                want = got
            assert torch.equal(got[0][:, :, :s.G], want[0][:, :, :s.G]) and torch.equal(got[1][:, :, :s.G], want[1][:, :, :s.G]), value
            assert torch.isfinite(got[0]).all()


def test_refused_forms():
    s = Setup([50, 20], G=2, D=64, Q=4)
    n, T, Hq = 2, 4, 4
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    with s.session() as x:
        for kw in (dict(cap=0.0), dict(cap=-1.0), dict(cap=float("nan")), dict(slopes_t=torch.zeros(Hq + 1, device="cuda")), dict(slopes_t=torch.zeros(Hq, device="cuda").half()),
                   dict(mask_t=ints(n, T)), dict(mask_t=ints(n, T, 2)), dict(mask_t=ints(n, T, 1).long()), dict(mask_t=ints(n, T, 1).cpu()), dict(n_new_t=ints(n + 1)),
                   dict(n_new_t=ints(2 * n)[::2]), dict(offset_t=ints(n, T)), dict(offset_t=ints(n, T + 1), slopes_t=torch.zeros(Hq, device="cuda"))):
            with pytest.raises(ValueError):
                x.attend(s.layer, s.q_t, **kw)
        for kw in (dict(cap=float("inf")), dict(cap=1e-44), dict(cap=3e38), dict(cap=1e300)):
            with pytest.raises(B.PdkvError) as e:
                x.attend(s.layer, s.q_t, **kw)
            assert e.value.status == B.PDKV_ERR_INVALID_ARG
        out = torch.empty_like(s.q_t)
        with pytest.raises(B.PdkvError):                        # written on what is read
            x.attend(s.layer, s.q_t, out_t=out, n_new_t=out.view(torch.int32).flatten()[:2])


@pytest.mark.parametrize("c", [
    dict(lens=[900, 700, 650], H=2, G=4, D=128, Q=160, block=64, form=dict(kind="documents", cap=20.0)),            # whole items of absent tokens
    dict(lens=[900, 700, 650], H=1, G=2, D=64, Q=200, block=64, prefix_len=[300], member=[0, 0, -1], form=dict(kind="tree")),
    dict(lens=[90, 70, 65], H=2, G=3, D=256, Q=40, block=64, prefix_len=[100], member=[0, -1, 0], form=dict(kind="any", slopes=True)),
], ids=["tile", "prefix", "warp"])
@pytest.mark.parametrize("news", [[1, 0, 64], [0, 0, 0], [65, 3, 1000]], ids=str)
def test_few_of_many_query_tokens_are_there(c, news):
    s, f, _ = setup(c)
    news = [min(x, s.Q) for x in news]
    f.news[:] = news
    f.kw["n_new_t"] = torch.tensor(news, dtype=torch.int32, device="cuda")
    scores = torch.rand(3, s.H, max(s.lens), device="cuda")
    before = scores.double().cpu().numpy()
    with s.session() as x:
        got = x.attend(s.layer, s.q_t, **f.kw)
        # scratch that holds NaN: what no kernel of this call has written is not read
        x.attend(s.layer, s.q_t, scores_t=scores, scratch_t=torch.full((max(16, x.scratch_bytes(True)),), 255, dtype=torch.uint8, device="cuda"), **f.kw)
        again = x.attend(s.layer, s.q_t, scratch_t=torch.full((max(16, x.scratch_bytes()),), 255, dtype=torch.uint8, device="cuda"), **f.kw)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
        x.status()
    want = f.expect()
    check(s, *got, want)
    check_scores(s, before, scores, want, s.lens)
