"""New tokens into the cache (norms and rotation on the way) and accepted paths, on the GPU against 64-bit definitions."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2408_08147_b200.sequences import CacheSession, Rotary, Sequences
from paper_2408_08147_b200.workloads import BLOCK_MAJOR, LAYER_MAJOR, Geometry

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


class Pool:
    """A pool of random numbers and sequences in it."""

    def __init__(self, lens, *, H=2, G=2, D=64, block=16, layout=BLOCK_MAJOR, dtype="bf16", layers=2, prefix_len=(), member=None, seed=0, q_tokens=1, elem=2):
        rng = np.random.default_rng(seed)
        self.rng, self.H, self.G, self.D, self.block, self.layout, self.layers, self.dtype, self.lens = rng, H, G, D, block, layout, layers, DT[dtype], list(lens)
        self.prefix_len, self.member = list(prefix_len), member
        counts = [-(-n // block) for n in list(prefix_len) + list(lens)]
        off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        blocks, P = int(off[-1]) + 3, len(prefix_len)
        perm = rng.permutation(blocks)[:off[-1]].astype(np.int32)
        self.seqs = Sequences(lens, off[P:] - off[P], perm[off[P]:], prefix_len or None, off[:P + 1] if P else None, perm[:off[P]] if P else None, member if P else None)
        self.geom = Geometry(layout, layers, H, D, elem, block, blocks)
        kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[elem]
        self.bits = torch.from_numpy(rng.integers(0, 200, self.geom.shape())).to(kind).cuda()
        self.pool_t = self.bits.view(self.dtype) if elem == 2 else self.bits
        self.before = self.bits.cpu().numpy().copy()
        self.q_tokens, self.attends = q_tokens, elem == 2

    def session(self, **kw):
        more = dict(num_q_heads=self.H * self.G, q_tokens=self.q_tokens, dtype=self.dtype) if self.attends else {}
        return CacheSession(self.geom, self.pool_t, self.seqs, **{**more, **kw})

    def values(self, *shape, scale=1.5):
        return torch.from_numpy(self.rng.standard_normal(shape) * scale).to(self.dtype).cuda()

    def rows_at(self, bits, layer, kv, r, slot):
        b, tt = int(self.seqs.tbl[self.seqs.tbl_off[r] + slot // self.block]), slot % self.block
        return bits[b, layer, kv, tt] if self.layout == BLOCK_MAJOR else bits[layer, kv, b, :, tt]


def tolerance(y, mag, dtype):
    """The sum of squares is 4 products and 3 sums in a lane and 5 sums between lanes, 2^-24 each; half of that enters the root; the reciprocal of the
    root is off by 2 units in the last place, mean, factor and product round four times: below 16 * 2^-24 of the normalised value.  An angle
    is off by pi * 2^-25 by its conversion and 2^-32 of a turn, its sine and cosine by 2 units in the last place: 2^-22 together; the
    scale, the weight, the products and the sum round five times.  (16 + 4 + 5) 2^-24 < 2^-19 of what is summed.  The result is rounded once,
    fp16 below 2^-14 to 2^-25."""
    half = torch.finfo(dtype).eps / 2
    return 1.01 * (half * np.abs(y) + 2.0 ** -19 * mag) + (2.0 ** -25 if dtype == torch.float16 else 0)


def check(p, layer, tokens, q_out, *, rotary=None, frequencies=None, positions=None, q_norm=None, k_norm=None, eps=1e-6, lens=None):
    """``tokens``: (sequence, number among its count new ones, count, row, q, k, v) with float64 heads; q_out indexed by row."""
    lens = p.lens if lens is None else lens
    after = p.bits.cpu().numpy()
    expect_same = np.ones(after.shape, bool)
    got_q = None if q_out is None else q_out.double().cpu().numpy()
    for r, i, count, row, q, k, v in tokens:
        slot = lens[r] - count + i
        before = p.prefix_len[p.member[r]] if p.prefix_len and p.member[r] >= 0 else 0
        at = before + slot if positions is None else positions[row] if positions.ndim == 1 else positions[:, row]

        def turn(x, w):
            if rotary is None:
                return O.turned(x, w, eps, 0, [], 0, False)
            return O.turned(x, w, eps, at, frequencies, rotary.dims, rotary.adjacent, None if rotary.axis_t is None else rotary.axis_t.cpu().numpy(), rotary.scale)

        if q_out is not None:
            for h in range(q.shape[0]):
                y, mag = turn(q[h], q_norm)
                tol = tolerance(y, mag, p.dtype)
                assert (np.abs(got_q[row][h] - y) <= tol).all(), (r, i, h, np.abs(got_q[row][h] - y).max())
        if slot < 0:
            continue
        got_k = torch.from_numpy(np.ascontiguousarray(p.rows_at(after, layer, 0, r, slot))).view(p.dtype).double().numpy()
        for h in range(p.H):
            y, mag = turn(k[h], k_norm)
            assert (np.abs(got_k[h] - y) <= tolerance(y, mag, p.dtype)).all(), (r, i, h, np.abs(got_k[h] - y).max())
        assert (p.rows_at(after, layer, 1, r, slot) == v).all(), (r, i)
        for kv in (0, 1):
            p.rows_at(expect_same, layer, kv, r, slot)[...] = False
    assert (after[expect_same] == p.before[expect_same]).all()


def f64(t):
    return t.double().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


CASES = [
    dict(lens=[1], new=1, dims=64),
    dict(lens=[300], new=1, H=4, dims=64, dtype="fp16"),
    dict(lens=[5, 17, 33, 64], new=5, G=3, dims=32, layout=LAYER_MAJOR, block=7),
    dict(lens=[40, 9], new=3, H=5, G=3, D=80, dims=80, block=24, norm="qk"),
    dict(lens=[40, 9], new=3, H=5, G=3, D=80, dims=20, block=24, norm="k", dtype="fp16"),          # half of the dims is 10: pairs in pieces
    dict(lens=[40, 9], new=2, H=3, G=1, D=80, dims=20, adjacent=True, norm="q"),                    # a run of eight dims turns in part
    dict(lens=[40, 9], new=2, H=3, G=1, D=64, dims=2, layout=LAYER_MAJOR),
    dict(lens=[21, 9], new=2, H=1, G=7, D=128, dims=128, adjacent=True, norm="qk", block=128),
    dict(lens=[21, 9], new=2, H=2, G=2, D=256, dims=64, norm="qk", layout=LAYER_MAJOR, block=100),
    dict(lens=[21, 9], new=2, H=2, G=2, D=256, dims=250, norm="qk", dtype="fp16"),
    dict(lens=[21, 9], new=2, H=2, G=2, D=200, dims=200, scale=1.25),
    dict(lens=[21, 9], new=2, H=2, G=2, D=96, dims=0, norm="qk"),
    dict(lens=[21, 9], new=2, H=2, G=2, D=8, dims=8, norm="qk"),
    dict(lens=[21, 9], new=2, H=2, G=2, D=24, dims=16, dtype="fp16"),
    dict(lens=[30, 3, 60], new=4, G=4, D=128, dims=128, prefix_len=[50, 7], member=[1, -1, 0], layout=LAYER_MAJOR),   # lengths below the new tokens, prefixes
    dict(lens=[30, 44], new=4, G=4, D=128, dims=128, axes=3, norm="qk"),
    dict(lens=[30, 44], new=4, G=4, D=80, dims=20, axes=2, dtype="fp16"),
    dict(lens=[3000], new=2800, H=1, G=1, D=64, dims=64, norm="qk"),                                # 2, 8 and more steps a warp
    dict(lens=[700, 700], new=650, H=8, G=4, D=64, dims=16, oracle_rows=40),
    dict(lens=[1800, 2000], new=1700, H=8, G=4, D=128, dims=128, norm="qk", oracle_rows=25, layers=1),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items() if k not in ("lens",)).replace(" ", ""))
@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
def test_append(c, packed):
    c = dict(c)
    new, dims, norm, axes, adjacent = c.pop("new"), c.pop("dims"), c.pop("norm", ""), c.pop("axes", 0), c.pop("adjacent", False)
    scale, most = c.pop("scale", 1.0), c.pop("oracle_rows", 10 ** 9)
    p = Pool(**c)
    n, layer = len(p.lens), p.layers - 1
    # packed: other numbers of tokens, none for some; else of the rows of a sequence only some count
    counts = [new if r == 0 else int(p.rng.integers(0, new + 1)) for r in range(n)]
    shape = (sum(counts),) if packed else (n, new)
    fused = p.values(*shape, p.H * (p.G + 2) * p.D)
    q, k, v = (x.unflatten(-1, (-1, p.D)) for x in fused.split([p.H * p.G * p.D, p.H * p.D, p.H * p.D], -1))
    freq = 10000.0 ** (-np.arange(dims // 2) / max(1, dims // 2))
    rotary = Rotary(dims, frequencies=freq, adjacent=adjacent, axes=np.arange(dims // 2) % axes if axes else None, scale=scale) if dims else None
    rows = int(np.prod(shape))
    positions = p.rng.integers(-50, 200000, (axes, rows)).astype(np.int32) if axes else None
    w = {x: 1 + 0.3 * p.rng.standard_normal(p.D).astype(np.float32) for x in norm}
    kw = dict(row_begin_t=torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")) if packed else dict(n_new_t=torch.tensor(counts, dtype=torch.int32, device="cuda"))
    mark = torch.full(q.shape, 77.0, dtype=p.dtype, device="cuda")
    with p.session() as s:
        out = s.append(layer, k, v, q, q_out_t=mark, rotary=rotary, position_t=None if positions is None else torch.from_numpy(positions).cuda(),
                       q_norm_t=torch.from_numpy(w["q"]).cuda() if "q" in w else None, k_norm_t=torch.from_numpy(w["k"]).cuda() if "k" in w else None, **kw)
        torch.cuda.synchronize()
    assert out is mark
    Q, K, V = f64(q).reshape(rows, -1, p.D), f64(k).reshape(rows, -1, p.D), bits(v).reshape(rows, -1, p.D)
    tokens, row0, live = [], 0, np.zeros(rows, bool)
    for r, m in enumerate(counts):
        for i in range(m):
            row = row0 + i if packed else r * new + i
            live[row] = True
            tokens.append((r, i, m, row, Q[row], K[row], V[row]))
        row0 += m
    flat = out.flatten(0, -3)
    assert (flat[torch.from_numpy(~live).cuda()] == 77).all()
    if len(tokens) > most:      # the definition of every row would take minutes: some of each sequence, the pool outside by its bits
        chosen = set(p.rng.permutation(len(tokens))[:most].tolist()) | {0, len(tokens) - 1}
        skipped = [t for i, t in enumerate(tokens) if i not in chosen]
        after = p.bits.cpu().numpy()
        for r, i, m, row, _, _, vv in skipped:
            slot = p.lens[r] - m + i
            assert (p.rows_at(after, layer, 1, r, slot) == vv).all()
            for kv in (0, 1):
                p.rows_at(p.before, layer, kv, r, slot)[...] = p.rows_at(after, layer, kv, r, slot)
        tokens = [t for i, t in enumerate(tokens) if i in chosen]
    check(p, layer, tokens, flat, rotary=rotary, frequencies=freq, positions=positions, q_norm=w.get("q"), k_norm=w.get("k"))


def every_token(p, q, k, v, new):
    Q, K, V = (f(x).reshape(-1, x.shape[-2], p.D) for f, x in ((f64, q), (f64, k), (bits, v)))
    return [(r, i, new, r * new + i, Q[r * new + i], K[r * new + i], V[r * new + i]) for r in range(len(p.lens)) for i in range(new)]


@pytest.mark.parametrize("far", [100003, 1 << 24, (1 << 31) - 1, -(1 << 31)])
def test_far_positions(far):
    """An angle of 32 bits would be off by 64 radians at the last of these."""
    p = Pool([8, 8], G=1, D=64)
    freq = np.array([1.0, 0.75, 2.0 ** -31, 3.5, -0.3, 6.0, 0.0, 7e-4] * 4)
    rotary = Rotary(64, frequencies=freq)
    q, k, v = p.values(2, 3, 2, 64), p.values(2, 3, 2, 64), p.values(2, 3, 2, 64)
    at = np.clip(far + np.arange(6) - 5 * (far > 0), -(1 << 31), (1 << 31) - 1)
    with p.session() as s:
        out = s.append(0, k, v, q, rotary=rotary, position_t=torch.from_numpy(at.astype(np.int32)).cuda())
        torch.cuda.synchronize()
    check(p, 0, every_token(p, q, k, v, 3), out.flatten(0, 1), rotary=rotary, frequencies=freq, positions=at)


def test_lengths_from_the_device_in_place_and_without_queries():
    p = Pool([40, 23, 9], G=2, D=64)
    rotary = Rotary(64, base=500000.0)
    freq = 500000.0 ** (-np.arange(32) / 32)
    q, k, v = p.values(3, 2, 4, 64), p.values(3, 2, 2, 64), p.values(3, 2, 2, 64)
    lens = [40, 11, 300]                                                  # the last is clamped to what its table is good for
    tokens = every_token(p, q, k, v, 2)
    with p.session() as s:
        t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        assert s.append(1, k, v, rotary=rotary, seq_len_t=t) is None
        torch.cuda.synchronize()
        check(p, 1, tokens, None, rotary=rotary, frequencies=freq, lens=[40, 11, 9])
        assert s.append(1, k, v, q, q_out_t=q, rotary=rotary, seq_len_t=t) is q
        torch.cuda.synchronize()
        check(p, 1, tokens, q.flatten(0, 1), rotary=rotary, frequencies=freq, lens=[40, 11, 9])


def test_values_are_copied_bit_for_bit_and_bad_numbers_stay_in_their_head():
    p = Pool([16], H=3, G=1, D=64)
    q, k, v = p.values(1, 1, 3, 64), p.values(1, 1, 3, 64), p.values(1, 1, 3, 64)
    v.view(torch.int16)[0, 0, 0, :6] = torch.tensor([0x7f81, 0x7fff, -1, -32768, 0x7f80, 1], dtype=torch.int16)   # NaNs with payloads, -0, infinity, a denormal
    k[0, 0, 1, 5] = float("nan")
    q[0, 0, 2, 9] = float("inf")
    with p.session() as s:
        out = s.append(0, k, v, q, rotary=Rotary(32), q_norm_t=torch.ones(64, device="cuda"), k_norm_t=torch.ones(64, device="cuda"))
        torch.cuda.synchronize()
    after = p.bits.cpu().numpy()
    assert (p.rows_at(after, 0, 1, 0, 15) == bits(v)[0, 0]).all()
    keys = torch.from_numpy(p.rows_at(after, 0, 0, 0, 15).copy()).view(p.dtype)
    assert torch.isnan(keys[1]).all() and torch.isfinite(keys[[0, 2]]).all()
    assert not torch.isfinite(out[0, 0, 2]).any() or torch.isnan(out[0, 0, 2]).any()
    assert torch.isfinite(out[0, 0, :2]).all()


def test_dims_that_do_not_turn_keep_infinities():
    """A dim outside the rotation is not mixed with its neighbour (infinity times a sine of 0 is NaN)."""
    p = Pool([16], H=1, G=1, D=64)
    for dims, adjacent in ((20, False), (20, True), (32, False), (32, True)):
        k = p.values(1, 1, 1, 64)
        k[..., dims] = float("inf")
        with p.session() as s:
            s.append(0, k, k, rotary=Rotary(dims, adjacent=adjacent))
            torch.cuda.synchronize()
        keys = torch.from_numpy(p.rows_at(p.bits.cpu().numpy(), 0, 0, 0, 15).copy()).view(p.dtype)[0]
        assert (bits(keys[dims:]) == bits(k[0, 0, 0, dims:])).all() and torch.isfinite(keys[:dims]).all()


ACCEPTS = [
    dict(lens=[12], new=8, paths=[[0, 2, 5]]),
    dict(lens=[12, 30, 9], new=8, paths=[[1, 2, 3, 7], [], [0, 1, 2, 3, 4, 5, 6, 7]], layout=LAYER_MAJOR, block=7),
    dict(lens=[12, 30, 9], new=8, news=[3, 8, 0], paths=[[0, 2, 5], [7], [0]]),                      # entries behind a sequence's tokens end its path
    dict(lens=[40, 40], new=9, paths=[[3, 3, 4], [2, 1, 5]]),                                        # not ascending
    dict(lens=[5], new=9, paths=[[1, 3, 5, 7, 8]]),                                                  # shorter than its new tokens
    dict(lens=[200, 150], new=130, paths=[sorted(range(0, 130, 2)), list(range(20, 120))], H=1, D=128, block=24),   # more than 32 entries
    dict(lens=[200, 150], new=100, paths=[list(range(36, 100)), list(range(32)) + [40]], H=1, D=64),
    dict(lens=[12, 30], new=8, paths=[[0, 2, 5], [4, 6]], elem=1, D=20),
    dict(lens=[12, 30], new=8, paths=[[0, 2, 5], [4, 6]], elem=4, D=7, layout=LAYER_MAJOR),
    dict(lens=[12, 30], new=8, paths=[[0, 2, 5], [4, 6]], elem=1, D=7, H=3),
    dict(lens=[12, 30], new=8, paths=[[0, 2, 5], [4, 6]], D=10),
]


@pytest.mark.parametrize("c", ACCEPTS, ids=lambda c: f"{c['lens']}-{c.get('elem', 2)}-{c.get('D', 64)}".replace(" ", ""))
@pytest.mark.parametrize("in_place", [False, True])
def test_accept(c, in_place):
    c = dict(c)
    paths, new, news = c.pop("paths"), c.pop("new"), c.pop("news", None)
    p = Pool(layers=3, **c)
    p.attends = False
    width = max(len(x) for x in paths) + 1
    path_t = torch.tensor([x + [-1] * (width - len(x)) for x in paths], dtype=torch.int32, device="cuda")
    with p.session() as s:
        lens_t = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
        got = s.accept(path_t, new_tokens=new, n_new_t=None if news is None else torch.tensor(news, dtype=torch.int32, device="cuda"), layers=(1, 3),
                       seq_len_t=lens_t if in_place else None, new_len_t=lens_t if in_place else None)
        torch.cuda.synchronize()
    want = O.accept(p.before, p.layout, p.block, p.seqs, p.lens, news or [new] * len(p.lens), paths, (1, 3))
    assert got.tolist() == want and (not in_place or got is lens_t)
    assert (p.bits.cpu().numpy() == p.before).all()


def test_append_and_accept_on_other_streams_and_in_a_graph():
    """Work before the call takes half a second: a call that does not wait for it works on old numbers."""
    p = Pool([64, 50], G=2, D=128, layers=2, q_tokens=6)
    freq = 10000.0 ** (-np.arange(64) / 64)
    rotary = Rotary(128)
    q, k, v = p.values(2, 6, 4, 128), p.values(2, 6, 2, 128), p.values(2, 6, 2, 128)
    path_t = torch.tensor([[0, 2, 5], [1, -1, -1]], dtype=torch.int32, device="cuda")
    late = [torch.zeros_like(x) for x in (q, k, v, path_t)]
    out, lens_t = torch.empty_like(q), torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with p.session() as s:
        side = torch.cuda.Stream()

        def step(stream=None):
            s.append(1, late[1], late[2], late[0], q_out_t=out, rotary=rotary, stream=stream)
            s.accept(late[3], new_len_t=lens_t, stream=stream)

        def expect(before):
            want = before.copy()
            for kv in (0, 1):                     # layer 1 of the new tokens as the append left it, checked on its own
                for r in range(2):
                    for i in range(6):
                        p.rows_at(want, 1, kv, r, p.lens[r] - 6 + i)[...] = p.rows_at(appended, 1, kv, r, p.lens[r] - 6 + i)
            lens = O.accept(want, p.layout, p.block, p.seqs, p.lens, [6, 6], [[0, 2, 5], [1]], (0, 2))
            return want, lens

        s.append(1, k, v, q, rotary=rotary)
        torch.cuda.synchronize()
        check(p, 1, every_token(p, q, k, v, 6), s.append(1, k, v, q, rotary=rotary).flatten(0, 1), rotary=rotary, frequencies=freq)
        appended = p.bits.cpu().numpy().copy()
        p.bits.copy_(torch.from_numpy(p.before))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(900_000_000)
            for a, b in zip(late, (q, k, v, path_t)):
                a.copy_(b)
        step(side.cuda_stream)
        side.synchronize()
        want, lens = expect(p.before)
        assert lens_t.tolist() == lens and (p.bits.cpu().numpy() == want).all()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for x in late:
            x.zero_()
        p.bits.copy_(torch.from_numpy(p.before))
        for a, b in zip(late, (q, k, v, path_t)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert lens_t.tolist() == lens and (p.bits.cpu().numpy() == want).all()


def test_a_session_of_the_other_type_takes_no_tokens():
    p = Pool([20], G=2, D=64)
    with p.session(num_q_heads=0, q_tokens=1, dtype=torch.float16) as s, pytest.raises(ValueError):      # (it may evict: elements are moved bit for bit)
        s.append(0, p.values(1, 1, 2, 64).half(), p.values(1, 1, 2, 64).half())
    assert (p.bits.cpu().numpy() == p.before).all()


def test_refused_tensors():
    p = Pool([20, 9], G=2, D=64, q_tokens=4)
    rotary, k, q = Rotary(64), p.values(2, 4, 2, 64), p.values(2, 4, 4, 64)
    with p.session() as s:
        def bad(*a, **kw):
            with pytest.raises(ValueError):
                s.append(0, *a, **kw)

        bad(k[:1], k[:1])
        bad(k, k[:, :3])
        bad(k.float(), k)
        bad(k.cpu(), k)
        bad(k, k, k)                                                      # as many query heads as KV heads
        bad(k, k, q_out_t=q)
        bad(k.transpose(2, 3), k)
        bad(k, k, rotary=rotary, position_t=torch.zeros(7, dtype=torch.int32, device="cuda"))
        bad(k, k, rotary=rotary, position_t=torch.zeros(8, dtype=torch.int64, device="cuda"))
        bad(k, k, position_t=torch.zeros(8, dtype=torch.int32, device="cuda"))
        bad(k, k, rotary=Rotary(64, axes=np.arange(32) % 3))
        bad(k, k, rotary=Rotary(64, device="cpu"))
        bad(k, k, k_norm_t=torch.ones(64, device="cuda", dtype=torch.bfloat16))
        bad(k, k, n_new_t=torch.zeros(3, dtype=torch.int32, device="cuda"))
        bad(k.flatten(0, 1), k.flatten(0, 1), row_begin_t=torch.zeros(2, dtype=torch.int32, device="cuda"))
        with torch.enable_grad():
            bad(k.clone().requires_grad_(), k)
        for path in (torch.zeros(2, 3, device="cuda"), torch.zeros(3, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32)):
            with pytest.raises(ValueError):
                s.accept(path)
        with pytest.raises(ValueError):
            s.accept(torch.zeros(2, 3, dtype=torch.int32, device="cuda"), layers=(1, 1))
    assert (p.bits.cpu().numpy() == p.before).all()


def test_offsets_past_32_bits():
    """A pool of 6 GB whose used blocks lie at its end: both layouts."""
    for layout in (BLOCK_MAJOR, LAYER_MAJOR):
        L, H, D, block, blocks = 2, 8, 128, 128, 6000
        geom = Geometry(layout, L, H, D, 2, block, blocks)
        pool_t = torch.zeros(geom.shape(), dtype=torch.bfloat16, device="cuda")
        tbl = np.array([blocks - 1, blocks - 3], np.int32)
        with CacheSession(geom, pool_t, Sequences([200], np.array([0, 2]), tbl), num_q_heads=8) as s:
            k, v = (torch.randn(1, 4, H, D, device="cuda").bfloat16() for _ in range(2))
            s.append(1, k, v)
            s.accept(torch.tensor([[1, 3]], dtype=torch.int32, device="cuda"), new_tokens=4)
            torch.cuda.synchronize()

        def row(kv, slot):
            b, tt = int(tbl[slot // block]), slot % block
            return pool_t[b, 1, kv, tt] if layout == BLOCK_MAJOR else pool_t[1, kv, b, :, tt]

        for kv, x in ((0, k), (1, v)):
            for slot, i in ((196, 1), (197, 3), (198, 2), (199, 3)):
                assert torch.equal(row(kv, slot), x[0, i]), (layout, kv, slot)
                row(kv, slot).zero_()
        assert not pool_t.view(torch.int16).any()
        del pool_t


def test_queries_in_place_in_a_fused_buffer():
    p = Pool([40, 23], G=2, D=64)
    freq = 10000.0 ** (-np.arange(32) / 32)
    fused = p.values(2, 3, 8 * 64)
    before = fused.clone()
    cut = lambda x: [y.unflatten(-1, (-1, 64)) for y in x.split([256, 128, 128], -1)]  # noqa: E731
    q, k, v = cut(fused)
    with p.session() as s:
        assert s.append(1, k, v, q, q_out_t=q, rotary=Rotary(64)) is q
        torch.cuda.synchronize()
    check(p, 1, every_token(p, *cut(before), 3), q.flatten(0, 1), rotary=Rotary(64), frequencies=freq)
    assert torch.equal(fused[..., 256:], before[..., 256:])


def test_nothing_to_append_and_empty_paths():
    p = Pool([20, 9], G=2, D=64, q_tokens=4)
    with p.session() as s:
        assert s.append(0, p.values(2, 0, 2, 64), p.values(2, 0, 2, 64), p.values(2, 0, 4, 64)).shape == (2, 0, 4, 64)
        none = torch.zeros(2, dtype=torch.int32, device="cuda")
        s.append(0, p.values(2, 4, 2, 64), p.values(2, 4, 2, 64), n_new_t=none)
        s.append(0, p.values(0, 2, 64), p.values(0, 2, 64), row_begin_t=torch.zeros(3, dtype=torch.int32, device="cuda"))
        assert s.accept(torch.zeros(2, 0, dtype=torch.int32, device="cuda")).tolist() == [16, 5]
        assert s.accept(torch.tensor([[0], [0]], dtype=torch.int32, device="cuda"), n_new_t=none).tolist() == [20, 9]
        torch.cuda.synchronize()
    assert (p.bits.cpu().numpy() == p.before).all()
