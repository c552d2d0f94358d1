"""Handles of cached sequences without a GPU: refusals, and the attention work list."""
import numpy as np
import pytest

from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200 import build as pdkv_build
from paper_2408_08147_b200 import workloads as W

FAKE = 0x7F0000000000


@pytest.fixture(scope="module", autouse=True)
def built():
    pdkv_build.build_library()
    B.pdkv_tune("dry_run", 1)
    yield
    B.pdkv_tune("dry_run", 0)


def pool(H=4, D=64, E=2, block=16, blocks=400, layers=2, layout=0, base=FAKE):
    d = B.make_desc(layout, layers, H, D, E, block, blocks)
    return B.pdkv_pool_create(d, base, B.pdkv_pool_bytes(d), 0)


def csr(lens, block, first=0):
    n = [-(-x // block) for x in lens]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
    return off, (first + np.arange(off[-1])).astype(np.int32)


def create(p, lens, block=16, Hq=8, q_tokens=1, dtype=0, **kw):
    off, tbl = csr(lens, block)
    return B.pdkv_seqs_create(p, lens, kw.pop("off", off), kw.pop("tbl", tbl), num_q_heads=Hq, q_tokens=q_tokens, dtype=dtype, **kw)


def status(fn, *a, **kw):
    with pytest.raises(B.PdkvError) as e:
        fn(*a, **kw)
    return e.value.status


def test_refused_descriptions():
    p = pool()
    assert status(create, p, [5, -1]) == B.PDKV_ERR_INVALID_ARG
    assert status(create, p, [40], tbl=np.array([0, 1, 400], np.int32)) == B.PDKV_ERR_TABLE
    assert status(create, p, [40], tbl=np.array([0, -1, 3], np.int32)) == B.PDKV_ERR_TABLE
    assert status(create, p, [40], off=np.array([0, 2], np.int64)) == B.PDKV_ERR_TABLE
    assert status(create, p, [40], off=np.array([-1, 3], np.int64)) == B.PDKV_ERR_TABLE
    assert status(create, p, [(1 << 30) + 1], off=np.array([0, 1 << 27], np.int64)) == B.PDKV_ERR_LIMIT
    assert status(create, p, [4], Hq=6) == B.PDKV_ERR_GEOMETRY          # not a multiple of the KV heads
    assert status(create, p, [4], q_tokens=0) == B.PDKV_ERR_INVALID_ARG
    assert status(create, p, [4], dtype=2) == B.PDKV_ERR_INVALID_ARG
    for kw in (dict(E=1), dict(E=4), dict(D=60), dict(D=264)):
        assert status(create, pool(**kw), [4]) == B.PDKV_ERR_GEOMETRY
        create(pool(**kw), [4], Hq=0)                                   # such pools can be evicted from
    pre = dict(prefix_len=[20], prefix_tbl_off=[0, 2], prefix_tbl=[50, 51])
    assert status(create, p, [4], seq_prefix=[1], **pre) == B.PDKV_ERR_INVALID_ARG
    assert status(create, p, [4], seq_prefix=[-2], **pre) == B.PDKV_ERR_INVALID_ARG
    assert status(create, p, [4], seq_prefix=None, **pre) == B.PDKV_ERR_INVALID_ARG
    assert status(create, p, [4], seq_prefix=[0], prefix_len=[33], prefix_tbl_off=[0, 2], prefix_tbl=[50, 51]) == B.PDKV_ERR_TABLE


def test_workspace_size_is_reported():
    p = pool()
    off, tbl = csr([40, 7], 16)
    need = create(p, [40, 7])[1]
    with pytest.raises(B.PdkvError) as e:
        B.pdkv_seqs_create(p, [40, 7], off, tbl, num_q_heads=8, q_tokens=1, workspace_ptr=FAKE, workspace_bytes=need - 1)
    assert e.value.status == B.PDKV_ERR_BUFFER_TOO_SMALL and e.value.needed_bytes == need
    assert status(B.pdkv_seqs_create, p, [40], off, tbl, num_q_heads=8, q_tokens=1, workspace_ptr=FAKE + 8,
                  workspace_bytes=1 << 20) == B.PDKV_ERR_INVALID_ARG


def args(n=2, Q=1, Hq=8, D=64, **over):
    a = B.pdkv_attend_args()
    a.q, a.out, a.scale = FAKE + (1 << 40), FAKE + (2 << 40), 0.125
    a.q_stride[:] = [Q * Hq * D, Hq * D, D]
    a.out_stride[:] = [Q * Hq * D, Hq * D, D]
    for k, v in over.items():
        if k.endswith("stride"):
            getattr(a, k)[:] = v
        else:
            setattr(a, k, v)
    return a


def test_refused_attention_calls():
    p = pool()
    s, _ = create(p, [40, 7], q_tokens=2)
    n = B.pdkv_attend_scratch(s, True)

    def call(layer=0, scratch=FAKE + (3 << 40), nbytes=n, h=s, **over):
        return status(B.pdkv_attend, h, layer, args(Q=2, **over), scratch, nbytes)

    bad = B.PDKV_ERR_INVALID_ARG
    assert call(layer=2) == bad and call(layer=-1) == bad
    assert call(q=0) == bad and call(out=0) == bad
    assert call(q=FAKE + (1 << 40) + 8) == bad and call(out=FAKE + (2 << 40) + 2) == bad
    assert call(scale=float("nan")) == bad and call(scale=float("inf")) == bad
    assert call(out_stride=[1024, 512, 60]) == bad                       # alignment
    assert call(out_stride=[1024, 512, 32]) == bad                       # heads overlap
    assert call(out_stride=[512, 512, 64]) == bad                        # sequences overlap
    assert call(out=FAKE) == bad                                         # on the pool
    assert call(out=FAKE + (1 << 40) + 256) == bad                       # on q
    assert call(out=FAKE + (3 << 40)) == bad                             # on the scratch
    assert call(scores_in=FAKE + (4 << 40)) == bad                       # nowhere to put the sums
    sc = dict(scores_out=FAKE + (5 << 40), scores_out_stride=[160, 40])
    assert call(scores_out=FAKE + (5 << 40), scores_out_stride=[160, 39]) == bad     # rows overlap
    assert call(scores_in=FAKE + (5 << 40), scores_in_stride=[160, 41], **sc) == bad  # in place, other strides
    assert call(scores_in=FAKE + (5 << 40) + 160, scores_in_stride=[160, 40], **sc) == bad  # shifted onto itself
    assert call(scratch=0) == bad
    assert call(nbytes=n - 1, **sc) == B.PDKV_ERR_BUFFER_TOO_SMALL
    assert call(**sc) == bad                                             # a host-only handle cannot be launched
    none, _ = create(p, [40, 7], Hq=0)
    assert call(h=none) == bad
    assert status(B.pdkv_attend_scratch, none, False) == bad


def test_refused_evictions():
    def make(lens, H=4, D=64, base=FAKE, **kw):
        return create(pool(H=H, D=D, base=base), lens, Hq=0, **kw)[0]

    def call(s, d, layers=(0, 2), **over):
        a = B.pdkv_evict_args()
        a.budget, a.sink, a.recent = 16, 2, 3
        a.scores, a.kept, a.kept_scores = FAKE + (1 << 41), FAKE + (2 << 41), FAKE + (3 << 41)
        a.scores_stride[:] = [400, 200, 50]
        a.kept_scores_stride[:] = [400, 200, 50]
        a.kept_scores_len = 16
        for k, v in over.items():
            if k.endswith("stride"):
                getattr(a, k)[:] = v
            else:
                setattr(a, k, v)
        return status(B.pdkv_evict, s, d, *layers, a)

    bad = B.PDKV_ERR_INVALID_ARG
    s, far = make([40, 7]), 1 << 40
    d = make([16, 7], base=FAKE + far)
    assert call(s, d) == bad                                             # host-only handles: everything else was in order
    assert call(s, d, layers=(0, 3)) == bad and call(s, d, layers=(1, 0)) == bad
    assert call(s, d, budget=4) == bad and call(s, d, sink=-1) == bad and call(s, d, recent=-1) == bad
    assert call(s, d, budget=0, sink=0, recent=0) == bad
    assert call(s, make([16], base=FAKE + far)) == bad                   # other number of sequences
    assert call(s, make([16, 7])) == bad                                 # another handle on the same memory
    assert call(s, make([15, 7], base=FAKE + far)) == B.PDKV_ERR_TABLE   # no room
    assert call(s, make([16, 7], H=2, base=FAKE + far)) == B.PDKV_ERR_GEOMETRY
    assert call(s, make([16, 7], D=32, base=FAKE + far)) == B.PDKV_ERR_GEOMETRY
    assert call(s, make([16, 7], base=FAKE + far, tbl=np.array([3, 3], np.int32))) == B.PDKV_ERR_TABLE
    twice = make([40, 7], tbl=np.array([0, 1, 2, 0], np.int32))
    assert call(twice, twice) == B.PDKV_ERR_TABLE                        # in place with a shared block
    assert call(s, d, kept=0) == bad and call(s, d, scores=0) == bad
    assert call(s, d, kept=FAKE + (1 << 41) + 64) == bad                  # on the scores
    assert call(s, d, kept=FAKE + (3 << 41) + 64) == bad                  # on the scores that are kept
    assert call(s, d, kept_scores_len=15) == bad
    assert call(s, d, kept_scores_stride=[400, 200, 15]) == bad
    assert call(s, d, kept_scores=FAKE + (1 << 41), kept_scores_stride=[400, 200, 40]) == bad
    assert call(s, d, kept_scores=FAKE + (1 << 41) + 4) == bad


def cover(s, H, lens, prefix_len, seq_prefix, rows):
    """Every (head, row, token) of every segment lies in exactly one item; CTAs in order."""
    items = B.pdkv_seqs_items(s)
    for kernel in (0, 1):
        assert (np.diff(items["cta"][items["kernel"] == kernel]) >= 0).all()
    todo = {("s", r): (n, rows) for r, n in enumerate(lens)}
    for p, n in enumerate(prefix_len):
        todo["p", p] = (n, rows * sum(x == p for x in seq_prefix))
    for (kind, i), (n, n_rows) in todo.items():
        seen = np.zeros((H, n_rows, n), np.int32)
        for it in items[items["seq"] == i] if kind == "s" else items[items["prefix"] == i]:
            assert 0 <= it["row_begin"] < it["row_end"] <= n_rows and 0 <= it["tok_begin"] < it["tok_end"] <= n
            assert it["row_end"] - it["row_begin"] <= 256
            seen[it["head"], it["row_begin"]:it["row_end"], it["tok_begin"]:it["tok_end"]] += 1
        assert (seen == 1).all(), (kind, i)
    return items


@pytest.mark.parametrize("H,G,Q,block,lens,prefix_len,seq_prefix", [
    (4, 2, 1, 16, [300], [], []),
    (4, 2, 1, 16, [1, 0, 17, 64, 65, 2000], [], []),
    (1, 1, 1, 7, [5], [], []),
    (2, 8, 3, 16, [63, 1, 700], [129, 0, 64], [0, 2, 0]),
    (8, 4, 1, 128, [2048] * 32, [], []),
    (3, 5, 4, 32, [10] * 40, [1000, 333], [i % 2 for i in range(40)]),
    (8, 16, 1, 16, [33] * 7, [4096], [0, 0, -1, 0, 0, 0, 0]),
    (2, 2, 1, 16, [], [40], []),
    (2, 2, 1, 16, [0, 0], [], []),
])
def test_work_items_cover_everything_once(H, G, Q, block, lens, prefix_len, seq_prefix):
    p = pool(H=H, block=block, blocks=1200)
    kw = {}
    if prefix_len:
        off, tbl = csr(prefix_len, block, first=sum(-(-x // block) for x in lens))
        kw = dict(prefix_len=prefix_len, prefix_tbl_off=off, prefix_tbl=tbl, seq_prefix=np.array(seq_prefix, np.int32))
    s, _ = create(p, lens, block=block, Hq=H * G, q_tokens=Q, **kw)
    cover(s, H, lens, prefix_len, seq_prefix, G * Q)


def test_work_items_random():
    rng = np.random.default_rng(5)
    for _ in range(40):
        H, G, Q = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 4, 7])), int(rng.choice([1, 2, 5]))
        n = int(rng.integers(1, 30))
        lens = [int(x) for x in rng.integers(0, rng.choice([3, 100, 900]), size=n)]
        P = int(rng.integers(0, 4))
        plen = [int(x) for x in rng.integers(0, 1500, size=P)]
        member = [int(x) for x in rng.integers(-1, P, size=n)] if P else []
        kw = {}
        if P:
            off, tbl = csr(plen, 16)
            kw = dict(prefix_len=plen, prefix_tbl_off=off, prefix_tbl=tbl, seq_prefix=np.array(member, np.int32))
        s, _ = create(pool(H=H, blocks=4000), lens, Hq=H * G, q_tokens=Q, **kw)
        cover(s, H, lens, plen, member, G * Q)


def test_items_share_the_work_evenly():
    """Ragged lengths: no CTA gets more than its share of token quanta plus the cut's granularity."""
    lens = W.draw_lengths("lognormal", 64, 5, median=1024, sigma=0.8, lo=16, hi=8192)
    s, _ = create(pool(H=8, D=128, blocks=8000), [int(x) for x in lens], Hq=32)
    it = B.pdkv_seqs_items(s)
    cost = np.bincount(it["cta"], weights=np.ceil((it["tok_end"] - it["tok_begin"]) / 64))
    assert cost.max() <= cost.mean() * 1.1 + 2
