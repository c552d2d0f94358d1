"""Corners of the handles of cached sequences and of their calls without a GPU."""
import numpy as np
import pytest
import torch

from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200 import workloads as W
from paper_2408_08147_b200.sequences import CacheSession, Sequences
from test_sequences_host import FAKE, args, built, create, csr, pool, status  # noqa: F401 (`built` is a fixture)


def test_row_counts_past_32_and_64_bits():
    """q_tokens x num_q_heads x n_seq is limited whatever it would wrap to (2^31 - 1, 2^31 - 4 and 4: below zero)."""
    p = pool()
    for lens, Hq, Q in (([4] * 4, 2 ** 31 - 4, 2 ** 31 - 1), ([4] * 8, 2 ** 30, 2 ** 31 - 1), ([4], 2 ** 30, 2 ** 30),
                        ([4] * 3, 4, 1 << 27), ([], 4, (1 << 28) + 1)):
        assert status(create, p, lens, Hq=Hq, q_tokens=Q) == B.PDKV_ERR_INVALID_ARG


def test_offsets_are_checked_before_ids_are_read():
    """Offsets that rise past the table's end and fall back to it: refused before an id behind the end is looked at (there is
    no table here at all, which would be INVALID_ARG)."""
    off = np.array([0, 10, 5], np.int64)
    assert status(B.pdkv_seqs_create, pool(), [160, 0], off, None, num_q_heads=8, q_tokens=1) == B.PDKV_ERR_TABLE
    off, tbl = csr([40, 7], 16)
    assert status(B.pdkv_seqs_create, pool(), [40, 7], off, tbl, prefix_len=[160, 0], prefix_tbl_off=np.array([0, 10, 5], np.int64), prefix_tbl=None,
                  seq_prefix=[0, 1], num_q_heads=8, q_tokens=1) == B.PDKV_ERR_TABLE


def test_what_attention_writes_lies_apart():
    """out, lse, scores_out and scratch on one another and on q, pool, lengths and scores_in: refused.  The scratch is a byte
    short, which is noticed after that."""
    p = pool()
    s, _ = create(p, [40, 7], q_tokens=2)
    n = B.pdkv_attend_scratch(s, True) - 1
    rows, scores = 2 * 2 * 2 * 8 * 64, 4 * (160 + 3 * 40 + 40)
    at = {k: (FAKE + (i << 40), size) for i, (k, size) in enumerate(
        dict(pool=B.pdkv_pool_bytes(B.make_desc(0, 2, 4, 64, 2, 16, 400)), q=rows, out=rows, lse=4 * 2 * 2 * 8, scores_out=scores, scores_in=scores,
             seq_len=8, scratch=n).items())}

    def call(**over):
        kw = {k: v for k, (v, _) in at.items() if k not in ("pool", "scratch")}
        kw.update(scores_out_stride=[160, 40], scores_in_stride=[160, 40])
        kw.update(over)
        scratch = kw.pop("scratch", at["scratch"][0])
        return status(B.pdkv_attend, s, 0, args(Q=2, **kw), scratch, n)

    assert call() == B.PDKV_ERR_BUFFER_TOO_SMALL
    assert call(scores_in=at["scores_out"][0]) == B.PDKV_ERR_BUFFER_TOO_SMALL
    for w in ("out", "lse", "scores_out", "scratch"):
        for r in at:
            if r == w or (w, r) == ("scores_out", "scores_in"):
                continue
            for spot in (at[r][0], at[r][0] + at[r][1] - 32 if r != "seq_len" else at[r][0]):   # its first and its last bytes
                spot -= spot % 32
                assert call(**{w: spot}) == B.PDKV_ERR_INVALID_ARG, (w, r)
            assert call(**{w: at[r][0] + (at[r][1] + 31) // 32 * 32}) == B.PDKV_ERR_BUFFER_TOO_SMALL, (w, r)   # right behind it
    assert call(scores_out=at["scores_in"][0] + 32) == B.PDKV_ERR_INVALID_ARG
    # views of one buffer that lie between one another: q and out, scores and their input
    buf = at["q"][0]
    wide = dict(q_stride=[4 * 512, 2 * 512, 64], out_stride=[4 * 512, 2 * 512, 64])
    assert call(out=buf + 2 * 512, **wide) == B.PDKV_ERR_BUFFER_TOO_SMALL
    assert call(out=buf + 2 * 448, **wide) == B.PDKV_ERR_INVALID_ARG
    both = dict(scores_in_stride=[320, 80], scores_out_stride=[320, 80])
    assert call(scores_in=at["scores_out"][0] + 160, **both) == B.PDKV_ERR_BUFFER_TOO_SMALL
    assert call(scores_in=at["scores_out"][0] + 156, **both) == B.PDKV_ERR_INVALID_ARG


def evict_args(**over):
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
    return a


def test_budgets_that_32_bit_indices_do_not_hold():
    """A kernel's index runs a block's threads past the last entry of a row of the budget: at 2^31 - 1 it would wrap."""
    s = create(pool(), [40, 7], Hq=0)[0]
    for over in (dict(budget=2 ** 31 - 1, kept_scores_len=40), dict(budget=2 ** 30 + 1, kept_scores_len=40),
                 dict(kept_scores_len=2 ** 31 - 1, kept_scores_stride=[1 << 36, 1 << 34, 1 << 32]),
                 dict(kept_scores_len=2 ** 30 + 1, kept_scores_stride=[1 << 36, 1 << 34, 1 << 32])):
        assert status(B.pdkv_evict, s, s, 0, 2, evict_args(kept_scores=FAKE + (1 << 45), **over)) == B.PDKV_ERR_LIMIT
    assert status(B.pdkv_evict, s, s, 0, 2, evict_args(budget=2 ** 30, kept_scores=0)) == B.PDKV_ERR_INVALID_ARG   # (a host-only handle)


def test_what_eviction_writes_lies_apart():
    """kept, kept_scores and new_len on one another, on scores, lengths and pools: refused; in place: taken.  The budget is over
    the limit, which is noticed after that."""
    def make(base):
        return create(pool(H=4, base=base), [40, 7], Hq=0)[0]

    far, budget = 1 << 44, 2 ** 30 + 1
    s, d = make(FAKE), make(FAKE + far)
    nbytes, scores = B.pdkv_pool_bytes(B.make_desc(0, 2, 4, 64, 2, 16, 400)), 4 * (400 + 200 + 3 * 50 + 40)
    at = {k: (FAKE + (i << 41), size) for i, (k, size) in enumerate(
        dict(src=nbytes, scores=scores, kept_scores=scores, new_len=8, seq_len=8, kept=4 * 2 * 2 * 4 * budget).items())}
    at["dst"] = (FAKE + far, nbytes)

    def call(dst=d, **over):
        kw = {k: v for k, (v, _) in at.items() if k not in ("src", "dst")}
        kw.update(budget=budget, kept_scores_len=40)
        kw.update(over)
        return status(B.pdkv_evict, s, dst, 0, 2, evict_args(**kw))

    assert call() == B.PDKV_ERR_LIMIT and call(dst=s) == B.PDKV_ERR_LIMIT
    assert call(kept_scores=at["scores"][0], new_len=at["seq_len"][0]) == B.PDKV_ERR_LIMIT
    assert call(kept_scores=0, new_len=0, seq_len=0) == B.PDKV_ERR_LIMIT
    for w in ("kept", "kept_scores", "new_len"):
        for r in at:
            if r == w or (w, r) in (("kept_scores", "scores"), ("new_len", "seq_len")):
                continue
            assert call(**{w: at[r][0]}) == B.PDKV_ERR_INVALID_ARG, (w, r)
            assert call(**{w: at[r][0] + at[r][1] - 4}) == B.PDKV_ERR_INVALID_ARG, (w, r)
            assert call(**{w: at[r][0] + (at[r][1] + 3) // 4 * 4}) == B.PDKV_ERR_LIMIT, (w, r)
    assert call(kept_scores=at["scores"][0] + 4) == B.PDKV_ERR_INVALID_ARG and call(new_len=at["seq_len"][0] + 4) == B.PDKV_ERR_INVALID_ARG
    for r in ("scores", "seq_len"):
        assert call(**{r: at["dst"][0] + 64}) == B.PDKV_ERR_INVALID_ARG, r
    # rows of one buffer that lie between one another
    wide = dict(scores_stride=[800, 400, 100], kept_scores_stride=[800, 400, 100])
    assert call(kept_scores=at["scores"][0] + 4 * 40, **wide) == B.PDKV_ERR_LIMIT
    assert call(kept_scores=at["scores"][0] + 4 * 39, **wide) == B.PDKV_ERR_INVALID_ARG


def test_unaligned_buffers_of_eviction():
    """Of every buffer, and also where no sequence has a token."""
    for lens in ([40, 7], [0, 0]):
        s = create(pool(H=4), lens, Hq=0)[0]
        for over in (dict(scores=FAKE + (1 << 41) + 2), dict(kept=FAKE + (2 << 41) + 1), dict(kept_scores=FAKE + (3 << 41) + 2),
                     dict(seq_len=FAKE + (4 << 41) + 2), dict(new_len=FAKE + (5 << 41) + 2), dict(kept=0),
                     dict(kept_scores_len=-1), dict(kept_scores_stride=[400, 200, 10])):
            over = {"budget": 2 ** 30 + 1, "kept_scores": 0, **over}     # (over the limit: noticed after that)
            if "kept_scores_len" in over or "kept_scores_stride" in over:
                over["kept_scores"] = FAKE + (1 << 45)
            assert status(B.pdkv_evict, s, s, 0, 2, evict_args(**over)) == B.PDKV_ERR_INVALID_ARG, (lens, over)
    assert status(B.pdkv_evict, s, s, 0, 2, evict_args(budget=2 ** 30 + 1, scores=0, kept_scores=0)) == B.PDKV_ERR_LIMIT


def test_scales_that_overflow_in_base_2():
    """Logits are kept in base 2: a scale that is finite alone, but not times log2(e), is refused."""
    s, _ = create(pool(), [40, 7])
    for scale, want in ((2.3e38, B.PDKV_ERR_BUFFER_TOO_SMALL), (2.4e38, B.PDKV_ERR_INVALID_ARG), (-3e38, B.PDKV_ERR_INVALID_ARG)):
        assert status(B.pdkv_attend, s, 0, args(scale=scale, scores_out=FAKE + (5 << 40), scores_out_stride=[160, 40]), FAKE + (3 << 40), 0) == want


def cpu_session(held=torch.bfloat16, **kw):
    """A session over host memory: its handle can be asked, not launched."""
    geom = W.Geometry(W.BLOCK_MAJOR, 2, 4, 64, 2, 16, 8)
    off, tbl = csr([40, 7], 16)
    kw = {"num_q_heads": 8, **kw}
    return CacheSession(geom, torch.zeros(geom.shape(), dtype=held), Sequences([40, 7], off, tbl), **kw)


def test_queries_that_ask_for_a_gradient():
    with cpu_session() as c:
        q = torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16, requires_grad=True)
        with pytest.raises(ValueError, match="gradient"):
            c.attend(0, q)
        with torch.no_grad(), pytest.raises(B.PdkvError):      # (a host-only handle)
            c.attend(0, q)
        with pytest.raises(B.PdkvError):
            c.attend(0, q.detach())


def test_type_of_the_pool():
    """16-bit words can be declared to be either type; a tensor of one type cannot be the other."""
    for held, named in ((torch.bfloat16, torch.float16), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float32)):
        with pytest.raises(ValueError):
            cpu_session(held, dtype=named)
    for held, named in ((torch.int16, torch.float16), (torch.float16, None), (torch.float16, torch.float16)):
        with cpu_session(held, dtype=named) as c:
            assert c.dtype == torch.float16
    cpu_session(torch.float16, dtype=torch.bfloat16, num_q_heads=0).close()     # rows are moved as they are


def test_ranges_of_layers_to_evict():
    """An empty range would return lengths that nobody wrote."""
    with cpu_session(num_q_heads=0) as c:
        for layers in ((1, 1), (0, 0), (1, 0), (-1, 1), (0, 3)):
            with pytest.raises(ValueError, match="layers"):
                c.evict(c, torch.zeros(max(0, layers[1] - layers[0]), 2, 4, 40), 8, layers=layers)
