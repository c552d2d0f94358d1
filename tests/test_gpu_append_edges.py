"""Appending and accepting at the ends of what a call allows, on the GPU."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200.sequences import pack_mask
from test_gpu_append import Pool
from test_gpu_forms import tree
from test_gpu_sequence_edges import cached_row
from test_gpu_sequences import Setup, check, check_scores

pytestmark = pytest.mark.gpu


def reported(s):
    with pytest.raises(B.PdkvError) as e:
        s.status()
    s.status()                       # once
    return e.value.status


def test_lengths_above_the_handles_are_reported():
    """There is no place for a token behind the handle's length: the call cannot say so itself, the handle's status does."""
    p = Pool([40, 9], G=2, D=64, q_tokens=2)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, path = p.values(2, 2, 2, 64), ints([1], [0])
    with p.session() as s:
        for lens in ((40, 9), (3, 0), (0, -5)):
            s.append(0, k, k, seq_len_t=ints(*lens))
            s.accept(path, seq_len_t=ints(*lens))
            s.status()
        for lens in ((40, 10), (41, 9), (1 << 30, 9)):
            s.append(1, k, k, seq_len_t=ints(*lens))
            assert reported(s) == B.PDKV_ERR_TABLE
            s.append(0, k.flatten(0, 1), k.flatten(0, 1), row_begin_t=ints(0, 2, 4), seq_len_t=ints(*lens))
            assert reported(s) == B.PDKV_ERR_TABLE
            s.accept(path, seq_len_t=ints(*lens))
            assert reported(s) == B.PDKV_ERR_TABLE
        s.append(0, k, k, n_new_t=ints(2, 0), seq_len_t=ints(40, 10))       # nothing new for the one that is too long
        s.status()


def test_a_counter_that_runs_past_the_handles_length_is_reported():
    p = Pool([12], G=1, D=64)
    k, lens = p.values(1, 1, 2, 64), torch.tensor([10], dtype=torch.int32, device="cuda")
    with p.session() as s:
        s.append(0, k, k, seq_len_t=lens)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.append(0, k, k, seq_len_t=lens)
            lens.add_(1)
        for _ in range(3):           # 10, 11, 12
            graph.replay()
        s.status()
        graph.replay()
        assert reported(s) == B.PDKV_ERR_TABLE


def test_trees_with_weights_accepted_then_evicted():
    """append a tree, attend with weights, accept, move the weights, evict, and decode over what is left: the kept tokens are those that weighed most."""
    Q, own = 8, [150, 97]
    s = Setup([n + Q for n in own], H=2, G=2, D=64, Q=Q, layers=1, layer=0)
    rng = np.random.default_rng(5)
    see = np.stack([tree(rng, Q, Q)[0] for _ in own])
    paths = [np.flatnonzero(see[0, Q - 1]).tolist(), np.flatnonzero(see[1, Q - 2]).tolist()]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    path_t = ints([p + [-1] * (Q - len(p)) for p in paths])
    k, v, q = (torch.from_numpy(rng.standard_normal((2, Q, h, 64)) * 1.5).to(s.dtype).cuda() for h in (2, 2, 4))
    scores = torch.zeros(1, 2, 2, max(s.lens), device="cuda")
    budget = 40
    with s.session() as x:
        q = x.append(0, k, v, q)
        out, lse = x.attend(0, q, scores_t=scores[0], mask_t=pack_mask(torch.from_numpy(see).cuda()))
        want = O.attend_formed(s.pool_t.double().cpu().numpy(), s.layout, s.block, 0, s.seqs, s.lens, q.double().cpu().numpy(), 2, 64 ** -0.5, see=see)
        check(s, out, lse, want)
        check_scores(s, np.zeros(scores[0].shape), scores[0], want, s.lens)
        lens_t = x.accept(path_t)
        lens = [n + len(p) for n, p in zip(own, paths)]
        assert lens_t.tolist() == lens
        for r, (n, p) in enumerate(zip(own, paths)):
            scores[0, r, :, n:n + len(p)] = scores[0, r, :, [n + i for i in p]]
            scores[0, r, :, n + len(p):] = 0
        before = s.pool_t.clone()
        kept, _, new_len = x.evict(x, scores, budget, sink=2, recent=4, seq_len_t=lens_t)
        x.status()
        host = scores[0].cpu().numpy()
        for r, n in enumerate(own):
            for h in range(2):
                ids = kept[0, r, h].tolist()
                assert ids == O.select(host[r, h, :lens[r]], budget, 2, 4).tolist()
                for kv, new in ((0, k), (1, v)):
                    after = torch.stack([cached_row(s, r, i, kv, h).clone() for i in range(budget)])
                    keep, s.pool_t = s.pool_t, before
                    old = torch.stack([cached_row(s, r, t, kv, h).clone() for t in ids])
                    s.pool_t = keep
                    assert torch.equal(after, old)
                    for t, row in zip(ids, old):
                        if t >= n:           # an accepted node
                            assert torch.equal(row, new[r, paths[r][t - n], h])
        # one more token behind what is left
        one = ints([1, 1])
        q1 = x.append(0, k[:, :1], v[:, :1], q[:, :1], seq_len_t=new_len + 1)
        wide = torch.zeros_like(q)
        wide[:, :1] = q1
        got = x.attend(0, wide, seq_len_t=new_len + 1, n_new_t=one)
        left = O.attend_formed(s.pool_t.double().cpu().numpy(), s.layout, s.block, 0, s.seqs, [budget + 1] * 2, wide.double().cpu().numpy(), 2, 64 ** -0.5, news=[1, 1])
        check(s, *got, left)
