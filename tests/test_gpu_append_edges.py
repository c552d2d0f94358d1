"""Appending and accepting at the ends of what a call allows, on the GPU."""
import pytest
import torch

from paper_2408_08147_b200 import binding as B
from test_gpu_append import Pool

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
