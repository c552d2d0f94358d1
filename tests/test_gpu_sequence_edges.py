"""Corners of attention, accumulated weights and eviction on the GPU."""
import numpy as np
import pytest
import torch

from paper_2408_08147_b200.sequences import CacheSession
from test_gpu_sequences import Evict, Setup

pytestmark = pytest.mark.gpu


def not_given_away(make):
    """The memory of the tensors that `make` gives up is not handed out while the stream that uses it is busy."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)      # a fifth of a second
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
