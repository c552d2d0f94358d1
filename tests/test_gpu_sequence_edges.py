"""Corners of attention, accumulated weights and eviction on the GPU."""
import numpy as np
import pytest
import torch

from paper_2408_08147_b200.sequences import CacheSession, Sequences
from paper_2408_08147_b200.workloads import LAYER_MAJOR, Geometry
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
