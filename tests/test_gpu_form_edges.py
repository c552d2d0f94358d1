"""Attention in other forms than plain causal, at the ends of what a call allows, on the GPU."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2408_08147_b200.workloads import LAYER_MAJOR
from test_gpu_forms import KERNELS, Form
from test_gpu_sequence_edges import cached_row
from test_gpu_sequences import Setup, check, check_scores

pytestmark = pytest.mark.gpu


def expect(s, f, scale=None):
    """As Form.expect, but of a capped logit that is off by a part of itself, not of the cap.  Up to 0.65 of the cap: the polynomial is off by 2^-22.6, its
    five coefficients, the factor and the steps, whose terms alternate and sum to at most 1.3 of the result, round by less than 8 * 2^-24, together
    below 2^-20.  Above: 2^-22 of the cap by the exponential, the reciprocal and three roundings, the cap at most 1 / 0.57 of the logit: below 2^-21."""
    q = s.q_t.double().cpu().numpy()
    out, lse, w, e = O.attend_formed(s.pool_t.double().cpu().numpy(), s.layout, s.block, s.layer, s.seqs, s.lens, q, s.H, s.D ** -0.5 if scale is None else scale,
                                     f.cap, f.slopes, f.see, f.news, f.offset)
    e["z"] = e["z"] * (1 + 2.0 ** -20 / (4 * 2.0 ** -24)) + e["bias"] * 6 / 4
    return out, lse, w, e


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
@pytest.mark.parametrize("cap", [3e-3, 11.0, 1e3, 1e4, 1e5, 1e6, 1e7, 1e12, 1e38])
@pytest.mark.parametrize("slopes", [False, True], ids=["capped", "biased"])
def test_caps_of_every_size(c, cap, slopes):
    """A cap far above the logits changes next to nothing: what it does must not be lost in an error that grows with it."""
    s = Setup(**c)
    f = Form(s, kind="tree", cap=cap, slopes=slopes, ragged=True)
    scores = torch.rand(2, s.H, max(s.lens), device="cuda")
    before = scores.double().cpu().numpy()
    with s.session() as x:
        got = x.attend(s.layer, s.q_t, scores_t=scores, **f.kw)
        x.status()
    want = expect(s, f)
    check(s, *got, want)
    check_scores(s, before, scores, want, s.lens)


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_large_caps_and_scales(c, scale):
    s = Setup(**c)
    f = Form(s, kind="tree", cap=1e6, ragged=True)
    with s.session() as x:
        check(s, *x.attend(s.layer, s.q_t, scale=scale, **f.kw), expect(s, f, scale))


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
@pytest.mark.parametrize("scale", [0.2, -0.2])
def test_large_caps_beside_infinite_values(c, scale):
    """What the pieces of V that hold values that are not finite add is found apart from the products; their other dims are finite."""
    s = Setup(**c)
    f = Form(s, kind="tree", cap=1e6)
    for r, n in enumerate(s.lens):
        cached_row(s, r, n - s.Q, 1, 0)[0] = float("inf")     # of the root, which every node sees
        cached_row(s, r, n - 1, 1, 0)[0] = float("nan")       # of the last node, which it alone sees
    with s.session() as x:
        out, lse = x.attend(s.layer, s.q_t, scale=scale, **f.kw)
        x.status()
    assert torch.isposinf(out[:, :-1, :s.G, 0]).all() and torch.isnan(out[:, -1, :s.G, 0]).all()
    y, want_lse, w, e = expect(s, f, scale)
    e["mag"] = (e["mag"] + np.abs(y))[..., 1:]                # (a direct result is rounded once more)
    check(s, out[..., 1:], lse, (y[..., 1:], want_lse, w, e))


@pytest.mark.parametrize("form", [dict(kind="tree"), dict(kind="tree", cap=2.0), dict(kind="tree", cap=30.0), dict(kind="tree", slopes=True), dict(kind="any", cap=30.0, slopes=True)],
                         ids=["masked", "small cap", "capped", "biased", "both"])
@pytest.mark.parametrize("c", [dict(lens=[40, 13, 70], G=2, Q=2), dict(lens=[40, 13, 70], G=2, Q=8, D=256), dict(lens=[150, 90, 33], G=4, D=128, Q=5, layout=LAYER_MAJOR)],
                         ids=["warp", "warp, many rows", "tile"])
def test_bits_do_not_depend_on_other_sequences(c, form):
    """Rows of several sequences behind one prefix share the work of a warp, not what is computed: what one sequence asks changes no bit of another's."""
    s = Setup(**c, prefix_len=[900], member=[0, 0, 0])
    f = Form(s, **form)
    asked = s.q_t[0].clone()
    with s.session() as x:
        assert (x.items()["seq"] < 0).any()
        got = []
        for factor in (1.0, 0.0, 0.03, 30.0, -1000.0, float("inf"), float("nan")):
            s.q_t[0] = asked * factor
            got.append(x.attend(s.layer, s.q_t, **f.kw))
        for out, lse in got[1:]:
            assert torch.equal(out[1:], got[0][0][1:]) and torch.equal(lse[1:], got[0][1][1:])


@pytest.mark.parametrize("c", KERNELS, ids=["warp", "tile"])
@pytest.mark.parametrize("scale, cap, q_scale", [(1e30, 3e26, 1e-30), (1e30, 5.0, 1e-30), (-1e25, 1e26, 1e-25), (1e-30, 2.3e-26, 1e4), (1e-20, 30.0, 1e21)])
def test_scales_and_caps_far_from_one(c, scale, cap, q_scale):
    """The terms of a capped logit stay in range, for products of zero too."""
    s = Setup(**c, q_scale=q_scale)
    s.q_t[0, 0] = 0
    f = Form(s, kind="tree", cap=cap)
    with s.session() as x:
        got = x.attend(s.layer, s.q_t, scale=scale, **f.kw)
        x.status()
    check(s, *got, expect(s, f, scale))
