"""Calls that put tokens into the cache and settle drafted ones, without a GPU: refusals, and angles per position."""
from fractions import Fraction

import numpy as np
import pytest

from paper_2408_08147_b200 import binding as B
from paper_2408_08147_b200 import build as pdkv_build

FAKE = 0x7F0000000000
BAD = B.PDKV_ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def built():
    pdkv_build.build_library()
    B.pdkv_tune("dry_run", 1)
    yield
    B.pdkv_tune("dry_run", 0)


def handle(lens=(40, 7), H=4, D=64, E=2, Hq=8, q_tokens=1, dtype=0, layers=2, blocks=400):
    d = B.make_desc(0, layers, H, D, E, 16, blocks)
    p = B.pdkv_pool_create(d, FAKE, B.pdkv_pool_bytes(d), 0)
    n = [-(-x // 16) for x in lens]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
    return B.pdkv_seqs_create(p, list(lens), off, np.arange(off[-1], dtype=np.int32), num_q_heads=Hq, q_tokens=q_tokens, dtype=dtype)[0]


def far(i):
    return FAKE + (i << 44)


def status(fn, *a):
    with pytest.raises(B.PdkvError) as e:
        fn(*a)
    return e.value.status


# A call of more rows than a launch takes gets LIMIT, behind every other check: what is in order says LIMIT, what is not INVALID_ARG.
ROWS, PER = 1 << 30, 1 << 29


def append(h, layer=0, H=4, Hq=8, D=64, rotary=None, **over):
    a = B.pdkv_append_args(rows=ROWS, q=far(1), k=far(2), v=far(3), q_out=far(4), q_norm=far(5), k_norm=far(6), norm_eps=1e-6, position=far(7), position_stride=ROWS)
    for name, heads in (("q", Hq), ("q_out", Hq), ("k", H), ("v", H)):
        getattr(a, name + "_stride")[:] = [PER * heads * D, heads * D, D]
    a.rotary = B.pdkv_rotary(**{**dict(dims=64, adjacent=0, n_axes=1, turns=far(8), scale=1.0), **(rotary or {})})
    for k, v in over.items():
        if k.endswith("_stride") and k != "position_stride":
            getattr(a, k)[:] = v
        else:
            setattr(a, k, v)
    return status(B.pdkv_append, h, layer, a)


def fused(**over):
    """8 query heads, 4 key heads and 4 value heads side by side in one buffer."""
    wide = 16 * 64
    at = {name + "_stride": [PER * wide, wide, 64] for name in ("q", "k", "v")}
    return {**dict(q=far(1), k=far(1) + 1024, v=far(1) + 1536, **at), **over}


@pytest.mark.parametrize("over", [
    {}, dict(q=0, q_out=0), dict(q_norm=0, k_norm=0, norm_eps=float("nan")), dict(rotary=dict(dims=0, turns=0, n_axes=0)), dict(position=0), dict(n_new=far(10), seq_len=far(11)),
    dict(row_begin=far(9), q_stride=[-7, 512, 64]), dict(q_out=far(1)), dict(rotary=dict(n_axes=3, axis=far(12))), dict(rotary=dict(dims=22, adjacent=1)),
    fused(), fused(q_out=far(1), q_out_stride=[PER * 1024, 1024, 64]),
    dict(k_stride=[PER * 256, 256, 0]), dict(v_stride=[0, 0, 0]),           # heads, rows that share keys: read only
])
def test_good_arguments(over):
    assert append(handle(), **over) == B.PDKV_ERR_LIMIT


def test_refused_handles_and_layers():
    h = handle()
    assert append(h, layer=2) == BAD and append(h, layer=-1) == BAD
    assert append(handle(Hq=0)) == BAD     # queries through a handle without query heads
    for kw in (dict(D=60), dict(E=1), dict(E=4), dict(D=264)):
        assert append(handle(Hq=0, **kw), q=0, q_out=0) == B.PDKV_ERR_GEOMETRY
    assert status(B.pdkv_append, h, 0, B.pdkv_append_args(rows=0)) == BAD   # in order, but the handle is host-only


@pytest.mark.parametrize("over", [
    dict(rows=5), dict(rows=-2), dict(q=0), dict(q_out=0), dict(k=0), dict(v=0),
    dict(q=far(1) + 8), dict(k=far(2) + 2), dict(v=far(3) + 8), dict(q_out=far(4) + 4), dict(q_norm=far(5) + 4), dict(k_norm=far(6) + 8), dict(position=far(7) + 2),
    dict(q_stride=[PER * 512, 512, 60]), dict(k_stride=[PER * 256, -256, 64]), dict(v_stride=[PER * 256 + 4, 256, 64]),
    dict(q_out_stride=[PER * 512, 512, 32]), dict(q_out_stride=[512, 512, 64]),
    dict(row_begin=far(9), n_new=far(10)), dict(row_begin=far(9) + 2), dict(n_new=far(10) + 1), dict(seq_len=far(11) + 2),
    dict(norm_eps=-1.0), dict(norm_eps=float("nan")),
    dict(rotary=dict(dims=66)), dict(rotary=dict(dims=-2)), dict(rotary=dict(dims=7)), dict(rotary=dict(turns=0)), dict(rotary=dict(turns=far(8) + 4)),
    dict(rotary=dict(n_axes=0)), dict(rotary=dict(n_axes=3)), dict(rotary=dict(n_axes=3, axis=far(12)), position_stride=5), dict(rotary=dict(n_axes=3, axis=far(12)), position=0),
    dict(rotary=dict(scale=float("inf"))), dict(rotary=dict(adjacent=2)),
    # what is written on what is read
    dict(k=FAKE), dict(v=FAKE + 1024), dict(q=FAKE), dict(q_out=FAKE), dict(position=FAKE + 64), dict(seq_len=FAKE), dict(n_new=FAKE), dict(q_norm=FAKE), dict(rotary=dict(turns=FAKE)),
    dict(position=far(4)), dict(k_norm=far(4)),
])
def test_refused_append_arguments(over):
    assert append(handle(), **over) == BAD


@pytest.mark.parametrize("over", [
    dict(q_out=far(1) + 64), dict(q_out=far(2)), dict(q_out=far(3) + 512), dict(q_out=far(1), q_out_stride=[1560, 520, 64]),
])
def test_refused_queries_on_what_is_read(over):
    """(Of few rows: these are looked at one by one.  In order, such a call is refused for its handle alone, with the same status.)"""
    few = dict(rows=6, position_stride=6)
    for name, heads in (("q", 8), ("q_out", 8), ("k", 4), ("v", 4)):
        few[name + "_stride"] = [3 * heads * 64, heads * 64, 64]
    assert append(handle(), **{**few, **over}) == BAD


def accept(h, layers=(0, 64), **over):
    a = B.pdkv_accept_args(path=far(1), path_stride=5, path_len=5, new_tokens=8, n_new=far(2), seq_len=far(3), new_len=far(4))
    for k, v in over.items():
        setattr(a, k, v)
    return status(B.pdkv_accept, h, *layers, a)


@pytest.fixture(scope="module")
def wide():
    """Bytes one by one, more of them than a launch takes: 64 * 2 * 400 * 251."""
    return handle(E=1, D=251, Hq=0, H=400, layers=64, blocks=8)


@pytest.mark.parametrize("over", [{}, dict(n_new=0, seq_len=0, new_len=0), dict(new_len=far(3)), dict(path=0, path_len=0), dict(path_stride=0)])
def test_good_accepts(wide, over):
    assert accept(wide, **over) == B.PDKV_ERR_LIMIT


@pytest.mark.parametrize("over", [
    dict(layers=(0, 65)), dict(layers=(1, 1)), dict(layers=(-1, 1)), dict(path=0), dict(path_len=-1), dict(path_stride=-5), dict(new_tokens=-1),
    dict(path=far(1) + 2), dict(n_new=far(2) + 1), dict(seq_len=far(3) + 2), dict(new_len=far(4) + 3),
    dict(path=FAKE), dict(n_new=FAKE + 128), dict(seq_len=FAKE), dict(new_len=FAKE), dict(new_len=far(1)), dict(new_len=far(2)), dict(new_len=far(3) + 4),
])
def test_refused_accepts(wide, over):
    assert accept(wide, **over) == BAD


def test_turns_are_the_fraction_of_a_turn():
    rng = np.random.default_rng(3)
    x = np.concatenate([[0.0, 1.0, -1.0, 0.5, 6.2, 1e-12, -3e-9, 2 * np.pi], rng.uniform(-6.3, 6.3, 200), 10000.0 ** (-np.arange(64) / 64)])
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582")
    for a, t in zip(x, B.pdkv_rotary_turns(x)):
        want = Fraction(float(a)) / two_pi % 1
        off = abs(Fraction(int(t), 1 << 64) - want)
        # 64 bits of a value of up to 1: the quotient and the constant 2^-64 each, the rounding 2^-65
        assert min(off, 1 - off) <= Fraction(3, 1 << 64), (a, t)
    assert B.pdkv_rotary_turns([]).shape == (0,)
    for bad in (np.nan, np.inf, -np.inf):
        assert status(B.pdkv_rotary_turns, [0.5, bad]) == BAD
