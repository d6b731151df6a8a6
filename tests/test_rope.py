"""Rotary positions on the host: the frequencies, and what is refused before anything is launched."""

import ctypes
import math

import numpy as np
import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")

TURN = 2 * math.pi


def frequencies(r, base, scaling, factor, trained):
    """The definition in Python's floats, written apart from the library's."""
    w = [base ** (-2 * i / r) for i in range(r // 2)]
    if scaling == "linear":
        return [x / factor for x in w]
    if scaling == "ntk":
        return [(base * factor ** (r / (r - 2))) ** (-2 * i / r) for i in range(r // 2)]
    if scaling == "bands":
        out = []
        for x in w:
            turns = trained * x / TURN
            mix = 0 if turns < 1 else 1 if turns > 4 else (turns - 1) / 3
            out.append(mix * x + (1 - mix) * x / factor)
        return out
    if scaling == "yarn":
        at = lambda turns: r * math.log(trained / (turns * TURN)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), r - 1)
        ramp = [min(1, max(0, (i - lo) / max(hi - lo, 0.001))) for i in range(r // 2)]
        return [x * (1 - m) + x / factor * m for x, m in zip(w, ramp)]
    return w


@pytest.mark.parametrize("r", [2, 4, 64, 100, 128, 256])
@pytest.mark.parametrize("scaling", ams.ROPE_SCALINGS)
@pytest.mark.parametrize("base,factor,trained", [(10000.0, 4.0, 4096), (500000.0, 8.0, 8192), (1e6, 1.0, 131072)])
def test_frequencies(r, scaling, base, factor, trained):
    if scaling == "ntk" and r == 2:
        factor = 1.0  # its one pair has frequency 1 whatever the base
        trained = 0
    turns, magnitude = ams.ams_rope_frequencies(r, base, scaling, factor, trained)
    want = frequencies(r, base, scaling, factor, trained) if r > 2 or scaling != "ntk" else [1.0]
    got = turns.view(np.uint64).astype(np.float64) / 2.0**64 * TURN
    # a few roundings to 53 bits each in powers, logarithms and products; turns hold whole multiples of 2^-64, rounded down (of the
    # smallest, 1e-6 / 4 radians = 4e-8 turns, that alone is 2^-64 / 4e-8 = 1.4e-12)
    assert np.allclose(got, want, rtol=1e-13, atol=TURN * 2.0**-64)
    assert magnitude == pytest.approx(1 + 0.1 * math.log(factor) if scaling == "yarn" else 1.0, rel=2.0**-23)


@pytest.mark.parametrize("args", [(0,), (3,), (1026,), (64, 0.5), (64, math.nan), (64, 1e4, "linear", 0.5), (64, 1e4, "linear", math.inf), (64, 1e4, "bands", 2.0, 0), (64, 1.0, "yarn", 2.0, 4096)])
def test_frequencies_refused(args):
    with pytest.raises(ams.AmsError):
        ams.ams_rope_frequencies(*args)


def test_unknown_scaling():
    with pytest.raises(ValueError):
        ams.ams_rope_frequencies(64, scaling="longer")
    out, m = np.empty(4, dtype=np.int64), ctypes.c_float()
    lib = ams.load_library()
    assert lib.ams_rope_frequencies(8, 1e4, 5, 2.0, 100, ams._np_ptr(out), ctypes.byref(m)) == -2
    assert lib.ams_rope_frequencies(8, 1e4, -1, 2.0, 100, ams._np_ptr(out), ctypes.byref(m)) == -2
    assert lib.ams_rope_frequencies(8, 1e4, 0, 2.0, 100, None, ctypes.byref(m)) == -3


def call(rows=4, head_dim=128, heads=2, kv_heads=1, turns=0x1000, positions=0x1000, kv_lens=None, q_starts=None, batch=0, rotary_dim=128, magnitude=1.0, q_in=0x1000, q_out=0x2000, k=True):
    """ams_rope with addresses that are never used: what is refused is refused before anything is launched."""
    rotation = ams._Rotation(turns, positions, kv_lens, q_starts, batch, rotary_dim, 0, 0, magnitude)
    q = ams._RopeRows(q_in, q_out, 256, 128, 256, 128, heads)
    rows_k = ams._RopeRows(0x3000, 0x3000, 256, 128, 256, 128, kv_heads)
    return ams.load_library().ams_rope(ctypes.byref(rotation), ctypes.byref(q), ctypes.byref(rows_k) if k else None, rows, head_dim, None)


NULL, SHAPE, ALIGN = -3, -2, -4


@pytest.mark.parametrize(
    "more,code",
    [
        (dict(rows=-1), SHAPE), (dict(rows=(1 << 28) + 1), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=1025), SHAPE), (dict(rotary_dim=130), SHAPE), (dict(rotary_dim=0), SHAPE),
        (dict(rotary_dim=7), SHAPE), (dict(heads=0), SHAPE), (dict(heads=1025), SHAPE), (dict(kv_heads=0), SHAPE), (dict(magnitude=math.inf), SHAPE), (dict(magnitude=math.nan), SHAPE),
        (dict(positions=None, kv_lens=0x1000, batch=3), SHAPE), (dict(batch=-1), SHAPE), (dict(batch=65537), SHAPE), (dict(turns=None), NULL), (dict(q_in=None), NULL), (dict(q_out=None), NULL),
        (dict(positions=None, batch=4), NULL), (dict(turns=0x1004), ALIGN), (dict(positions=0x1002), ALIGN), (dict(q_in=0x1001), ALIGN), (dict(q_out=0x2001, k=False), ALIGN),
    ],
)
def test_refused(more, code):
    assert call(**more) == code


def test_no_rotation():
    lib = ams.load_library()
    assert lib.ams_rope(None, None, None, 1, 128, None) == NULL


@pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")
def test_no_gpu():
    assert call() == -7


def test_python_refusals():
    q, turns = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros(32, dtype=torch.int64)
    at, lens = torch.zeros(3, dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        ams.ams_rope(q, None, turns)  # neither positions nor lengths
    with pytest.raises(ValueError):
        ams.ams_rope(q, None, turns, positions=at, kv_lens=lens)
    with pytest.raises(ValueError):
        ams.ams_rope(q, None, turns, positions=at, q_starts=lens)
    with pytest.raises(ValueError):
        ams.ams_rope(q, q[:2], turns, positions=at)
    with pytest.raises(ValueError):
        ams.ams_rope(q[0], None, turns, positions=at)
    with pytest.raises(ValueError):
        ams.ams_rope(q, None, turns, positions=at[:2])
    with pytest.raises(ValueError):
        ams.ams_rope(q, None, turns, kv_lens=lens, q_starts=lens)
    with pytest.raises(ValueError):
        ams.ams_rope(q, q, turns, positions=at, out=(q, None))
    with pytest.raises(ValueError):
        ams.ams_rope(q, None, turns, positions=at)  # not on a GPU
