"""Capped, biased and prefix scores: what is refused before anything is launched, and the oracle's own pins."""

import ctypes
import math

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O

NULL, SHAPE, ALIGN = -3, -2, -4


def call(softcap=0.0, slopes=None, prefix=None, causal=1, scale=0.125, scores=True):
    """ams_kv_attention_scored with addresses that are never used: what is refused is refused before anything is launched."""
    cache = ams._KvCache(0x1000, 0x1000, 0x1000, None, 4, 2, 2, 1, 2, 128, 64, 32)
    s = ams._KvScores(slopes, prefix, softcap)
    return ams.load_library().ams_kv_attention_scored(ctypes.byref(cache), ctypes.byref(s) if scores else None, 0x1000, 0x1000, None, 1, 4, 512, 128, 512, 128, 0, scale, causal, 0, 0, None, 0, None)


@pytest.mark.parametrize(
    "more,code",
    [(dict(softcap=-1.0), SHAPE), (dict(softcap=math.nan), SHAPE), (dict(softcap=math.inf), SHAPE), (dict(softcap=3e38), SHAPE), (dict(softcap=1e-38, scale=10.0), SHAPE), (dict(prefix=0x1000, causal=0), SHAPE),
     (dict(slopes=0x1002), ALIGN), (dict(prefix=0x1001), ALIGN), (dict(scale=0.0), SHAPE), (dict(scores=False, scale=-1.0), SHAPE)],
)
def test_refused(more, code):
    assert call(**more) == code


def test_no_gpu():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("for machines without a GPU")
    assert call() == call(softcap=30.0, slopes=0x1000, prefix=0x1000) == call(scores=False) == -7


def test_the_oracle():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 2, 8)), rng.standard_normal((9, 1, 8)), rng.standard_normal((9, 1, 8))
    plain = O.attention(q, k, v, 0.3, True, 4)
    for a, b in zip(plain, O.scored_attention(q, k, v, 0.3, True, 4)):
        assert np.array_equal(a, b)
    # by hand: row 0 of head 1, at position 4, window 2, prefix 7
    out, lse, _ = O.scored_attention(q, k, v, 0.3, True, 2, 2.0, [0.0, 0.5], 7)
    seen = [0, 1, 2, 3, 4, 5, 6]
    s = [2.0 * math.tanh(0.3 * float(q[0, 1] @ k[j, 0]) / 2.0) - 0.5 * abs(4 - j) for j in seen]
    w = [math.exp(x) for x in s]
    assert lse[0, 1] == pytest.approx(math.log(sum(w)), rel=1e-13)
    assert np.allclose(out[0, 1], sum(x * v[j, 0] for x, j in zip(w, seen)) / sum(w), rtol=1e-12)
    # a row without a position sees nothing
    out, lse, _ = O.scored_attention(rng.standard_normal((11, 1, 8)), k, v, 0.3, True, 0, 0, None, 5)
    assert np.isinf(lse[:2]).all() and not out[:2].any() and np.isfinite(lse[2:]).all()
