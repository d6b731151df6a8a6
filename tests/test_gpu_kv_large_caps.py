"""Scores under large caps: next to plain ones where they are small beside the cap, capped where they are not.

Bound: that of plain scores, and what capped ones are off by themselves: up to a cap of 256 2^-22 of the cap, above it 2^-20 of the score (its
exponential's factor and rounding, 2^-22.5 at a quarter of the cap, where the tangent takes over twice that, is what is largest).  A weight
is off by as much as its score and the sum of all, so by twice that."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O
from tests.test_gpu_kv_attention import counts_are_zero, workspace  # noqa: F401  (the fixtures of that file)
from tests.test_gpu_kv_cache import dev, host
from tests.test_gpu_kv_scores import Scored
from tests.test_gpu_kv_variants import lengths, plan_of, variants

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(c, **more):
    lse = torch.full((len(c.q), c.heads), 7.0, dtype=torch.float32, device="cuda")
    out, lse = host(c.run(lse=lse, **c.scores(), **more)).astype(np.float64), lse.cpu().numpy().astype(np.float64)
    scale, at = more.get("softmax_scale", c.D**-0.5), 0
    for b, ((k, v), n) in enumerate(zip(c.seqs, c.counts)):
        k, v = O.held(k, c.G), O.held(v, c.G)
        prefix = 0 if c.prefix is None else c.prefix[b]
        want, want_lse, size = O.scored_attention(c.q[at : at + n], k, v, scale, c.causal, c.window, c.softcap, c.slopes, prefix)
        most = max(float(np.abs(c.q[at : at + n, h].astype(np.float64) @ k[:, h * k.shape[1] // c.heads].astype(np.float64).T).max()) * scale for h in range(c.heads))
        most = min(most, c.softcap)
        own = 2.0**-22 * c.softcap if c.softcap <= 256 else 2.0**-20 * most
        biased = 0 if c.slopes is None else float(np.abs(c.slopes).max()) * (len(k) + n)
        inexact = 2 * own + 2 * 3 * 2.0**-24 * biased
        # products of fp32: 2^-24 of the score for each doubling of their number
        rounded = max(2e-5, 2 * 8 * 2.0**-24 * most)
        bound = (2.0**-11 + rounded + inexact) * (np.abs(want) + size) + 2.0**-24 + len(k) * 2.0**-32 * (size + 1)
        off = np.abs(out[at : at + n] - want) / bound
        assert off.max() <= 1, (b, off.max())
        assert np.all(np.abs(lse[at : at + n] - want_lse) <= rounded + 1e-5 * (1 + np.abs(want_lse)) + inexact), b
        at += n


CAPS = [255.0, 256.0, 257.0, 1e3, 1e4, 1e6, 1e8, 1e15, 5e37]


@pytest.mark.parametrize("softcap", CAPS)
@pytest.mark.parametrize("count", [1, 9, 300])
@pytest.mark.parametrize("bias", [False, True])
def test_scores_far_below_the_cap(softcap, count, bias):
    check(Scored([400], [count], heads=4, kv_heads=2, softcap=softcap, bias=bias), max_q_len=count)


@pytest.mark.parametrize("softcap", [300.0, 2e3, 1e4, 1e5])
@pytest.mark.parametrize("share", [0.2, 1.0, 4.0])
@pytest.mark.parametrize("count", [1, 300])
def test_scores_about_the_cap(softcap, share, count):
    """The scale makes the largest score that many times the cap: the series, the exponential and both; tangents near their ends."""
    c = Scored([400], [count], heads=2, kv_heads=1, softcap=softcap)
    k = O.held(c.seqs[0][0], c.G).astype(np.float64)
    most = float(np.abs(c.q.astype(np.float64).reshape(-1, c.D) @ k[:, 0].T).max())
    check(c, max_q_len=count, softmax_scale=float(np.float32(share * softcap / most)))


@pytest.mark.parametrize("D,G", [(64, 32), (128, 128), (256, 64)])
@pytest.mark.parametrize("count", [1, 40, 300])
def test_with_prefix_and_window(D, G, count):
    check(Scored([700], [count], heads=2, kv_heads=1, D=D, G=G, prefix=[100], window=50, softcap=1e6, bias=True), max_q_len=count)


def test_without_a_mask():
    check(Scored([70, 400], [9, 300], heads=4, kv_heads=2, causal=False, softcap=1e4, bias=True), max_q_len=300)


@pytest.mark.parametrize("prefix", [None, [2500, 9, 33, 4, 0]])
def test_pieces(prefix):
    """Keys shared out to several workgroups, without rows' prefixes too."""
    c = Scored([3000, 5, 1111, 7, 260], [1] * 5, heads=8, kv_heads=1, prefix=prefix, window=0 if prefix is None else 500, softcap=1e5, bias=True)
    if prefix is not None:
        c.prefix = [min(p, n) for p, n in zip(prefix, c.lens)]
    check(c)
    assert torch.equal(c.run(**c.scores()), c.run(**c.scores()))


@pytest.mark.parametrize("D,G,columns,waves,split", variants())
def test_every_kernel_for_few_rows(D, G, columns, waves, split):
    if waves == 8:
        kv_heads, batch, idle = {"whole": (8, 7, 0), "parts": (8, 7, 0), "across": (32, 7, 0)}[split]
    else:
        kv_heads, batch, idle = {"whole": (64, 7, 0), "parts": (64, 4, 3), "across": (64, 7, 0)}[split]
    count = 1 if columns == 1 else 16 * columns - 3
    n = batch + idle
    lens = lengths(n, 1000 if split == "whole" else 1100, count)
    if idle:
        lens[1], lens[n // 2] = 1100, 70
    c = Scored(lens, [count if b < batch else 0 for b in range(n)], heads=kv_heads, kv_heads=kv_heads, D=D, G=G, page=64, softcap=300.0, bias=True)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    plan = plan_of(c)
    assert (plan["kernel"], plan["rows"], plan["waves"]) == ("stream", 16 * columns, waves), plan
    c.check(heads=[0, kv_heads - 1], max_q_len=count, workspace=ws)
    assert not bool(ws[:65536].any())


@pytest.mark.parametrize("D,G,waves", [(64, 32, 4), (64, 64, 8), (128, 32, 4), (128, 128, 8), (256, 64, 4)])
def test_every_kernel_for_prompts(D, G, waves):
    c = Scored([1300, 260], [1024, 260], heads=64, kv_heads=64, D=D, G=G, page=64, spare=60 if waves == 8 else 1, softcap=300.0, bias=True)
    plan = plan_of(c)
    assert (plan["kernel"], plan["waves"]) == ("tile", waves), plan
    c.check(heads=[0, 63], max_q_len=1024)


def test_captured():
    ams.ams_init()
    c = Scored([300, 40], [1, 1], softcap=1e3, bias=True)
    q, out, scores = dev(c.q), torch.zeros((2, 4, 128), dtype=torch.float16, device="cuda"), c.scores()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(q=q, out=out, **scores)
    for seed in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        assert torch.equal(out, c.run(q=q, **scores)) and bool(out.any())
