"""Packed projections, the 4-bit cache and attention together, as attention_layer.py uses them: prompts, then captured decode
steps, against the same block in 64 bits on the same packed weights."""

import subprocess
import sys

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import ams_oracle as AO
from oracle import kv_oracle as O
from paper_2510_16045_amd import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV_HEADS, D, PAGE, G = 512, 8, 2, 64, 16, 32


def reference(weights, x_of, lens_of):
    """Outputs of the calls, in 64 bits; what a call rounds to fp16 on its way is rounded here too (projections, cache, attention's output)."""
    half = lambda a: a.astype(np.float16).astype(np.float64)  # noqa: E731
    dense = []
    for w in weights:
        codes, scales, _ = AO.ams_quantize(w, AO.FP425)
        dense.append(AO.dequant_scaled(codes, scales, AO.FP425).astype(np.float64))
    kv = [[np.zeros((0, KV_HEADS, D))] * 2 for _ in lens_of[0]]
    outs = []
    for x, lens in zip(x_of, lens_of):
        rows = half(x.astype(np.float64) @ dense[0].T).reshape(len(x), HEADS + 2 * KV_HEADS, D)
        at, ys = 0, []
        for b, n in enumerate(lens):
            mine = rows[at : at + n]
            at += n
            for i in range(2):
                new = O.held(mine[:, HEADS + i * KV_HEADS : HEADS + (i + 1) * KV_HEADS].astype(np.float16), G)
                kv[b] = [np.concatenate([old, new]) if j == i else old for j, old in enumerate(kv[b])]
            if n:
                ys.append(O.attention(mine[:, :HEADS].astype(np.float16), *kv[b], D**-0.5)[0])
        y = half(np.concatenate(ys)).reshape(len(x), HEADS * D)
        outs.append(y @ dense[1].T)
    return outs


def test_prompts_then_captured_steps():
    from paper_2510_16045_amd.attention_layer import AttentionLayer, DecodeStep

    rng = np.random.default_rng(0)
    weights = synth.gaussian_weights((HEADS + 2 * KV_HEADS) * D, HIDDEN, 5), synth.gaussian_weights(HIDDEN, HEADS * D, 6)
    prompts, steps = [45, 7, 0, 20], 5
    pages = 5
    table = torch.from_numpy(rng.permutation(len(prompts) * pages).astype(np.int32).reshape(len(prompts), pages)).cuda()
    layer = AttentionLayer(*weights, HEADS, KV_HEADS, len(prompts) * pages, table, PAGE, G, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))
    xs = [rng.standard_normal((n, HIDDEN)).astype(np.float16) for n in [sum(prompts)] + [len(prompts)] * steps]
    dev = [torch.from_numpy(x.view(np.int16)).cuda().view(torch.float16) for x in xs]
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    starts = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32, device="cuda")
    got = [layer(dev[0], lens, q_starts=starts, max_q_len=max(prompts)).clone()]
    step = DecodeStep(layer, lens)
    assert lens.tolist() == prompts  # capturing ran nothing
    for x in dev[1:]:
        got.append(step(x).clone())
        torch.cuda.synchronize()
    assert lens.tolist() == [n + steps for n in prompts]
    # The reference rounds where the calls do, but to the same side only mostly: a sum that falls next to a tie gives another fp16 value
    # of q, or another code of k or v (a quarter of its run's scale).  1e-2 of the output's norm leaves room for one value in some hundreds.
    for y, want in zip(got, reference(weights, xs, [prompts] + [[1] * len(prompts)] * steps)):
        y = y.float().cpu().numpy().astype(np.float64)
        assert np.linalg.norm(y - want) / np.linalg.norm(want) < 1e-2


def test_the_first_call_of_a_process_may_be_captured():
    code = """
import torch, paper_2510_16045_amd as ams
q = torch.randn((2, 4, 64), device="cuda").half()
cache, table, lens = ams.ams_kv_cache(4, 2, 64, 16, 32), torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda"), torch.tensor([20, 3], dtype=torch.int32, device="cuda")
out = torch.zeros_like(q)
ams.ams_init()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    ams.ams_kv_write(cache, q[:, :2], q[:, 2:], table, lens, 32)
    ams.ams_kv_attention(q, cache, table, lens, 32, out=out)
g.replay()
torch.cuda.synchronize()
want = ams.ams_kv_attention(q, cache, table, lens, 32)
torch.cuda.synchronize()
assert torch.equal(out, want) and bool(out.any())
print("same")
"""
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110)
    assert run.stdout.split() == ["same"], run.stderr
