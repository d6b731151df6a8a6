"""Rotary positions, the cache, scored attention, packed projections and log probabilities together, as a model's step uses them: prompts,
then captured steps, against the same in 64 bits on the same packed weights."""

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

HIDDEN, HEADS, KV_HEADS, D, PAGE, G, VOCAB = 512, 8, 2, 64, 16, 32, 3001
half = lambda a: np.asarray(a).astype(np.float16).astype(np.float64)  # noqa: E731


def dense(w):
    codes, scales, _ = AO.ams_quantize(w, AO.FP425)
    return AO.dequant_scaled(codes, scales, AO.FP425).astype(np.float64)


def rotated(x, positions, rot, interleaved, base=10000.0):
    y = x.copy()
    i = np.arange(rot // 2) * (2 if interleaved else 1)
    j = i + (1 if interleaved else rot // 2)
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * base ** (-2 * np.arange(rot // 2) / rot)
    y[..., i], y[..., j] = x[..., i] * np.cos(angle) - x[..., j] * np.sin(angle), x[..., j] * np.cos(angle) + x[..., i] * np.sin(angle)
    return half(y)


FORMS = [
    dict(rot=64, interleaved=False, softcap=20.0),
    dict(rot=16, interleaved=True, softcap=0.0, window=24, prefix=[3, 7, 0, 11]),
    dict(rot=0, softcap=0.0, slopes=True),
]


@pytest.mark.parametrize("form", FORMS)
def test_prompts_then_captured_steps(form):
    from paper_2510_16045_amd.attention_layer import AttentionLayer, Rotary, Vocabulary

    rng = np.random.default_rng(0)
    weights = synth.gaussian_weights((HEADS + 2 * KV_HEADS) * D, HIDDEN, 5), synth.gaussian_weights(HIDDEN, HEADS * D, 6), synth.gaussian_weights(VOCAB, HIDDEN, 7)
    prompts, steps, pages = [45, 7, 0, 20], 5, 5
    slopes = np.array([2.0 ** -(h + 1) for h in range(HEADS)], dtype=np.float32) if form.get("slopes") else None
    scores = dict(softcap=form["softcap"], window=form.get("window", 0), slopes=None if slopes is None else torch.from_numpy(slopes).cuda(),
                  prefix_lens=torch.tensor(form["prefix"], dtype=torch.int32, device="cuda") if "prefix" in form else None)
    table = torch.from_numpy(rng.permutation(len(prompts) * pages).astype(np.int32).reshape(len(prompts), pages)).cuda()
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")  # one for attention and the log probabilities
    rotary = Rotary(form["rot"], interleaved=form["interleaved"]) if form["rot"] else None
    layer = AttentionLayer(*weights[:2], HEADS, KV_HEADS, len(prompts) * pages, table, PAGE, G, workspace=ws, rotary=rotary, **scores)
    vocabulary = Vocabulary(weights[2], workspace=ws)
    xs = [rng.standard_normal((n, HIDDEN)).astype(np.float16) for n in [sum(prompts)] + [len(prompts)] * steps]
    dev = [torch.from_numpy(x.view(np.int16)).cuda().view(torch.float16) for x in xs]
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    starts = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32, device="cuda")
    got = [layer(dev[0], lens, q_starts=starts, max_q_len=max(prompts)).clone()]

    # the step and what is reported of its answer, in one graph
    tokens = torch.tensor([5, 3000, -1, 17], dtype=torch.int32, device="cuda")
    ams.ams_init()
    x, y = torch.zeros_like(dev[1]), torch.zeros((len(prompts), HIDDEN), dtype=torch.float16, device="cuda")
    eager = vocabulary(got[0][: len(prompts)], tokens, top=6, temperature=0.8)
    report = ams.LogProbs(*(torch.zeros_like(t) for t in eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens += 1
        layer(x, lens, out=y)
        vocabulary(y, tokens, top=6, temperature=0.8, out=report)
    reports = []
    for row in dev[1:]:
        x.copy_(row)
        graph.replay()
        got.append(y.clone())
        reports.append(ams.LogProbs(*(t.clone() for t in report)))
        torch.cuda.synchronize()
        again = vocabulary(y, tokens, top=6, temperature=0.8)  # eager work between the replays
        assert all(torch.equal(a, b) for a, b in zip(again, report))
    assert lens.tolist() == [n + steps for n in prompts]

    w = [dense(x) for x in weights]
    kv, at_len = [[np.zeros((0, KV_HEADS, D))] * 2 for _ in prompts], [0] * len(prompts)
    for x, y, counts in zip(xs, got, [prompts] + [[1] * len(prompts)] * steps):
        rows = half(x.astype(np.float64) @ w[0].T).reshape(len(x), HEADS + 2 * KV_HEADS, D)
        at, ys = 0, []
        for b, n in enumerate(counts):
            mine = rows[at : at + n]
            at += n
            if n == 0:
                continue
            positions = range(at_len[b], at_len[b] + n)
            at_len[b] += n
            if form["rot"]:
                mine = np.concatenate((rotated(mine[:, : HEADS + KV_HEADS], positions, form["rot"], form["interleaved"]), mine[:, HEADS + KV_HEADS :]), 1)
            for i in range(2):
                new = O.held(mine[:, HEADS + i * KV_HEADS : HEADS + (i + 1) * KV_HEADS].astype(np.float16), G)
                kv[b] = [np.concatenate([old, new]) if j == i else old for j, old in enumerate(kv[b])]
            ys.append(O.scored_attention(mine[:, :HEADS].astype(np.float16), *kv[b], D**-0.5, True, form.get("window", 0), form["softcap"], slopes, min(form["prefix"][b], at_len[b]) if "prefix" in form else 0)[0])
        want = half(np.concatenate(ys)).reshape(len(x), HEADS * D) @ w[1].T
        # as in the test of the plain layer: 1e-2 of the norm leaves room for one value in some hundreds that another side of a rounding gives
        y = y.float().cpu().numpy().astype(np.float64)
        assert np.linalg.norm(y - want) / np.linalg.norm(want) < 1e-2
    for y, r in zip(got[1:], reports):
        logits = half(y.cpu().double().numpy() @ w[2].T)
        z = logits / 0.8
        lp = z - z.max(1, keepdims=True)
        lp -= np.log(np.exp(lp).sum(1, keepdims=True))
        # each logit is rounded to fp16 on one side or the other of the reference's: 2^-11 of the largest, in the token's and in the sum's
        near = 2 * 2.0**-11 / 0.8 * np.abs(logits).max() + 1e-4
        for b, token in enumerate(tokens.tolist()):
            assert r.logprob[b].item() == 0 if token < 0 else abs(r.logprob[b].item() - lp[b, token]) <= near
        top = r.top_tokens.cpu().numpy()
        assert np.all(np.abs(np.take_along_axis(lp, top, 1) - r.top_logprobs.cpu().numpy()) <= near)
        assert np.all(np.sort(lp, 1)[:, ::-1][:, :6] - r.top_logprobs.cpu().numpy() <= near) and all(len(set(t)) == 6 for t in top.tolist())
        assert np.all(np.abs(-(np.exp(lp) * lp).sum(1) - r.entropy.cpu().numpy()) <= near * 10)


def test_decode_step_rotates_by_the_lengths():
    """DecodeStep of a layer with a rotary embedding: each replay rotates by the lengths of that step."""
    from paper_2510_16045_amd.attention_layer import AttentionLayer, DecodeStep, Rotary

    weights = synth.gaussian_weights((HEADS + 2 * KV_HEADS) * D, HIDDEN, 5), synth.gaussian_weights(HIDDEN, HEADS * D, 6)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    layers = [AttentionLayer(*weights, HEADS, KV_HEADS, 8, table, PAGE, G, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), rotary=Rotary(D, 500000.0, "bands", 8.0, 8192)) for _ in range(2)]
    lens, eager_lens = (torch.tensor([0, 30], dtype=torch.int32, device="cuda") for _ in range(2))
    step = DecodeStep(layers[0], lens)
    for i in range(4):
        x = torch.randn((2, HIDDEN), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").half()
        got = step(x)
        torch.cuda.synchronize()
        eager_lens += 1
        assert torch.equal(got, layers[1](x, eager_lens)), i


def test_the_first_calls_of_a_process_may_be_captured():
    code = """
import torch, paper_2510_16045_amd as ams
q = torch.randn((2, 4, 64), device="cuda").half()
cache, table, lens = ams.ams_kv_cache(4, 2, 64, 16, 32), torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda"), torch.tensor([20, 3], dtype=torch.int32, device="cuda")
turns, prefix, slopes = torch.from_numpy(ams.ams_rope_frequencies(64)[0]).cuda(), torch.tensor([2, 1], dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
ws, logits = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.randn((2, 40000), device="cuda").half()
def run(ws):
    r = ams.ams_rope(q, None, turns, kv_lens=lens)[0]
    a = ams.ams_kv_attention(r, cache, table, lens, 32, softcap=5.0, slopes=slopes, workspace=ws)
    b = ams.ams_kv_attention(r, cache, table, lens, 32, prefix_lens=prefix, window=4, workspace=ws)
    return [r, a, b, *ams.ams_logprobs(logits, top=3, workspace=ws)[2:]]
ams.ams_init()
ams.ams_kv_write(cache, q[:, :2], q[:, 2:], table, lens, 32)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    out = run(ws)
for _ in range(3):
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, run(ws)))
print("same")
"""
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110)
    assert run.stdout.split() == ["same"], run.stderr
