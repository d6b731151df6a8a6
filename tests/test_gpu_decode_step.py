"""The captured decode step of attention_layer.py: batches of more rows than a Linear takes at once, and sequences whose pages are full."""

import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2510_16045_amd import synth
from tests.test_gpu_attention_layer import D, G, HEADS, HIDDEN, KV_HEADS, PAGE, reference

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def layer_of(batch, pages, seed=5):
    from paper_2510_16045_amd.attention_layer import AttentionLayer

    weights = synth.gaussian_weights((HEADS + 2 * KV_HEADS) * D, HIDDEN, seed), synth.gaussian_weights(HIDDEN, HEADS * D, seed + 1)
    table = torch.arange(batch * pages, dtype=torch.int32, device="cuda").view(batch, pages)
    return weights, AttentionLayer(*weights, HEADS, KV_HEADS, batch * pages, table, PAGE, G, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))


def steps_of_a_large_batch(batch, steps=5):
    """Relative errors of the steps against the reference in 64 bits, eager work and synchronizations between the replays."""
    from paper_2510_16045_amd.attention_layer import DecodeStep

    weights, layer = layer_of(batch, 1)
    rng = np.random.default_rng(batch)
    xs = [rng.standard_normal((batch, HIDDEN)).astype(np.float16) for _ in range(steps)]
    step = DecodeStep(layer, torch.zeros(batch, dtype=torch.int32, device="cuda"))
    got = []
    for x in xs:
        got.append(step(torch.from_numpy(x).cuda()).float().cpu().numpy())
        torch.cuda.synchronize()
        torch.zeros((64, HIDDEN), device="cuda") @ torch.zeros((HIDDEN, 64), device="cuda")
        torch.cuda.synchronize()
    return [float(np.linalg.norm(y - want) / np.linalg.norm(want)) for y, want in zip(got, reference(weights, xs, [[1] * batch] * steps))]


@pytest.mark.parametrize("batch", [32, 33, 70])
def test_a_large_batch_may_be_the_first_call_of_a_process(batch):
    run = subprocess.run([sys.executable, "-c", f"from tests.test_gpu_decode_step import *; print(*steps_of_a_large_batch({batch}))"], capture_output=True, text=True, timeout=110, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert run.returncode == 0, run.stderr[-2000:]
    errors = [float(x) for x in run.stdout.split()]
    assert len(errors) == 5 and max(errors) < 1e-2  # the bound of test_gpu_attention_layer.py: a value in some hundreds on the other side of a tie


def test_a_step_that_finds_no_place_is_refused():
    from paper_2510_16045_amd.attention_layer import DecodeStep

    _, layer = layer_of(3, 2)
    lens = torch.tensor([2 * PAGE - 2, 5, 0], dtype=torch.int32, device="cuda")
    step = DecodeStep(layer, lens)
    x = torch.ones((3, HIDDEN), dtype=torch.float16, device="cuda")
    for _ in range(2):
        step(x)
    before = layer.cache.clone(), lens.tolist()
    assert before[1] == [2 * PAGE, 7, 2]
    for _ in range(2):
        with pytest.raises(ValueError, match="no place"):
            step(x)
    torch.cuda.synchronize()
    assert torch.equal(layer.cache, before[0]) and lens.tolist() == before[1]
    lens[0] = 0  # the sequence has ended: its slot begins anew
    for _ in range(2 * PAGE - 7):
        step(x)
    assert lens.tolist() == [2 * PAGE - 7, 2 * PAGE, 2 * PAGE - 5]
    with pytest.raises(ValueError, match="no place"):
        step(x)
    lens.copy_(torch.tensor([1, 1, 2 * PAGE - 1], dtype=torch.int32))
    step(x)
    lens[1] = 2 * PAGE - 1  # a longer one in its place: the host is told
    step.recount()
    with pytest.raises(ValueError, match="no place"):
        step(x)
    lens[2] = 3
    step(x)
    assert lens.tolist() == [3, 2 * PAGE, 4]


def test_sequences_that_are_full_from_the_beginning():
    from paper_2510_16045_amd.attention_layer import DecodeStep

    _, layer = layer_of(2, 1)
    lens = torch.tensor([PAGE, 1], dtype=torch.int32, device="cuda")
    step = DecodeStep(layer, lens)
    with pytest.raises(ValueError, match="no place"):
        step(torch.ones((2, HIDDEN), dtype=torch.float16, device="cuda"))
    assert lens.tolist() == [PAGE, 1]
