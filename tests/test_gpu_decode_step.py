"""The captured decode step of attention_layer.py: batches of more rows than a Linear takes at once."""

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
