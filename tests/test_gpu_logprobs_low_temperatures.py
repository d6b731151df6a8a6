"""Log probabilities at temperatures so low that a logit over the temperature is a number of millions or more.

What lies below the largest logit there has probability 0 (neighbouring fp16 values are further apart than an exponential reaches), so
probabilities are 1 / n for the n equal largest ones, and log probabilities are differences of logits over the temperature: off by 2^-24 of
them each for the difference, the factor, its product, what the logarithm adds, ln 2 and the last product: 6 x 2^-24.  What does not grow
with them is bounded as at other temperatures."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from tests.test_gpu_logprobs import reference

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TEMPERATURES = [float(np.float32(t)) for t in (1e-6, 5e-6, 1e-5, 2e-5, 1e-3)]


@pytest.fixture(scope="module")
def workspace():
    return torch.zeros(ams.KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


def check(got, x, tokens, top, temperature):
    want = reference(x, tokens, top, temperature)
    vocab = x.shape[1]
    base = 2.0**-22 * (np.log(vocab) + 8) + 2.0**-23 * (vocab / 1024 + 40)
    for i in (0, 3):
        a, b = got[i].cpu().double().numpy(), want[i]
        assert np.array_equal(a == -np.inf, b == -np.inf)
        there = b != -np.inf
        off = np.abs(a[there] - b[there]) / (base + 6 * 2.0**-24 * np.abs(b[there]))
        assert (off <= 1).all(), (i, off.max())
    off = np.abs(got.entropy.cpu().double().numpy() - want[2]) / (base * (np.log(vocab) + 3))
    assert (off <= 1).all(), off.max()
    assert np.array_equal(got.rank.cpu().numpy(), want[1]) and np.array_equal(got.top_tokens.cpu().numpy(), want[4])


@pytest.mark.parametrize("with_workspace", [False, True])
@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("wide", [False, True])
def test_large_logits(workspace, wide, temperature, with_workspace):
    """Largest ones of 1 to 65504, of either sign, alone and several times."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    most = torch.tensor([1.0, 20.0, 100.0, 1000.0, 4264.0, 5000.0, 29824.0, 59904.0, 65504.0, -1.0, -300.0, -4264.0, -30016.0], device="cuda")
    x = most[:, None] - 500 * torch.rand((len(most), 20011), generator=gen, device="cuda")
    x = x.clamp(-65504, 65504).half()
    for r in range(len(most)):
        x[r, r * 1500], x[r, 19000 - r] = most[r], most[r] if r % 2 else x[r, 0]
    x = x.float() if wide else x
    tokens = torch.tensor([(r * 1500, 19000 - r, 77)[r % 3] for r in range(len(most))], dtype=torch.int32, device="cuda")
    got = ams.ams_logprobs(x, tokens, top=5, temperature=temperature, workspace=workspace if with_workspace else None)
    check(got, x, tokens.tolist(), 5, temperature)
    assert not workspace[: 64 << 10].any()


@pytest.mark.parametrize("with_workspace", [False, True])
@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("rows,vocab", [(3, 9000), (2, 50001), (1, 30011), (600, 9000)])
def test_masks_of_the_lowest_value(workspace, rows, vocab, temperature, with_workspace):
    """Whole chunks, wavefronts and parts of a row that hold nothing but the type's lowest value, and rows that do."""
    x = torch.full((rows, vocab), torch.finfo(torch.float16).min, dtype=torch.float16, device="cuda")
    for r in range(rows):
        at = (r * 2500 + 2100) % (vocab - 4)
        if r % 7 != 6:
            x[r, at : at + 4] = torch.tensor([1.0, 2.0, 3.0, 10.3], device="cuda").half()
    tokens = torch.tensor([((r * 2500 + 2100) % (vocab - 4) + r % 4, vocab - 1)[r % 5 == 4] for r in range(rows)], dtype=torch.int32, device="cuda")
    got = ams.ams_logprobs(x, tokens, top=6, temperature=temperature, workspace=workspace if with_workspace else None)
    some = sorted({r for r in (0, 1, 2, 4, 6, 13, 34, rows - 1) if r < rows})
    check(ams.LogProbs(*(t[some] for t in got)), x[some], tokens[some].tolist(), 6, temperature)
    assert not any(bool(t.isnan().any()) for t in (got.logprob, got.entropy, got.top_logprobs))


@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_nan_and_infinity(workspace, temperature):
    x = torch.full((4, 9000), -65504.0, dtype=torch.float16, device="cuda")
    x[:, 5000] = 30000.0
    x[0, 8000], x[1, 5], x[2, 7:] = float("nan"), float("inf"), -float("inf")
    tokens = torch.tensor([5000, 5000, 8, 5000], dtype=torch.int32, device="cuda")
    got = ams.ams_logprobs(x, tokens, top=3, temperature=temperature, workspace=workspace)
    assert got.logprob[:2].isnan().all() and got.entropy[:2].isnan().all() and got.top_logprobs[:2].isnan().all()
    check(ams.LogProbs(*(t[2:] for t in got)), x[2:], tokens[2:].tolist(), 3, temperature)
