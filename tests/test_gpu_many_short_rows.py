"""More rows than one launch can have threads for."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from tests.test_gpu_logprobs import check as check_logprobs
from tests.test_gpu_rope import check as check_rope
from tests.test_gpu_rope import turns_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [(1 << 24) - 1, 1 << 24, (1 << 24) + 5])
def test_log_probabilities(n):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((n, 3), generator=gen, device="cuda").half()
    tokens = torch.randint(0, 3, (n,), generator=gen, device="cuda", dtype=torch.int32)
    got = ams.ams_logprobs(x, tokens, top=2)
    some = [0, 1, 511, 1 << 22, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 24) - 3, n - 2, n - 1]
    check_logprobs(ams.LogProbs(*(t[some] for t in got)), x[some], tokens[some].tolist(), 2)
    # all rows, by torch in fp32
    lp = torch.log_softmax(x.float(), 1)
    assert torch.equal(got.top_tokens[:, 0].long(), x.argmax(1)) and float((got.logprob - lp.gather(1, tokens.long()[:, None])[:, 0]).abs().max()) < 1e-4


@pytest.mark.parametrize("of_cache", [False, True])
def test_rotations(of_cache):
    n = (1 << 26) + 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((n, 1, 2), generator=gen, device="cuda").half()
    turns = turns_of(2)
    some = np.array([0, 1, 4097, (1 << 24) - 1, 1 << 24, (1 << 25) - 1, 1 << 25, (1 << 26) - 5, (1 << 26) - 4, (1 << 26) - 1, 1 << 26, n - 1])
    if of_cache:
        starts = [0, 1 << 25, (1 << 26) - 4, n]
        lens = [1 << 25, 1 << 26, 100]
        got, _ = ams.ams_rope(q, None, turns, kv_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), q_starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        b = np.searchsorted(starts, some, side="right") - 1
        at = [lens[i] - starts[i + 1] + int(r) for i, r in zip(b, some)]
    else:
        positions = (torch.arange(n, dtype=torch.int32, device="cuda") * 7) % 100003
        got, _ = ams.ams_rope(q, None, turns, positions=positions)
        at = positions[some].tolist()
    check_rope(got[some], q[some], at, 2)
    # a rotation keeps each pair's length: no row was left out (of the four roundings each half a step)
    a, b = q.float().square().sum(-1), got.float().square().sum(-1)
    assert bool(((a - b).abs() <= 4 * 2.0**-11 * a + 1e-6).all())
