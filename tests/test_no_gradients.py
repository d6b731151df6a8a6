"""Rotations and log probabilities record nothing for torch's autograd: a tensor that a gradient is asked of is refused, not silently cut off."""

import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")


def test_rotations():
    q, turns, at = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros(32, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    leaf = q.clone().requires_grad_()
    for bad in (lambda: ams.ams_rope(leaf, None, turns, positions=at), lambda: ams.ams_rope(q, leaf, turns, positions=at), lambda: ams.ams_rope(q, None, turns, positions=at, out=(leaf, None)),
                lambda: ams.ams_rope(leaf * 2, None, turns, positions=at)):
        with pytest.raises(RuntimeError, match="gradient"):
            bad()
    with torch.no_grad(), pytest.raises(ValueError):  # as without one: not on a GPU
        ams.ams_rope(leaf, None, turns, positions=at)


def test_log_probabilities():
    x = torch.zeros((3, 50), dtype=torch.float16, requires_grad=True)
    with pytest.raises(RuntimeError, match="gradient"):
        ams.ams_logprobs(x)
    with torch.no_grad(), pytest.raises(ValueError):
        ams.ams_logprobs(x)


@pytest.mark.gpu
def test_on_the_gpu():
    """The short way, too; and what is called without a gradient's record runs."""
    q, k = torch.randn((3, 2, 64), device="cuda").half(), torch.randn((3, 1, 64), device="cuda").half()
    turns, at = torch.from_numpy(ams.ams_rope_frequencies(64)[0]).cuda(), torch.arange(3, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q), torch.empty_like(k)
    ams.ams_rope(q, k, turns, positions=at, out=out)
    want = out[0].clone(), out[1].clone()
    leaf = q.clone().requires_grad_()
    for args in ((leaf, k, out), (q, k.clone().requires_grad_(), out), (q, k, (leaf, out[1]))):
        with pytest.raises(RuntimeError, match="gradient"):
            ams.ams_rope(*args[:2], turns, positions=at, out=args[2])
    assert torch.equal(leaf.detach(), q)
    with torch.no_grad():
        got = ams.ams_rope(leaf, k, turns, positions=at, out=(torch.empty_like(q), torch.empty_like(k)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    x = torch.randn((2, 100), device="cuda", requires_grad=True)
    real = torch.empty(2, device="cuda")
    with pytest.raises(RuntimeError, match="gradient"):
        ams.ams_logprobs(x, out=ams.LogProbs(None, None, real, None, None))
    with torch.no_grad():
        assert ams.ams_logprobs(x, out=ams.LogProbs(None, None, real, None, None)).entropy is real
    assert torch.equal(ams.ams_logprobs(x.detach()).entropy, real)

    class Rotated(torch.autograd.Function):  # how a training program has them
        @staticmethod
        def forward(ctx, x):
            return ams.ams_rope(x, None, turns, positions=at)[0]

        @staticmethod
        def backward(ctx, g):
            return ams.ams_rope(g.contiguous(), None, turns, positions=at, transposed=True)[0]

    y = Rotated.apply(leaf)
    y.backward(k.expand(3, 2, 64))
    assert torch.equal(y.detach(), want[0]) and torch.equal(leaf.grad, ams.ams_rope(k.expand(3, 2, 64).contiguous(), None, turns, positions=at, transposed=True)[0])
