"""The calls of rotary positions, log probabilities and scored attention in native code (csrc/ams_binding.cpp) against the same calls in
Python: the same results, and everything that is not a plain tensor or that is wrong takes the long way and raises there."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")

ams._bind_call()


def native():
    from paper_2510_16045_amd import _binding

    return _binding


def test_what_is_not_on_the_gpu_or_no_tensor_is_left_alone():
    b, q, at, turns = native(), torch.zeros((2, 1, 64), dtype=torch.float16), torch.zeros(2, dtype=torch.int32), torch.zeros(32, dtype=torch.int64)
    assert b.rope() is None and b.rope(q, None, turns, at, None, None, 1.0, False, False, q, None) is None
    x = torch.zeros((2, 10), dtype=torch.float16)
    assert b.logprobs() is None and b.logprobs(x, None, 0, 1.0, None, None, None, None, None, None) is None
    assert b.rope(*[None] * 11) is None and b.logprobs(*[None] * 10) is None


@pytest.fixture
def problem():
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((7, 4 + 2, 128), generator=gen, device="cuda").half()
    lens, starts = torch.tensor([20, 40], dtype=torch.int32, device="cuda"), torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda")
    turns = torch.from_numpy(ams.ams_rope_frequencies(64)[0]).cuda()
    logits, tokens = torch.randn((7, 5000), generator=gen, device="cuda").half(), torch.arange(7, dtype=torch.int32, device="cuda")
    cache = torch.randint(0, 100, (6, 2, ams.ams_kv_block_bytes(128, 16, 64)), generator=gen, device="cuda").to(torch.uint8)
    return dict(q=x[:, :4], k=x[:, 4:], lens=lens, starts=starts, turns=turns, logits=logits, tokens=tokens, ws=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), cache=cache,
                table=torch.tensor([[3, 1, -1], [0, 5, 2]], dtype=torch.int32, device="cuda"), at=torch.arange(7, dtype=torch.int32, device="cuda") * 99)


def all_calls(p):
    q, k = torch.zeros((7, 4, 128), dtype=torch.float16, device="cuda"), torch.zeros((7, 2, 128), dtype=torch.float16, device="cuda")
    a = ams.ams_rope(p["q"], p["k"], p["turns"], kv_lens=p["lens"], q_starts=p["starts"], out=(q, k))
    b = ams.ams_rope(p["q"], None, p["turns"], positions=p["at"], magnitude=1.5, interleaved=True, transposed=True, out=(torch.zeros_like(q), None))
    real, whole = (lambda *n: torch.zeros(n, device="cuda")), (lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda"))
    c = ams.ams_logprobs(p["logits"], p["tokens"], top=5, temperature=0.7, workspace=p["ws"], out=ams.LogProbs(real(7), whole(7), real(7), real(7, 5), whole(7, 5)))
    d = ams.ams_logprobs(p["logits"].float(), workspace=p["ws"], out=ams.LogProbs(None, None, real(7), None, None))
    lse = real(7, 4)
    e = ams.ams_kv_attention(p["q"], p["cache"], p["table"], p["lens"], 64, q_starts=p["starts"], workspace=p["ws"], out=torch.zeros_like(q), lse=lse, window=9, softcap=3.0,
                             slopes=torch.arange(4, device="cuda") / 8, prefix_lens=torch.tensor([1, 2], dtype=torch.int32, device="cuda"))
    return [*a, b[0], *c, d.entropy, e, lse]


@pytest.mark.gpu
def test_the_same_either_way(problem, monkeypatch):
    taken = []
    for name in ("_rope_call", "_logprobs_call", "_kv_call"):
        call = getattr(ams, name)
        monkeypatch.setattr(ams, name, lambda *a, call=call: taken.append(call(*a)) or taken[-1])
    fast = all_calls(problem)
    assert taken == [True] * 5
    for name in ("_rope_call", "_logprobs_call", "_kv_call"):
        monkeypatch.setattr(ams, name, lambda *a: None)
    for x, y in zip(fast, all_calls(problem)):
        assert torch.equal(x, y) and bool(x.any())


@pytest.mark.gpu
def test_the_current_stream(problem):
    want = all_calls(problem)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_calls(problem)
    side.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


class Sub(torch.Tensor):
    pass


@pytest.mark.gpu
def test_rotations_that_are_wrong_take_the_long_way(problem):
    p, b = problem, native()
    q, k = torch.zeros((7, 4, 128), dtype=torch.float16, device="cuda"), torch.zeros((7, 2, 128), dtype=torch.float16, device="cuda")
    good = [p["q"], p["k"], p["turns"], None, p["lens"], p["starts"], 1.0, False, False, q, k]
    assert b.rope(*good) is True
    for i, bad in ((0, p["q"][0]), (0, p["q"].float()), (0, p["q"][:6]), (0, p["q"].cpu()), (0, p["q"].transpose(1, 2)), (0, p["q"].as_subclass(Sub)), (1, None), (1, p["k"][:, :, :64]), (1, p["k"][:6]), (2, p["turns"].int()),
                   (2, p["turns"][:0]), (2, torch.zeros(65, dtype=torch.int64, device="cuda")), (3, p["at"]), (4, None), (4, p["lens"][:1]), (4, p["lens"].long()), (5, p["starts"][:2]), (6, "1"), (6, float("nan")),
                   (7, 1), (8, 0), (9, q[:6]), (9, q[:, :3]), (10, None), (10, k[:, :1])):
        assert b.rope(*good[:i], bad, *good[i + 1 :]) is None, (i, bad)
    assert b.rope(*good[:3], p["at"], None, None, *good[6:]) is True
    assert b.rope(*good[:3], p["at"][:6], None, None, *good[6:]) is None and b.rope(*good[:3], None, None, None, *good[6:]) is None and b.rope(*good[:3], p["at"], None, p["starts"], *good[6:]) is None
    with pytest.raises(ValueError):
        ams.ams_rope(p["q"], p["k"], p["turns"], kv_lens=p["lens"], q_starts=p["starts"], out=(q[:6], k))


@pytest.mark.gpu
def test_log_probabilities_that_are_wrong_take_the_long_way(problem):
    p, b = problem, native()
    real, whole = (lambda *n: torch.zeros(n, device="cuda")), (lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda"))
    good = [p["logits"], p["tokens"], 5, 1.0, p["ws"], real(7), whole(7), real(7), real(7, 5), whole(7, 5)]
    assert b.logprobs(*good) is True
    for i, bad in ((0, p["logits"][0]), (0, p["logits"].bfloat16()), (0, p["logits"].cpu()), (0, p["logits"].t()), (0, p["logits"].as_subclass(Sub)), (1, p["tokens"][:6]), (1, p["tokens"].long()), (1, None), (2, 65), (2, -1),
                   (2, 4), (2, 5.0), (3, 0.0), (3, "1"), (4, p["ws"].cpu()), (5, real(6)), (5, whole(7)), (6, real(7)), (7, whole(7)), (8, None), (8, real(7, 4)), (8, real(5, 7).t()), (9, real(7, 5)), (9, None)):
        assert b.logprobs(*good[:i], bad, *good[i + 1 :]) is None, (i, bad)
    assert np.isfinite(good[7].cpu().numpy()).all()


@pytest.mark.gpu
def test_scores_that_are_wrong_take_the_long_way(problem):
    p, b = problem, native()
    out, slopes, prefix = torch.zeros((7, 4, 128), dtype=torch.float16, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    good = [3, p["cache"], p["table"], p["lens"], 64, p["starts"], p["q"], out, None, None, True, 0, p["ws"], None, 2.0, slopes, prefix]
    assert b.kv(*good) is True
    for i, bad in ((0, 2), (6, p["q"].float()), (10, False), (14, -1.0), (14, "2"), (14, float("nan")), (15, slopes[:3]), (15, slopes.half()), (15, slopes.cpu()), (16, prefix[:1]), (16, prefix.long()), (16, prefix.view(1, 2))):
        assert b.kv(*good[:i], bad, *good[i + 1 :]) is None, (i, bad)
    assert b.kv(*good[:14], 0, None, None) is True and b.kv(*good[:14]) is None
