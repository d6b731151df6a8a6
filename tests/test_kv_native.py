"""The calls of the KV cache in native code (csrc/ams_binding.cpp) against the same calls in Python: the same results, the current
stream, and everything that is not a plain tensor or that is wrong, which takes the long way and raises there."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")


ams._bind_call()


def native(*a):
    from paper_2510_16045_amd import _binding

    return _binding.kv(*a)


def long_way(monkeypatch):
    monkeypatch.setattr(ams, "_kv_call", lambda *a: None)


def test_what_is_not_on_the_gpu_or_no_tensor_is_left_alone():
    cache, rows = ams.ams_kv_cache(2, 1, 64, 16, 32, device="cpu"), torch.zeros((1, 1, 64), dtype=torch.float16)
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    assert native() is None and native(0) is None
    assert native(0, cache, table, lens, 32, None, rows, rows) is None
    assert native(1, cache, table, lens, 32, None, 64, rows, rows) is None
    assert native(2, cache, table, lens, 32, None, rows, rows, None, None, True, 0, None, None) is None
    assert native(0, None, table, lens, 32, None, rows, rows) is None and native("0", cache, table, lens, 32, None, rows, rows) is None


@pytest.fixture
def problem():
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((7, 4 + 2 * 2, 128), generator=gen, device="cuda").half()
    return dict(
        cache=ams.ams_kv_cache(6, 2, 128, 16, 64), table=torch.tensor([[3, 1, -1], [0, 5, 2]], dtype=torch.int32, device="cuda"), lens=torch.tensor([20, 40], dtype=torch.int32, device="cuda"),
        starts=torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda"), q=x[:, :4], k=x[:, 4:6], v=x[:, 6:], ws=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"),
    )


def all_three(p, **more):
    out = {n: torch.zeros((7, h, 128), dtype=torch.float16, device="cuda") for n, h in (("k", 2), ("v", 2), ("o", 4))}
    lse = torch.zeros((7, 4), device="cuda")
    ams.ams_kv_write(p["cache"], p["k"], p["v"], p["table"], p["lens"], 64, q_starts=p["starts"])
    ams.ams_kv_read(p["cache"], p["table"], p["lens"], 64, 128, q_starts=p["starts"], out=(out["k"], out["v"]))
    ams.ams_kv_attention(p["q"], p["cache"], p["table"], p["lens"], 64, q_starts=p["starts"], workspace=p["ws"], out=out["o"], lse=lse, **more)
    return [out["k"], out["v"], out["o"], lse]


@pytest.mark.gpu
@pytest.mark.parametrize("more", [{}, dict(causal=False), dict(window=9, max_q_len=4), dict(softmax_scale=0.5)])
def test_the_same_either_way(problem, monkeypatch, more):
    taken = []
    monkeypatch.setattr(ams, "_kv_call", lambda *a: taken.append(native(*a)) or taken[-1])
    fast = all_three(problem, **more)
    assert taken == [True] * 3
    long_way(monkeypatch)
    for x, y in zip(fast, all_three(problem, **more)):
        assert torch.equal(x, y) and bool(x.any())


@pytest.mark.gpu
def test_the_current_stream(problem):
    want = all_three(problem)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    problem["cache"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = all_three(problem)
    side.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.gpu
def test_what_is_wrong_takes_the_long_way(problem):
    p = problem
    out = torch.zeros((7, 4, 128), dtype=torch.float16, device="cuda")
    good = [2, p["cache"], p["table"], p["lens"], 64, p["starts"], p["q"], out, None, None, True, 0, p["ws"], None]
    assert native(*good) is True
    for i, bad in (
        (1, p["cache"].cpu()), (1, p["cache"][0]), (1, p["cache"][:, :, :-1]), (2, p["table"].long()), (2, p["table"][:1]), (2, p["table"].t()), (3, p["lens"][:1]), (3, np.zeros(2, np.int32)), (4, 48), (4, 64.0),
        (5, p["starts"][:2]), (6, p["q"][:, :3]), (6, p["q"].float()), (6, p["q"].transpose(1, 2)), (7, out[:6]), (8, 1.5), (9, 0.0), (9, 1), (10, 1), (11, -1), (12, p["ws"].cpu()), (13, torch.zeros(7, device="cuda")),
    ):
        assert native(*good[:i], bad, *good[i + 1 :]) is None, (i, bad)
    with pytest.raises(ams.AmsError):
        ams.ams_kv_attention(p["q"][:, :3], p["cache"], p["table"], p["lens"], 64, q_starts=p["starts"], out=out[:, :3])

    class Sub(torch.Tensor):
        pass

    assert native(*good[:6], p["q"].as_subclass(Sub), *good[7:]) is None
