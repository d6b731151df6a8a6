"""Rotary positions on the GPU against the definition in 64 bits.

Tolerance: cos and sin are off by at most 2^-23 (angle 2^-29 turns after its conversion to 24 bits, series and roundings of 2^-24 each),
products and their sum by 2^-24 each, together below 2^-21 (|a| + |b|) |magnitude|; then one rounding to fp16, half a step of the result,
2^-11 of it or 2^-25 where it is subnormal."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BASE = 10000.0


def turns_of(rot, base=BASE):
    turns, _ = ams.ams_rope_frequencies(rot, base)
    return torch.from_numpy(turns).cuda()


def rotated(x, positions, rot, interleaved=False, transposed=False, magnitude=1.0, base=BASE):
    """(values, bound) in 64 bits."""
    y = x.cpu().double().numpy().copy()
    w = base ** (-2 * np.arange(rot // 2) / rot) * (-1 if transposed else 1)
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * w
    c, s = np.cos(angle), np.sin(angle)
    i = np.arange(rot // 2) * (2 if interleaved else 1)
    j = i + (1 if interleaved else rot // 2)
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = magnitude * (a * c - b * s), magnitude * (b * c + a * s)
    size = np.zeros_like(y)
    size[..., i] = size[..., j] = (np.abs(a) + np.abs(b)) * abs(magnitude)
    return y, size * 2.0**-21 + np.maximum(np.abs(y) * 2.0**-11, 2.0**-25)


def check(got, x, positions, rot, **more):
    want, bound = rotated(x, positions, rot, **more)
    got = got.cpu().double().numpy()
    off = np.abs(got - want) / bound
    assert off.max() <= 1, (off.max(), np.unravel_index(off.argmax(), off.shape))
    assert np.array_equal(got[..., rot:], x.cpu().double().numpy()[..., rot:])


def rows(n, heads, dim, seed=0):
    return torch.randn((n, heads, dim), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").half()


SIZES = [(128, 128), (128, 64), (64, 64), (256, 64), (80, 80), (80, 20), (96, 24), (112, 56), (2, 2), (50, 6), (7, 4), (512, 512), (1024, 1024), (1000, 998)]


@pytest.mark.parametrize("dim,rot", SIZES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,kv_heads", [(1, 32, 8), (5, 3, 1), (70, 12, 12)])
def test_given_positions(dim, rot, interleaved, n, heads, kv_heads):
    q, k = rows(n, heads, dim), rows(n, kv_heads, dim, 1)
    at = torch.tensor([(i * 7919) % 131072 for i in range(n)], dtype=torch.int32, device="cuda")
    got = ams.ams_rope(q, k, turns_of(rot), positions=at, interleaved=interleaved)
    for x, y in zip((q, k), got):
        check(y, x, at.tolist(), rot, interleaved=interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions(interleaved):
    at = [0, 1, -1, 131071, 1048575, -131071, 2**31 - 1, -(2**31), 65536, 12345678]
    q = rows(len(at), 4, 128)
    # at 2^31 the definition's own angle is off by 2^31 2^-53 radians, far below the bound
    got, none = ams.ams_rope(q, None, turns_of(128), positions=torch.tensor(at, dtype=torch.int32, device="cuda"), interleaved=interleaved)
    assert none is None
    check(got, q, at, 128, interleaved=interleaved)
    assert torch.equal(got[0], q[0])  # not rotated at all


@pytest.mark.parametrize("scaling,factor,trained", [("linear", 4.0, 0), ("ntk", 8.0, 0), ("bands", 8.0, 8192), ("yarn", 4.0, 8192)])
def test_scaled(scaling, factor, trained):
    from test_rope import frequencies

    turns, magnitude = ams.ams_rope_frequencies(128, 500000.0, scaling, factor, trained)
    at = [0, 17, 8191, 65535, 131071]
    q = rows(len(at), 2, 128)
    got, _ = ams.ams_rope(q, None, torch.from_numpy(turns).cuda(), positions=torch.tensor(at, dtype=torch.int32, device="cuda"), magnitude=magnitude)
    x = q.cpu().double().numpy()
    angle = np.asarray(at, dtype=np.float64)[:, None, None] * np.array(frequencies(128, 500000.0, scaling, factor, trained))
    a, b = x[..., :64], x[..., 64:]
    want = magnitude * np.concatenate((a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)), -1)
    size = np.concatenate((np.abs(a) + np.abs(b),) * 2, -1) * magnitude
    assert (np.abs(got.cpu().double().numpy() - want) <= size * 2.0**-21 + np.maximum(np.abs(want) * 2.0**-11, 2.0**-25)).all()


STARTS = [([5, 20, 3], [0, 2, 7, 10]), ([5, 0, 9], [0, 1, 1, 4]), ([1], [0, 1]), ([2, 5], [0, 4, 6]), ([100] * 70, list(range(0, 213, 3))), ([9] * 200, [min(i, 150) for i in range(201)]), ([7, 8], [3, 5, 9])]


@pytest.mark.parametrize("lens,starts", STARTS)
@pytest.mark.parametrize("dim,rot", [(128, 128), (80, 20)])
def test_the_cache_s_rows(lens, starts, dim, rot):
    """The last rows of their sequences; rows before the first sequence and behind the last are left as they were."""
    n = starts[-1] + 4
    q, k = rows(n, 8, dim), rows(n, 2, dim, 1)
    out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    ams.ams_rope(q, k, turns_of(rot), kv_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), q_starts=torch.tensor(starts, dtype=torch.int32, device="cuda"), out=out)
    at = [lens[b] - starts[b + 1] + r for b in range(len(lens)) for r in range(starts[b], starts[b + 1])]
    for x, y in zip((q, k), out):
        check(y[starts[0] : starts[-1]], x[starts[0] : starts[-1]], at, rot)
        assert (y[: starts[0]] == 7).all() and (y[starts[-1] :] == 7).all()


def test_one_row_of_each_sequence():
    lens = [5, 131072, 0, 1, -3]
    q = rows(5, 4, 128)
    got, _ = ams.ams_rope(q, None, turns_of(128), kv_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    check(got, q, [max(x, 0) - 1 for x in lens], 128)


def test_starts_that_do_not_ascend_stay_within_the_rows():
    q = rows(6, 2, 64)
    out = torch.full((8, 2, 64), 7.0, dtype=torch.float16, device="cuda")
    lens, starts = torch.tensor([4, 4, 4], dtype=torch.int32, device="cuda"), torch.tensor([-5, 100, 2, 2**31 - 1], dtype=torch.int32, device="cuda")
    ams.ams_rope(q, None, turns_of(64), kv_lens=lens, q_starts=starts, out=(out[1:7], None))
    assert (out[0] == 7).all() and (out[7] == 7).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (256, 64), (80, 20)])
def test_in_place_in_a_projection(dim, rot, interleaved):
    """Views of one projection's output, rotated where they lie; what is beside them stays."""
    x = rows(9, 4 + 2 + 2, dim)
    before = x.clone()
    at = torch.arange(100, 109, dtype=torch.int32, device="cuda")
    q, k = x[:, :4], x[:, 4:6]
    got = ams.ams_rope(q, k, turns_of(rot), positions=at, interleaved=interleaved, out=(q, k))
    assert got[0] is q and got[1] is k
    want = ams.ams_rope(before[:, :4], before[:, 4:6], turns_of(rot), positions=at, interleaved=interleaved)
    assert torch.equal(x[:, :4], want[0]) and torch.equal(x[:, 4:6], want[1]) and torch.equal(x[:, 6:], before[:, 6:])


@pytest.mark.parametrize("shift", [1, 4])
def test_unaligned(shift):
    """Rows that are aligned to two or eight bytes only, of odd strides."""
    flat = torch.randn(4 * 1000, device="cuda").half()
    q = torch.as_strided(flat, (5, 3, 64), (431, 67, 1), shift)
    at = torch.arange(5, dtype=torch.int32, device="cuda") * 1000
    got, _ = ams.ams_rope(q, None, turns_of(64), positions=at)
    check(got, q, at.tolist(), 64)
    out = torch.zeros(4 * 1000, dtype=torch.float16, device="cuda")
    ams.ams_rope(q, None, turns_of(64), positions=at, out=(torch.as_strided(out, (5, 3, 64), (431, 67, 1), shift), None))
    assert torch.equal(torch.as_strided(out, (5, 3, 64), (431, 67, 1), shift), got)
    assert int((out != 0).sum()) <= 5 * 3 * 64


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("magnitude", [1.0, 1.25])
def test_the_gradient(interleaved, magnitude):
    """transposed takes the gradient of the outputs to that of the inputs: the formula's by autograd in 64 bits, and by differences."""
    n, rot, dim = 6, 48, 64
    x, g = rows(n, 3, dim), rows(n, 3, dim, 1)
    at = torch.tensor([0, 3, 77, 4095, 99999, -5], dtype=torch.int32, device="cuda")
    got, _ = ams.ams_rope(g, None, turns_of(rot), positions=at, interleaved=interleaved, transposed=True, magnitude=magnitude)
    check(got, g, at.tolist(), rot, interleaved=interleaved, transposed=True, magnitude=magnitude)
    leaf = x.cpu().double().requires_grad_()
    w = torch.tensor(BASE, dtype=torch.float64) ** (-2 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    angle = at.cpu().double()[:, None, None] * w
    c, s = magnitude * angle.cos(), magnitude * angle.sin()
    a, b = (leaf[..., :rot:2], leaf[..., 1:rot:2]) if interleaved else (leaf[..., : rot // 2], leaf[..., rot // 2 : rot])
    y = [a * c - b * s, b * c + a * s]
    y = torch.cat((torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1), leaf[..., rot:]), -1)
    (y * g.cpu().double()).sum().backward()
    bound = rotated(g, at.tolist(), rot, interleaved, True, magnitude)[1]
    assert (np.abs(got.cpu().double().numpy() - leaf.grad.numpy()) <= bound).all()
    # the map is linear: <g, rope(x + e) - rope(x)> = <rope^T g, e>, each side within its outputs' bounds
    e = rows(n, 3, dim, 2)
    moved, bounds = [], 0.0
    for z in ((x.double() + e.double()).half(), x):
        y, _ = ams.ams_rope(z, None, turns_of(rot), positions=at, interleaved=interleaved, magnitude=magnitude)
        moved.append(y.cpu().double().numpy())
        bounds += float((np.abs(g.cpu().double().numpy()) * rotated(z, at.tolist(), rot, interleaved, False, magnitude)[1]).sum())
    step = (x.double() + e.double()).half().double() - x.double()  # what was added, after its rounding
    left = float((g.cpu().double().numpy() * (moved[0] - moved[1])).sum())
    right = float((got.cpu().double().numpy() * step.cpu().numpy()).sum())
    assert abs(left - right) <= bounds + float((np.abs(step.cpu().numpy()) * bound).sum())


def test_there_and_back():
    q = rows(40, 8, 128)
    at = torch.arange(40, dtype=torch.int32, device="cuda") * 3001
    y, _ = ams.ams_rope(q, None, turns_of(128), positions=at)
    back, _ = ams.ams_rope(y, None, turns_of(128), positions=at, transposed=True)
    # two roundings: of y, whose error turns into that of the pair, and of the result
    pair = q.cpu().double().numpy()
    size = np.abs(pair[..., :64]) + np.abs(pair[..., 64:])
    bound = np.concatenate((size, size), -1) * (2.0**-11 * 2 + 2.0**-20) + 2.0**-11 * np.abs(pair) + 2.0**-23
    assert (np.abs(back.cpu().double().numpy() - pair) <= bound).all()


def test_captured_and_on_another_stream():
    q, k = rows(4, 8, 128), rows(4, 2, 128, 1)
    lens = torch.tensor([3, 900, 17, 60], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q), torch.empty_like(k)
    turns = turns_of(128)
    ams.ams_init()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens += 1
        ams.ams_rope(q, k, turns, kv_lens=lens, out=out)
    for _ in range(3):
        q.copy_(rows(4, 8, 128, int(lens[0])))
        graph.replay()
        want = ams.ams_rope(q, k, turns, kv_lens=lens)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = ams.ams_rope(q, k, turns, kv_lens=lens)
    side.synchronize()
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


def test_many_rows():
    """More rows than a wavefront each fills the chip with, and parts of a row on several wavefronts."""
    for n, heads in ((20011, 9), (300, 40), (1, 1000)):
        q = rows(n, heads, 64)
        at = (torch.arange(n, device="cuda") * 13 % 131072).to(torch.int32)
        got, _ = ams.ams_rope(q, None, turns_of(64), positions=at)
        pick = torch.linspace(0, n - 1, 50).long().unique()
        check(got[pick.cuda()], q[pick.cuda()], at.cpu()[pick].tolist(), 64)


def test_nothing_to_do():
    q = rows(1, 2, 64)[:0]
    got, _ = ams.ams_rope(q, None, turns_of(64), positions=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert got.shape == (0, 2, 64)
