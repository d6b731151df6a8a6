"""Log probabilities on the GPU against the definition in 64 bits.

Tolerances.  y = log2(e) / T (x - m) is off by at most 2^-22 of it or of m's product (the factor's rounding, the products' and the
difference's), 2^y by 2^-23 more; a lane adds at most vocab / 1024 + 8 terms of one sign to each of its sums, each addition off by 2^-24 of
it.  So log S is off by (vocab / 1024 + 40) 2^-23 plus what the terms' exponents are off, which their weights keep below 2^-22 (log vocab +
8), and a log probability by that and 2^-22 |it|; the entropy is a mean of such terms: the same, times one more than the largest weighed
distance, which is below log vocab + 2."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def workspace():
    return torch.zeros(ams.KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


def reference(logits, tokens, top, temperature):
    raw = logits.cpu().double().numpy()
    x = raw / temperature
    most = x.max(1, keepdims=True)
    with np.errstate(all="ignore"):
        x = x - np.where(np.isinf(most), 0, most)  # first: beside 3e38 the logarithm would vanish
        lp = np.where(x == -np.inf, -np.inf, x - np.log(np.exp(x).sum(1, keepdims=True)))
        entropy = -np.where(lp == -np.inf, 0, np.exp(lp) * np.where(lp == -np.inf, 0, lp)).sum(1)
    order = np.argsort(-raw, axis=1, kind="stable")
    rows = np.arange(len(raw))
    best = order[:, :top]
    t = np.asarray(tokens)
    ok = (t >= 0) & (t < raw.shape[1])
    safe = np.where(ok, t, 0)
    given = raw[rows, safe][:, None]
    ahead = ((raw > given) | ((raw == given) & (np.arange(raw.shape[1]) < safe[:, None]))).sum(1)
    return np.where(ok, lp[rows, safe], 0), np.where(ok, ahead, -1), entropy, np.take_along_axis(lp, best, 1), best


def check(got, logits, tokens, top, temperature=1.0):
    want = reference(logits, tokens, top, temperature)
    vocab = logits.shape[1]
    base = 2.0**-22 * (np.log(vocab) + 8) + 2.0**-23 * (vocab / 1024 + 40)
    for i in (0, 3):
        a, b = got[i].cpu().double().numpy()[:, : want[i].shape[1] if i else None] if i else got[i].cpu().double().numpy(), want[i]
        assert np.array_equal(a == -np.inf, b == -np.inf)
        there = b != -np.inf
        off = np.abs(a[there] - b[there]) / (base + 2.0**-22 * np.abs(b[there]))
        assert off.size == 0 or off.max() <= 1, (i, off.max())
    off = np.abs(got.entropy.cpu().double().numpy() - want[2]) / (base * (np.log(vocab) + 3))
    assert off.max() <= 1, off.max()
    assert np.array_equal(got.rank.cpu().numpy(), want[1])
    n = min(top, vocab)
    assert np.array_equal(got.top_tokens.cpu().numpy()[:, :n], want[4])
    assert (got.top_tokens.cpu().numpy()[:, n:] == -1).all() and (got.top_logprobs.cpu().numpy()[:, n:] == -np.inf).all()


def draw(rows, vocab, wide=False, seed=0, scale=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = scale * torch.randn((rows, vocab), generator=gen, device="cuda")
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    return (x if wide else x.half()), tokens


VOCABULARIES = [1, 2, 7, 8, 63, 64, 65, 500, 2047, 2048, 2049, 8191, 8193, 32000, 49999, 128256]


@pytest.mark.parametrize("vocab", VOCABULARIES)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("rows,top,with_workspace", [(1, 5, True), (3, 64, True), (17, 0, True), (2, 1, False), (5, 20, False)])
def test_sizes(workspace, vocab, wide, rows, top, with_workspace):
    x, tokens = draw(rows, vocab, wide)
    got = ams.ams_logprobs(x, tokens, top=top, workspace=workspace if with_workspace else None)
    check(got, x, tokens.tolist(), top)
    assert not workspace[: 64 << 10].any()  # counts are left at zero


@pytest.mark.parametrize("rows", [64, 300, 1100, 2500])
def test_many_rows(workspace, rows):
    x, tokens = draw(rows, 3001)
    check(ams.ams_logprobs(x, tokens, top=7, workspace=workspace), x, tokens.tolist(), 7)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("rows,vocab", [(256, 17000), (257, 17000), (3, 32768), (3, 32769), (128, 50001), (129, 50001), (200, 70001), (512, 9000), (513, 9000), (600, 40000)])
def test_every_split(workspace, rows, vocab, wide):
    """Rows in parts, whole on eight wavefronts or sixteen, and of many on four."""
    x, tokens = draw(rows, vocab, wide)
    got = ams.ams_logprobs(x, tokens, top=11, workspace=workspace)
    some = [0, 1, rows // 2, rows - 2, rows - 1]
    check(ams.LogProbs(*(t[some] for t in got)), x[some], tokens[some].tolist(), 11)
    alone = ams.ams_logprobs(x, tokens, top=11)
    assert torch.equal(got.top_tokens, alone.top_tokens) and torch.equal(got.rank, alone.rank)
    assert not workspace[: 64 << 10].any()


@pytest.mark.parametrize("temperature", [0.1, 0.7, 1.5, 100.0])
@pytest.mark.parametrize("wide", [False, True])
def test_temperature(workspace, temperature, wide):
    x, tokens = draw(4, 32000, wide)
    check(ams.ams_logprobs(x, tokens, top=9, temperature=temperature, workspace=workspace), x, tokens.tolist(), 9, temperature)


@pytest.mark.parametrize("with_workspace", [False, True])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values", "rising in 16ths"])
@pytest.mark.parametrize("wide", [False, True])
def test_orders(workspace, order, wide, with_workspace):
    """What a list that is filled as the row goes by could get wrong, and equal logits, of which the first count."""
    n = 20011
    i = torch.arange(n, device="cuda")
    x = {"rising": i / 1000.0, "falling": -i / 1000.0, "equal": 0.0 * i, "two values": (i % 3000 == 2999).float(), "rising in 16ths": torch.floor(i / 16.0) / 64}[order]
    x = x.view(1, -1).repeat(2, 1)
    x = x if wide else x.half()
    tokens = torch.tensor([5, 20010], dtype=torch.int32, device="cuda")
    for top in (1, 20, 64):
        check(ams.ams_logprobs(x, tokens, top=top, workspace=workspace if with_workspace else None), x, tokens.tolist(), top)


@pytest.mark.parametrize("with_workspace", [False, True])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("kept", [0, 1, 3, 500])
def test_ruled_out(workspace, kept, wide, with_workspace):
    """Rows of which few tokens are allowed, or none at all."""
    x, _ = draw(5, 30011, wide)
    gen = torch.Generator(device="cuda").manual_seed(7)
    allowed = torch.zeros_like(x, dtype=torch.bool)
    if kept:
        allowed.scatter_(1, torch.randint(0, 30011, (5, kept), generator=gen, device="cuda"), True)
    x = torch.where(allowed, x, -float("inf"))
    tokens = x.float().argmax(1).to(torch.int32)
    tokens[0] = 30010 if kept else 0
    got = ams.ams_logprobs(x, tokens, top=8, workspace=workspace if with_workspace else None)
    if kept:
        check(got, x, tokens.tolist(), 8)
    else:  # nothing is possible: log probabilities -inf, no entropy, the first tokens
        assert (got.logprob == -float("inf")).all() and (got.top_logprobs == -float("inf")).all() and (got.entropy == 0).all()
        assert torch.equal(got.top_tokens.cpu(), torch.arange(8, dtype=torch.int32).repeat(5, 1)) and torch.equal(got.rank, tokens)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("others", ["all", "most"])
def test_the_type_s_lowest_value(workspace, wide, others):
    """A mask of the type's lowest value: far below everything, or, where all are, a uniform row."""
    x, tokens = draw(3, 9000, wide)
    lowest = torch.finfo(x.dtype).min
    if others == "all":
        x[:] = lowest
    else:
        x[:, 10:] = lowest
        tokens %= 10
    check(ams.ams_logprobs(x, tokens, top=5, workspace=workspace), x, tokens.tolist(), 5)


@pytest.mark.parametrize("wide", [False, True])
def test_nan_and_infinity(workspace, wide):
    x, tokens = draw(4, 9000, wide)
    x[0, 8000], x[1, 5], x[2, :] = float("nan"), float("inf"), float("nan")
    before = x[0].clone()
    before[8000] = -float("inf")
    got = ams.ams_logprobs(x, tokens, top=3, workspace=workspace)
    assert got.logprob[:3].isnan().all() and got.entropy[:3].isnan().all() and got.top_logprobs[:2].isnan().all()
    assert got.top_tokens[1, 0] == 5 and (got.top_tokens[2] == -1).all()
    assert torch.equal(got.top_tokens[0].long(), torch.sort(before.float(), descending=True, stable=True)[1][:3])
    check(ams.LogProbs(*(t[3:] for t in got)), x[3:], tokens[3:].tolist(), 3)


def test_tokens_outside(workspace):
    x, tokens = draw(5, 1000)
    tokens[1], tokens[2], tokens[3] = -1, 1000, 2**31 - 1
    got = ams.ams_logprobs(x, tokens, top=2, workspace=workspace)
    check(got, x, tokens.tolist(), 2)
    assert (got.logprob[1:4] == 0).all() and (got.rank[1:4] == -1).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("vocab,stride,shift", [(5001, 5001, 0), (5000, 5007, 3), (4096, 4096, 1), (5000, 0, 1)])
def test_strides_and_alignment(workspace, wide, vocab, stride, shift):
    flat, _ = draw(1, 6 * 5100, wide)
    x = torch.as_strided(flat[0], (5, vocab), (stride, 1), shift)
    tokens = torch.arange(5, dtype=torch.int32, device="cuda") * 900
    check(ams.ams_logprobs(x, tokens, top=6, workspace=workspace), x, tokens.tolist(), 6)


def test_what_is_not_asked_for(workspace):
    x, tokens = draw(6, 20000)
    whole = ams.ams_logprobs(x, tokens, top=4, workspace=workspace)
    alone = ams.ams_logprobs(x, workspace=workspace)
    assert alone.logprob is None and alone.rank is None and alone.top_tokens.shape == (6, 0) and torch.equal(alone.entropy, whole.entropy)
    out = ams.LogProbs(torch.full((6,), 7.0, device="cuda"), None, None, None, None)
    got = ams.ams_logprobs(x, tokens, workspace=workspace, out=out)
    assert got.logprob is out.logprob and got.rank is None and torch.equal(got.logprob, whole.logprob)
    with pytest.raises(ValueError):
        ams.ams_logprobs(x, tokens, top=4, out=whole._replace(rank=torch.zeros(5, dtype=torch.int32, device="cuda")))
    with pytest.raises(TypeError):
        ams.ams_logprobs(x, tokens, top=4, out=whole._replace(rank=torch.zeros(6, device="cuda")))
    with pytest.raises(ValueError):
        ams.ams_logprobs(x, tokens[:5])
    with pytest.raises(ValueError):
        ams.ams_logprobs(x.t())
    with pytest.raises(ams.AmsError):
        ams.ams_logprobs(x, top=65)


def test_workspaces(workspace):
    """Too small a one is not used, nothing behind a view is written; the same results to the rounding of the sums."""
    x, tokens = draw(3, 60000)
    need = ams.ams_logprobs_workspace_bytes(x, 5)
    assert need > 0
    for size in (16, need - 16, need, need + 64):
        ws = torch.zeros(size + 256, dtype=torch.uint8, device="cuda")
        ws[size:] = 77
        check(ams.ams_logprobs(x, tokens, top=5, workspace=ws[:size]), x, tokens.tolist(), 5)
        assert (ws[size:] == 77).all()
        assert bool(ws[64 << 10 : size].any()) == (size >= need)


def test_deterministic(workspace):
    x, tokens = draw(9, 128256)
    first = ams.ams_logprobs(x, tokens, top=20, workspace=workspace)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, ams.ams_logprobs(x, tokens, top=20, workspace=workspace)))


def test_captured_and_on_another_stream(workspace):
    x, tokens = draw(8, 50001)
    ams.ams_init()
    out = ams.ams_logprobs(x, tokens, top=5, workspace=workspace)
    out = ams.LogProbs(*(torch.zeros_like(t) for t in out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ams.ams_logprobs(x, tokens, top=5, workspace=workspace, out=out)
    for seed in range(1, 4):
        y, t = draw(8, 50001, seed=seed)
        x.copy_(y), tokens.copy_(t)
        graph.replay()
        want = ams.ams_logprobs(x, tokens, top=5, workspace=workspace)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = ams.ams_logprobs(x, tokens, top=5, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_rows_behind_four_gigabytes(workspace):
    """Offsets of rows pass 32 bits."""
    x = torch.zeros((3, 128256), dtype=torch.float16, device="cuda")
    far = torch.empty(3 << 30, dtype=torch.float16, device="cuda")
    y = torch.as_strided(far, (3, 128256), ((1 << 30) + 7, 1), 5)
    x[:], tokens = draw(3, 128256)
    y.copy_(x)
    check(ams.ams_logprobs(y, tokens, top=5, workspace=workspace), x, tokens.tolist(), 5)


def test_nothing_to_do(workspace):
    got = ams.ams_logprobs(torch.zeros((0, 100), dtype=torch.float16, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), top=3, workspace=workspace)
    assert got.logprob.shape == (0,) and got.top_tokens.shape == (0, 3)
