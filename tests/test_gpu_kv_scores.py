"""Attention over the 4-bit KV cache with capped scores, a bias by distance and prefixes that every row sees, against the definition in 64 bits.

Bound: that of plain scores (2^-11 of the weights and 2e-5 for scores of fp32), and what the capped and biased scores are off by themselves:
the hyperbolic tangent by 2^-22 of the cap, times what it is in log2 (1.45) 2^-21.4, roundings of fp32 2^-24 of the bias each, three of them."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O
from tests.test_gpu_kv_attention import Case, counts_are_zero, workspace  # noqa: F401  (the fixtures of that file)
from tests.test_gpu_kv_cache import SIZES, dev, host, rows_of, starts_of, write_all
from tests.test_gpu_kv_variants import lengths, plan_of, variants

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Scored(Case):
    def __init__(self, lens, counts, softcap=0.0, bias=False, prefix=None, **more):
        super().__init__(lens, counts, **more)
        self.softcap, self.prefix = softcap, prefix
        self.slopes = np.array([2.0 ** (-8.0 * (h + 1) / self.heads) for h in range(self.heads)], dtype=np.float32) if bias else None

    def scores(self):
        return dict(softcap=self.softcap, slopes=None if self.slopes is None else dev(self.slopes), prefix_lens=None if self.prefix is None else dev(np.array(self.prefix, dtype=np.int32)))

    def check(self, heads=None, **more):
        """heads: only those, where each has a kv head of its own and all would take the oracle long."""
        lse = torch.full((len(self.q), self.heads), 7.0, dtype=torch.float32, device="cuda")
        out, lse = host(self.run(lse=lse, **self.scores(), **more)).astype(np.float64), lse.cpu().numpy().astype(np.float64)
        all_slopes, q = self.slopes, self.q
        if heads is not None:
            out, lse, q, all_slopes = out[:, heads], lse[:, heads], q[:, heads], None if all_slopes is None else all_slopes[heads]
        at = 0
        for b, ((k, v), n) in enumerate(zip(self.seqs, self.counts)):
            if n == 0:
                continue
            k, v = (O.held(x if heads is None else x[:, heads], self.G) for x in (k, v))
            prefix = 0 if self.prefix is None else min(max(self.prefix[b], 0), len(k))
            want, want_lse, size = O.scored_attention(q[at : at + n], k, v, more.get("softmax_scale", self.D**-0.5), self.causal, self.window, self.softcap, all_slopes, prefix)
            biased = 0 if all_slopes is None else min(float(np.abs(all_slopes).max()) * (len(k) + n), 200.0)  # a key further off has no weight: scores here are within 50 or so
            inexact = 2.0**-21.4 * self.softcap + 3 * 2.0**-24 * biased * 1.45
            bound = (2.0**-11 + 2e-5 + inexact) * (np.abs(want) + size) + 2.0**-24 + len(k) * 2.0**-32 * (size + 1)
            off = np.abs(out[at : at + n] - want) / bound
            assert off.size == 0 or off.max() <= 1, (b, off.max(), np.unravel_index(off.argmax(), off.shape))
            got = lse[at : at + n]
            assert np.array_equal(np.isinf(got), np.isinf(want_lse))
            there = np.isfinite(want_lse)
            assert np.all(np.abs(got[there] - want_lse[there]) <= 1e-5 * (1 + np.abs(want_lse[there])) + inexact), b
            at += n
        return out


ALL = dict(softcap=5.0, bias=True)
FORMS = [dict(softcap=50.0), dict(softcap=1.5), dict(bias=True), ALL]


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("form", FORMS)
def test_single_rows(D, G, form):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 0]
    Scored(lens, [1] * len(lens), D=D, G=G, **form).check()
    Scored(lens, [1] * len(lens), D=D, G=G, prefix=[0, 2, 40, 16, 1, 5, 32, 33, 64, 70, 129, 3, 9], window=20, **form).check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (7, 1), (32, 2), (17, 1), (96, 1)])
def test_head_layouts(heads, kv_heads):
    """Slopes are those of the query heads."""
    Scored([45, 200], [1, 1], heads=heads, kv_heads=kv_heads, **ALL).check()
    Scored([45, 200], [3, 6], heads=heads, kv_heads=kv_heads, D=64, G=64, prefix=[4, 50], **ALL).check()


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("causal,window,prefix", [(True, 0, None), (False, 0, None), (True, 1, None), (True, 37, None), (True, 0, [33, 2, 0, 64, 1]), (True, 1, [33, 2, 0, 64, 1]), (True, 37, [33, 2, 0, 64, 1])])
def test_several_rows(D, G, causal, window, prefix):
    Scored([70, 5, 33, 64, 130], [70, 5, 1, 17, 40], D=D, G=G, causal=causal, window=window, prefix=prefix, **ALL).check()


def test_rows_without_a_position():
    """More rows than tokens: those before the first see nothing, of the prefix neither; without a mask the bias goes by their distance."""
    Scored([3, 0, 40], [5, 2, 50], D=64, G=32, prefix=[2, 5, 30], **ALL).check()
    Scored([3, 0, 40], [5, 2, 50], D=64, G=32, causal=False, **ALL).check()
    Scored([3, 0, 400], [5, 2, 600], heads=2, kv_heads=1, D=64, G=32, prefix=[2, 5, 100], bias=True).check(max_q_len=600)


@pytest.mark.parametrize("prefix", [-5, 0, 1, 31, 32, 33, 64, 500, 640, 645, 700, 2000])
@pytest.mark.parametrize("window", [0, 1, 50, 600])
@pytest.mark.parametrize("count", [1, 40, 300, 700])
def test_prefixes(prefix, window, count):
    """Single rows, a draft, a prompt, a whole sequence: before, inside, at the end of and beyond the window and the rows."""
    Scored([700], [count], heads=2, kv_heads=1, D=64, G=32, page=16, prefix=[prefix], window=window, softcap=0.0).check(max_q_len=count)


@pytest.mark.parametrize("D,G,columns,waves,split", variants())
def test_every_kernel_for_few_rows(D, G, columns, waves, split):
    """As in the test of plain scores: every variant by its plan, whole tiles, parts of one tile, shares that cross tiles."""
    if waves == 8:
        kv_heads, batch, idle = {"whole": (8, 7, 0), "parts": (8, 7, 0), "across": (32, 7, 0)}[split]
    else:
        kv_heads, batch, idle = {"whole": (64, 7, 0), "parts": (64, 4, 3), "across": (64, 7, 0)}[split]
    count = 1 if columns == 1 else 16 * columns - 3
    n = batch + idle
    lens = lengths(n, 1000 if split == "whole" else 1100, count)
    counts = [count if b < batch else 0 for b in range(n)]
    if split == "parts" and idle:
        lens[1], lens[n // 2] = 1100, 70
    prefix = [[0, 40, 1, 333, 64, 7, 1100][b % 7] for b in range(n)]
    c = Scored(lens, counts, heads=kv_heads, kv_heads=kv_heads, D=D, G=G, page=64, prefix=prefix, **ALL)
    ws = torch.zeros(ams.KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    for c.softcap, c.window, c.prefix in ((c.softcap, 0, prefix), (0.0, 200, prefix), (c.softcap, 0, None)):
        plan = plan_of(c)
        assert (plan["kernel"], plan["rows"], plan["waves"]) == ("stream", 16 * columns, waves), plan
        c.check(heads=[0, kv_heads - 1], max_q_len=count, workspace=ws)
        assert not bool(ws[:65536].any())


@pytest.mark.parametrize("D,G,waves", [(D, G, waves) for D, G in SIZES for waves in (4, 8) if waves == 4 or D < 256])
def test_every_kernel_for_prompts(D, G, waves):
    # 1284 rows of 64 heads: 640 tiles of 128 rows; a table for 4096 keys makes them 256 rows
    c = Scored([1300, 260], [1024, 260], heads=64, kv_heads=64, D=D, G=G, page=64, spare=60 if waves == 8 else 1, **ALL)
    for c.softcap, c.window, c.prefix in ((5.0, 0, [100, 1300]), (0.0, 300, [64, 0]), (30.0, 0, None), (0.0, 129, None)):
        plan = plan_of(c)
        assert (plan["kernel"], plan["waves"]) == ("tile", 8 if waves == 8 and not 0 < c.window < 4096 else 4), plan
        c.check(heads=[0, 63], max_q_len=1024)


def test_a_window_s_sinks_far_behind():
    """The first keys and the last ones of long sequences, in one row each and in prompts: what lies between is not looked at."""
    Scored([9000, 5000, 70], [1, 1, 1], heads=4, kv_heads=1, window=100, prefix=[4, 70, 64], page=64).check()
    Scored([9000, 5000], [30, 30], heads=4, kv_heads=1, window=100, prefix=[4, 200], page=64, bias=True).check()
    Scored([6000], [600], heads=4, kv_heads=2, window=100, prefix=[130], page=64).check(max_q_len=600)


@pytest.mark.parametrize("workspace", ["own", None, 200000])
def test_pieces(workspace):
    c = Scored([3000, 5, 1111, 0, 260], [1] * 5, heads=8, kv_heads=1, prefix=[2500, 9, 33, 4, 0], window=500, **ALL)
    ws = workspace if workspace in ("own", None) else torch.zeros(workspace, dtype=torch.uint8, device="cuda")
    c.check(workspace=ws)
    a = c.run(workspace=ws, **c.scores())
    for _ in range(3):
        assert torch.equal(a, c.run(workspace=ws, **c.scores()))


def test_more_sequences_than_a_wavefront_has_lanes():
    rng = np.random.default_rng(9)
    lens = [int(n) for n in rng.integers(0, 60, 150)]
    lens[70] = 2000
    prefix = [int(n) for n in rng.integers(0, 40, 150)]
    Scored(lens, [1] * 150, heads=2, kv_heads=1, D=64, G=32, page=16, prefix=prefix, window=30, **ALL).check()


@pytest.mark.parametrize("gain", [0.0, 30.0, 1000.0])
@pytest.mark.parametrize("count", [1, 200])
def test_capped_scores_of_any_size(gain, count):
    """At the cap the weights of many keys are alike; the cap keeps fp32 scores of thousands from being off."""
    Scored([600], [count], heads=2, kv_heads=1, gain=gain, softcap=50.0).check(max_q_len=count)


@pytest.mark.parametrize("softcap", [0.01, 1e-6, 1e4, 1e8])
def test_caps_of_any_size(softcap):
    """Next to nothing: all keys alike; beyond the scores: next to plain ones, to 2^-21.4 of the cap."""
    c = Scored([300], [3], heads=2, kv_heads=1, softcap=softcap)
    if softcap < 1e8:
        c.check()
    else:
        assert np.isfinite(host(c.run(**c.scores()))).all()


def test_steep_slopes():
    """Biases of thousands, where nearly all weight lies on the row's own key, and of millions."""
    for steep in (30.0, 1e4):
        for count in (1, 9, 300):
            c = Scored([400], [count], heads=2, kv_heads=1, bias=True)
            c.slopes[:] = steep
            c.check(max_q_len=count)


def test_slopes_below_zero():
    """A bias towards far keys."""
    c = Scored([200], [5], heads=4, kv_heads=2, bias=True)
    c.slopes *= -0.1
    c.check()


def test_what_unseen_keys_hold_has_no_effect():
    for D, G, count in ((128, 32, 1), (64, 64, 5), (128, 128, 40), (256, 32, 9), (64, 32, 300)):
        n = 100 if count < 100 else 400
        c = Scored([n], [count], D=D, G=G, window=20, prefix=[10], **ALL)
        want = c.run(**c.scores(), max_q_len=count)
        k, v = (x.copy() for x in c.seqs[0])
        k[10 : n - count - 20 + 1], v[10 : n - count - 20 + 1] = np.nan, np.inf
        write_all(c.cache, c.table, [(k, v)], G)
        assert torch.equal(c.run(**c.scores(), max_q_len=count), want)


@pytest.mark.parametrize("D,G,count", [(128, 32, 40), (64, 64, 9), (256, 128, 20), (128, 128, 300), (64, 32, 600)])
def test_nan_in_the_prefix_reaches_every_row(D, G, count):
    n = max(200, count)
    c = Scored([n], [count], D=D, G=G, window=8, prefix=[5], softcap=20.0)
    want = host(c.run(**c.scores(), max_q_len=count)).copy()
    k, v = (x.copy() for x in c.seqs[0])
    v[4, 1, 0] = np.inf
    write_all(c.cache, c.table, [(k, v)], G)
    out = host(c.run(**c.scores(), max_q_len=count))
    assert np.array_equal(out[:, :2], want[:, :2]) and np.isnan(out[:, 2:, :G]).all() and np.array_equal(out[:, 2:, G:], want[:, 2:, G:])
    v[4, 1, 0], k[4, 1, 0] = 0, np.nan
    write_all(c.cache, c.table, [(k, v)], G)
    out = host(c.run(**c.scores(), max_q_len=count))
    assert np.array_equal(out[:, :2], want[:, :2]) and np.isnan(out[:, 2:]).all()
    # behind the prefix and the window of the last rows: the rows before them
    k[4, 1, 0], k[5, 1, 0] = 0, np.nan
    write_all(c.cache, c.table, [(k, v)], G)
    out = host(c.run(**c.scores(), max_q_len=count))
    seeing = (np.arange(n - count, n) >= 5) & (np.arange(n - count, n) < 5 + 8)
    assert np.isnan(out[seeing, 2:]).all() and np.isfinite(out[~seeing]).all()


def test_pages_that_are_not_there_are_left_out():
    for count in (1, 200):
        c = Scored([300], [count], heads=2, kv_heads=1, page=16, prefix=[90], window=100, bias=True)
        c.table[0, 3] = -1
        c.table[0, 16] = 1 << 20
        out = host(c.run(**c.scores(), max_q_len=count))
        k, v = (O.held(x, 32) for x in c.seqs[0])
        there = np.ones(300, dtype=bool)
        there[48:64] = there[256:272] = False
        for i in range(0, count, 7):
            p = 300 - count + i
            at = np.nonzero(there & (((np.arange(300) <= p) & (np.arange(300) > p - 100)) | (np.arange(300) < 90)))[0]
            for h in range(2):
                s = c.q[i, h].astype(np.float64) @ k[at, 0].T * c.D**-0.5 - c.slopes[h] * np.abs(p - at)
                w = np.exp(s - s.max())
                want, size = w @ v[at, 0] / w.sum(), w @ np.abs(v[at, 0]) / w.sum()
                assert np.all(np.abs(out[i, h] - want) <= (2.0**-11 + 5e-5) * (np.abs(want) + size) + 2.0**-24)


def test_a_captured_step_follows_lengths_and_prefixes():
    c = Scored([300, 40, 9], [1, 1, 1], heads=4, kv_heads=2, window=32, prefix=[4, 4, 4], **ALL)
    s, q, out, ws = c.scores(), dev(c.q), torch.zeros((3, 4, 128), dtype=torch.float16, device="cuda"), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    ams.ams_init()
    c.kv_lens -= 8
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.kv_lens += 1
        s["prefix_lens"] += 2
        c.run(q=q, out=out, workspace=ws, **s)
    for i in range(5):
        q.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.run(q=q, workspace=ws, **s)), i
        assert bool(out.any())


def test_on_another_stream():
    c = Scored([500, 40], [1, 1], **ALL)
    s = c.scores()
    want, q = c.run(**s), dev(c.q)
    side = torch.cuda.Stream()
    ws, out = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(q=q * 1, workspace=ws, out=out, **s)
    side.synchronize()
    assert torch.equal(out, want)


def test_nothing_asked_for_is_plain_attention():
    c = Scored([500, 40], [20, 3])
    assert torch.equal(c.run(), c.run(softcap=0.0, slopes=None, prefix_lens=None))
    c.slopes, c.prefix = np.zeros(4, dtype=np.float32), [0, 0]
    c.check()


def test_row_starts_that_make_no_sense_touch_nothing_else():
    c = Scored([60, 40, 20], [3, 2, 4], heads=2, kv_heads=1, prefix=[1 << 30, -7, 12], window=9, **ALL)
    q = dev(c.q)
    for starts in ([0, 100, 50, 9], [5, 2, 8, -4], [1 << 30, 0, 0, 0], [-5, -5, 3, 1 << 30]):
        for hint in (None, 100):
            store = torch.full((c.q.shape[0] + 2, 2, 128), 7.0, dtype=torch.float16, device="cuda")
            ams.ams_kv_attention(q, c.cache, c.table, c.kv_lens, c.G, q_starts=dev(np.array(starts, dtype=np.int32)), max_q_len=hint, workspace=None, out=store[1:-1], window=9, **c.scores())
            assert bool((store[0] == 7).all()) and bool((store[-1] == 7).all())


def test_refusals():
    c = Scored([50], [1])
    half = torch.zeros(4, dtype=torch.float16, device="cuda")
    for error, more in [
        (ams.AmsError, dict(softcap=-1.0)), (ams.AmsError, dict(softcap=float("nan"))), (ams.AmsError, dict(softcap=float("inf"))), (ValueError, dict(slopes=torch.zeros(3, device="cuda"))),
        (TypeError, dict(slopes=half)), (ValueError, dict(slopes=torch.zeros(4))), (ValueError, dict(prefix_lens=torch.zeros(2, dtype=torch.int32, device="cuda"))),
        (TypeError, dict(prefix_lens=torch.zeros(1, device="cuda"))),
    ]:
        with pytest.raises(error):
            c.run(**more)
    c.causal = False
    with pytest.raises(ams.AmsError):
        c.run(prefix_lens=torch.zeros(1, dtype=torch.int32, device="cuda"))
