"""Attention over the 4-bit KV cache against the definition in 64 bits.

Bound of an output: it is rounded to fp16 once (2^-11 of itself), and each weight before it once (2^-11 of the weight, so 2^-11 of
sum p |v|); scores are fp32 sums of up to 256 products, 1e-5 of the weights at the sizes here; weights below 2^-22 of the largest lose
up to 2^-33 of it each.  lse is fp32 throughout."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O
from tests.test_gpu_kv_cache import SIZES, dev, host, rows_of, starts_of, table_for, write_all

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
WORKSPACE = None


@pytest.fixture(autouse=True, scope="module")
def workspace():
    """One for all calls of this file, whatever their shapes; its counts are zero after each test."""
    global WORKSPACE
    WORKSPACE = torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")
    yield
    WORKSPACE = None


@pytest.fixture(autouse=True)
def counts_are_zero():
    yield
    assert not bool(WORKSPACE[:65536].any())


def near(out, want, size, keys):
    err = np.abs(out.astype(np.float64) - want)
    bound = (2.0**-11 + 2e-5) * (np.abs(want) + size) + 2.0**-24 + keys * 2.0**-32 * (size + 1)
    return bool(np.all(err <= bound)), float(np.max(err / bound))


class Case:
    def __init__(self, lens, counts, heads=4, kv_heads=2, D=128, G=32, page=32, seed=0, causal=True, window=0, gain=1.0, spare=1):
        rng = np.random.default_rng(seed + 31 * D + G + 7 * page)
        self.__dict__.update(lens=list(lens), counts=list(counts), D=D, G=G, causal=causal, window=window, heads=heads)
        table, n_pages = table_for(lens, page, rng, spare)
        self.table_host, self.table = table, dev(table)
        self.cache = ams.ams_kv_cache(n_pages, kv_heads, D, page, G)
        self.seqs = [(rows_of(rng, n, kv_heads, D), rows_of(rng, n, kv_heads, D)) for n in lens]
        if sum(lens):
            write_all(self.cache, self.table, self.seqs, G)
        self.q = (rng.standard_normal((sum(counts), heads, D)) * gain).astype(np.float16)
        self.kv_lens = dev(np.array(lens, dtype=np.int32))
        self.starts = None if all(c == 1 for c in counts) else starts_of(counts)

    def run(self, workspace="own", q=None, out=None, lse=None, **more):
        if workspace == "own":
            workspace = WORKSPACE
        return ams.ams_kv_attention(dev(self.q) if q is None else q, self.cache, self.table, self.kv_lens, self.G, q_starts=self.starts, causal=self.causal, window=self.window,
                                    workspace=workspace, out=out, lse=lse, **more)

    def want(self, scale=None):
        outs, lses, sizes, at = [], [], [], 0
        for (k, v), n in zip(self.seqs, self.counts):
            o, l, s = O.attention(self.q[at : at + n], O.held(k, self.G), O.held(v, self.G), scale or self.D**-0.5, self.causal, self.window) if len(k) >= n else self.short(k, v, at, n)
            outs.append(o), lses.append(l), sizes.append(s)
            at += n
        return np.concatenate(outs), np.concatenate(lses), np.concatenate(sizes)

    def short(self, k, v, at, n):  # more rows than tokens: the first ones have no position
        no = n - len(k)
        o, l, s = O.attention(self.q[at + no : at + n], O.held(k, self.G), O.held(v, self.G), self.D**-0.5, self.causal, self.window)
        o0, l0, s0 = np.zeros((no, *o.shape[1:])), np.full((no, l.shape[1]), -np.inf), np.zeros((no, *o.shape[1:]))
        if not self.causal and len(k):  # without a mask their position is of no account
            o0, l0, s0 = O.attention(self.q[at : at + no], O.held(k, self.G), O.held(v, self.G), self.D**-0.5, False) if no <= len(k) else (o0, l0, s0)
        return np.concatenate([o0, o]), np.concatenate([l0, l]), np.concatenate([s0, s])

    def check(self, **more):
        lse = torch.full((len(self.q), self.heads), 7.0, dtype=torch.float32, device="cuda")
        out = host(self.run(lse=lse, **more))
        want, want_lse, size = self.want()
        ok, worst = near(out, want, size, max(self.lens, default=0))
        assert ok, worst
        got = lse.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isinf(got), np.isinf(want_lse))
        at = np.isfinite(want_lse)
        assert np.all(np.abs(got[at] - want_lse[at]) <= 1e-5 * (1 + np.abs(want_lse[at])))
        return out


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("page", [16, 64])
def test_single_rows(D, G, page):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 0]
    Case(lens, [1] * len(lens), D=D, G=G, page=page).check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (7, 1), (32, 2), (17, 1), (40, 2), (96, 1)])
def test_head_layouts(heads, kv_heads):
    Case([45, 200], [1, 1], heads=heads, kv_heads=kv_heads).check()
    Case([45, 200], [3, 6], heads=heads, kv_heads=kv_heads, D=64, G=64).check()


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 37)])
def test_several_rows(D, G, causal, window):
    Case([70, 5, 33, 64, 130], [70, 5, 1, 17, 40], D=D, G=G, causal=causal, window=window).check()


@pytest.mark.parametrize("D,G", [(64, 32), (128, 32), (128, 128), (256, 64)])
@pytest.mark.parametrize("hint", [None, 1, 150])
def test_prompts(D, G, hint):
    # 150 and 129 rows of two heads to a kv head: more than any one tile; hints that are wrong choose another kernel, not other results
    Case([150, 400, 16], [150, 129, 3], D=D, G=G, page=16).check(max_q_len=hint)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100)])
def test_long_prompt(causal, window):
    Case([700], [520], heads=2, kv_heads=1, causal=causal, window=window, page=64).check()


def test_rows_without_a_key():
    # more rows than tokens, and no token at all
    Case([3, 0, 40], [5, 2, 50], D=64, G=32).check()
    assert not host(Case([0, 0], [1, 1], heads=2).run(workspace=None)).any()


@pytest.mark.parametrize("workspace", ["own", None, 200000, 16])
def test_pieces(workspace):
    c = Case([3000, 5, 1111, 0, 260], [1] * 5, heads=8, kv_heads=1)
    ws = workspace if workspace in ("own", None) else torch.zeros(workspace, dtype=torch.uint8, device="cuda")
    c.check(workspace=ws)
    a = c.run(workspace=ws)
    for _ in range(3):
        assert torch.equal(a, c.run(workspace=ws))


def test_pieces_of_several_rows_and_windows():
    Case([2500, 900], [9, 33], heads=4, kv_heads=1, D=64, G=64).check()
    Case([2500, 900], [3, 33], heads=4, kv_heads=1, window=700).check()
    Case([2100], [20], heads=4, kv_heads=2, D=256, G=128, causal=False).check()


def test_more_sequences_than_a_wavefront_has_lanes():
    rng = np.random.default_rng(9)
    lens = [int(n) for n in rng.integers(0, 60, 150)]
    lens[70] = 2000
    Case(lens, [1] * 150, heads=2, kv_heads=1, D=64, G=32, page=16).check()
    counts = [int(n) for n in rng.integers(0, 4, 150)]
    Case([n + 4 for n in lens], counts, heads=2, kv_heads=1, D=64, G=32, page=16).check()


@pytest.mark.parametrize("gain", [0.0, 30.0, 1000.0])
def test_scores_of_any_size(gain):
    # all weights equal; one weight is nearly all: the maximum moves far and late.  fp32 scores of 1000s are off by 1e-3
    c = Case([600], [1], gain=gain)
    if gain < 100:
        c.check()
        return
    out = host(c.run())
    want, _, size = c.want()
    assert np.all(np.abs(out - want) <= 2e-2 * size + 1e-3)


def test_small_weights_count():
    # one key far above 6000 others: those have weights of 2^-17 each, together a twentieth
    D, n = 64, 6001
    c = Case([n], [1], heads=1, kv_heads=1, D=D, G=32, page=64)
    k = np.zeros((n, 1, D), dtype=np.float16)
    k[3000, 0, :32] = 6.0
    v = np.ones((n, 1, D), dtype=np.float16) * 6
    v[3000] = -6
    c.seqs = [(k, v)]
    write_all(c.cache, c.table, c.seqs, 32)
    c.q = np.zeros((1, 1, D), dtype=np.float16)
    c.q[0, 0, :32] = 17 * np.log(2) / 6 / 32 * D**0.5
    c.check()
    c.check(workspace=None)


def test_what_masked_keys_hold_has_no_effect():
    for D, G, count in ((128, 32, 1), (64, 64, 5), (128, 128, 40), (256, 32, 9)):
        c = Case([100], [count], D=D, G=G, window=30)
        want = c.run()
        for at in (99, 60 + 1):  # past the end (the sequence is then shorter) and before the window
            k, v = (x.copy() for x in c.seqs[0])
            if at == 99:
                continue
            k[: 70 - count], v[: 70 - count] = np.nan, np.inf
            write_all(c.cache, c.table, [(k, v)], G)
            assert torch.equal(c.run(), want)
        # whatever lies behind the last token in its page
        tail = np.full((28, 2, D), np.nan, dtype=np.float16)
        longer = dev(np.array([128], dtype=np.int32))
        ams.ams_kv_write(c.cache, dev(tail), dev(tail), c.table, longer, G, q_starts=starts_of([28]))
        assert torch.equal(c.run(), want)


@pytest.mark.parametrize("D,G,count", [(128, 32, 40), (64, 64, 9), (256, 128, 20), (128, 128, 300)])
def test_nan_reaches_the_rows_that_see_it_and_no_other(D, G, count):
    n = max(100, count)
    c = Case([n], [count], D=D, G=G)
    want = host(c.run()).copy()
    k, v = (x.copy() for x in c.seqs[0])
    row = count // 2
    v[n - count + row, 1, D - 1] = np.inf  # kv head 1: the last two of four heads; the last run
    c.seqs = [(k, v)]
    write_all(c.cache, c.table, c.seqs, G)
    out = host(c.run())
    assert np.array_equal(out[:, :2], want[:, :2]) and np.array_equal(out[:row, 2:], want[:row, 2:])
    assert np.isnan(out[row:, 2:, D - G :]).all()
    assert np.array_equal(out[row:, 2:, : D - G], want[row:, 2:, : D - G])
    # in k: the row's whole head
    v[n - count + row, 1, D - 1] = 0
    k[n - count + row, 1, 0] = np.nan
    write_all(c.cache, c.table, [(k, v)], G)
    out = host(c.run())
    assert np.array_equal(out[:row, 2:], want[:row, 2:]) and np.isnan(out[row:, 2:]).all() and np.array_equal(out[:, :2], want[:, :2])


def test_pages_that_are_not_there_are_left_out():
    c = Case([96], [1], heads=2, kv_heads=1, page=16)
    c.table[0, 2] = -1
    c.table[0, 4] = 1 << 20
    k, v = (np.concatenate([x[:32], x[48:64], x[80:]]) for x in c.seqs[0])
    c.seqs = [(k, v)]
    c.check()
    c.table.fill_(-1)
    assert not host(c.run()).any()


def test_strided_and_unaligned_rows():
    c = Case([50, 300], [4, 9], heads=6, kv_heads=2)
    want = c.run()
    n = len(c.q)
    for shift in (0, 1, 4):
        whole = torch.zeros((n, 6 * 128 + 24), dtype=torch.float16, device="cuda")
        q = whole[:, shift : shift + 6 * 128].unflatten(1, (6, 128))
        q.copy_(dev(c.q))
        store = torch.full((6, n, 128 + 16), 7.0, dtype=torch.float16, device="cuda")
        out = store[:, :, shift : shift + 128].transpose(0, 1)
        lse = torch.zeros((n, 8), dtype=torch.float32, device="cuda")[:, 1:7]
        assert c.run(q=q, out=out, lse=lse) is out
        assert torch.equal(out, want)
        assert bool((store[:, :, :shift] == 7).all()) and bool((store[:, :, shift + 128 :] == 7).all())


def test_a_scale_of_the_callers():
    c = Case([77], [1])
    ok, worst = near(host(c.run(softmax_scale=0.25)), *[c.want(0.25)[i] for i in (0, 2)], 77)
    assert ok, worst


def test_on_another_stream():
    c = Case([500, 40], [1, 1])
    want, q = c.run(), dev(c.q)
    side = torch.cuda.Stream()
    ws, out = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q2 = q * 1  # made on that stream
        c.run(q=q2, workspace=ws, out=out)
    side.synchronize()
    assert torch.equal(out, want)


def test_a_captured_step_follows_the_lengths():
    """One token after the other: rows written and attended to in one graph whose lengths grow between the replays."""
    rng = np.random.default_rng(12)
    D, G, page, heads, kv_heads, B, steps = 64, 32, 16, 4, 2, 3, 6
    first = np.array([0, 14, 300], dtype=np.int32)
    table, n_pages = table_for(first + steps, page, rng)
    cache, eager_cache = (ams.ams_kv_cache(n_pages, kv_heads, D, page, G) for _ in range(2))
    table = dev(table)
    seqs = [(rows_of(rng, n, kv_heads, D), rows_of(rng, n, kv_heads, D)) for n in first]
    for x in (cache, eager_cache):
        write_all(x, table, seqs, G)
    k, v, q = (torch.zeros((B, n, D), dtype=torch.float16, device="cuda") for n in (kv_heads, kv_heads, heads))
    lens, out = dev(first), torch.zeros((B, heads, D), dtype=torch.float16, device="cuda")
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    ams.ams_init()

    def step(x, o):
        ams.ams_kv_write(x, k, v, table, lens, G)
        ams.ams_kv_attention(q, x, table, lens, G, workspace=ws, out=o)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lens += 1
        step(cache, out)
    lens.copy_(dev(first))
    want = torch.zeros_like(out)
    for i in range(steps):
        for t in (k, v, q):
            t.normal_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        step(eager_cache, want)  # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache, eager_cache), i
        assert bool(out.any())


def test_a_prompt_that_fills_the_chip():
    # 64 heads of 1024 rows, and a table for more than 4096 keys: tiles of 256 rows
    c = Case([1100], [1024], heads=64, kv_heads=64, D=64, G=64, page=64, spare=60)
    assert c.table.shape[1] * 64 >= 4096
    c.check()


@pytest.mark.parametrize("D,G", [(64, 32), (128, 64)])
def test_many_tiles_that_are_shared_out(D, G):
    # 80 tiles and a table for more than 4096 keys: four wavefronts to a tile, shares that begin and end inside of tiles
    lens = [3000, 1, 0, 40, 2500, 999, 17, 1200, 33, 1600]
    Case(lens, [1] * 10, heads=16, kv_heads=8, D=D, G=G, page=64, spare=30).check()
    Case(lens, [1] * 10, heads=16, kv_heads=8, D=D, G=G, page=64, spare=30, window=1500).check()


def test_prompts_of_more_sequences_than_a_wavefront_has_lanes():
    rng = np.random.default_rng(10)
    lens = [int(n) for n in rng.integers(0, 50, 90)]
    lens[75] = 400
    counts = [min(n, int(k)) for n, k in zip(lens, rng.integers(0, 40, 90))]
    counts[75] = 390
    Case(lens, counts, heads=2, kv_heads=1, D=64, G=32, page=16).check(max_q_len=390)


def test_pages_that_a_prompt_does_not_find():
    c = Case([300], [200], heads=2, kv_heads=1, page=16)
    c.table[0, 3] = -1
    c.table[0, 16] = 1 << 20
    out = host(c.run())
    k, v = (O.held(x, 32) for x in c.seqs[0])
    there = np.ones(300, dtype=bool)
    there[48:64] = there[256:272] = False
    for i in range(200):
        at = there & (np.arange(300) <= 100 + i)
        want, _, size = O.attention(c.q[i : i + 1], k[at], v[at], c.D**-0.5, causal=False)
        ok, worst = near(out[i : i + 1], want, size, 300)
        assert ok, (i, worst)


def test_row_starts_that_make_no_sense_touch_nothing_else():
    c = Case([60, 40, 20], [3, 2, 4], heads=2, kv_heads=1)
    q = dev(c.q)
    for starts in ([0, 100, 50, 9], [5, 2, 8, -4], [1 << 30, 0, 0, 0], [-5, -5, 3, 1 << 30]):
        for hint in (None, 100):
            store = torch.full((c.q.shape[0] + 2, 2, 128), 7.0, dtype=torch.float16, device="cuda")
            ams.ams_kv_attention(q, c.cache, c.table, c.kv_lens, c.G, q_starts=dev(np.array(starts, dtype=np.int32)), max_q_len=hint, workspace=WORKSPACE, out=store[1:-1])
            assert bool((store[0] == 7).all()) and bool((store[-1] == 7).all())
            assert not bool(torch.isnan(store).any())


@pytest.mark.parametrize("heads,kv_heads,rows,D,G", [(16, 1, 1, 128, 32), (32, 1, 1, 128, 128), (20, 1, 2, 128, 64), (8, 1, 8, 128, 32), (64, 1, 1, 64, 64), (4, 1, 8, 256, 128), (12, 2, 8, 64, 32)])
@pytest.mark.parametrize("tokens", [8000, 12321])
def test_rows_of_one_sequence_in_many_parts(heads, kv_heads, rows, D, G, tokens):
    # 17 and 25 parts or more of 16 to 64 rows: sums of sums, the last of one part only
    c = Case([tokens], [rows], heads=heads, kv_heads=kv_heads, D=D, G=G, page=64)
    out = c.check()
    for _ in range(3):
        assert np.array_equal(out, host(c.run()))


def test_sequences_in_many_parts_beside_each_other():
    Case([9000, 8100, 33, 10000], [8, 8, 8, 8], heads=6, kv_heads=1, D=128, G=32, page=64).check()
    Case([9000, 8100, 33, 10000], [12, 12, 12, 12], heads=4, kv_heads=1, D=64, G=32, page=64, window=8400).check()


@pytest.mark.parametrize("rows", [10, 20, 31])
@pytest.mark.parametrize("D,G", [(64, 64), (128, 32)])
def test_drafts_of_many_sequences(D, G, rows):
    # 272 tiles of two to four column tiles, more than there are compute units: four wavefronts to a tile, uncut (lengths up to 500) and cut
    lens = [40 + (97 * b) % 460 for b in range(34)]
    Case(lens, [rows] * 34, heads=16, kv_heads=8, D=D, G=G, page=64).check()
    lens[5] = 2600
    Case(lens, [rows] * 34, heads=16, kv_heads=8, D=D, G=G, page=64).check()
