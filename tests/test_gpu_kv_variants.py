"""Every variant of the attention kernels by the plan that a call gets: each size of head and run, each number of column tiles and wavefronts,
with whole tiles, with parts of one tile each and with equal shares that cross tiles; prompts in tiles of 128 and 256 rows; rows whose keys fill
more than one look-up of pages."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O
from tests.test_gpu_kv_attention import Case, counts_are_zero, near, workspace  # noqa: F401  (the fixtures of that file)
from tests.test_gpu_kv_cache import SIZES, dev, host, starts_of, table_for

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
STEP, UNCUT = 32, 32  # keys of a step; steps of a tile that is not cut


def plan_of(c, workspace_bytes=ams.KV_WORKSPACE_BYTES):
    most = max(c.counts)
    text = ams.ams_kv_attention_plan(dev(c.q), c.cache, c.table, c.kv_lens, c.G, q_starts=c.starts, max_q_len=most, window=c.window, workspace_bytes=workspace_bytes)
    kernel, *pairs = text.split()
    return dict(kernel=kernel, **{name: int(value) for name, value in (x.split("=") for x in pairs)})


def split_of(c, plan, kv_heads):
    """How the kernel shares out what the plan allows it to, from the lengths."""
    tiles = [-(-n * (c.heads // kv_heads) // plan["rows"]) for n in c.counts]
    longest = max(-(-t // STEP) for t, n in zip(c.lens, tiles) if n)
    if not plan["shared"] or longest <= UNCUT:
        return "whole"
    return "parts" if 1 < sum(tiles) <= plan["workgroups"] // kv_heads // 2 else "across"


def check_some_heads(c, heads, **more):
    """Where all would take the oracle long."""
    lse = torch.zeros((len(c.q), c.heads), dtype=torch.float32, device="cuda")
    out, lse = host(c.run(lse=lse, **more)), lse.cpu().numpy().astype(np.float64)
    at = 0
    for (k, v), n in zip(c.seqs, c.counts):
        if n == 0:
            continue
        rows = slice(at, at + n)
        want, want_lse, size = O.attention(c.q[rows][:, heads], O.held(k[:, heads], c.G), O.held(v[:, heads], c.G), c.D**-0.5, c.causal, c.window)
        ok, worst = near(out[rows][:, heads], want, size, len(k))
        assert ok, worst
        assert np.all(np.abs(lse[rows][:, heads] - want_lse) <= 1e-5 * (1 + np.abs(want_lse)))
        at += n


def lengths(n, long, count):
    return [long if b == n // 2 else count + (37 * b + 5) % 90 for b in range(n)]


def variants():
    for D, G in SIZES:
        for columns in (1, 2) if D == 256 else (1, 2, 3, 4):
            for waves in (4, 8) if D == 128 or (D == 64 and columns == 1) else (4,):
                for split in ("whole", "parts", "across"):
                    yield D, G, columns, waves, split


@pytest.mark.parametrize("D,G,columns,waves,split", variants())
def test_few_rows(D, G, columns, waves, split):
    # kv heads, sequences with rows, and without: what makes the plan choose so many wavefronts, and the lengths the split
    if waves == 8:
        kv_heads, batch, idle = {"whole": (8, 7, 0), "parts": (8, 7, 0), "across": (32, 7, 0)}[split]
    else:
        kv_heads, batch, idle = {"whole": (64, 7, 0), "parts": (64, 4, 3), "across": (64, 7, 0)}[split]
    count = 1 if columns == 1 else 16 * columns - 3
    lens = lengths(batch + idle, 1000 if split == "whole" else 1100, count)
    counts = [count if b < batch else 0 for b in range(batch + idle)]
    if split == "parts" and idle:
        lens[1], lens[(batch + idle) // 2] = 1100, 70
    c = Case(lens, counts, heads=kv_heads, kv_heads=kv_heads, D=D, G=G, page=64)
    plan = plan_of(c)
    assert (plan["kernel"], plan["rows"], plan["waves"]) == ("stream", 16 * columns, waves), plan
    assert split_of(c, plan, kv_heads) == split, plan
    ws = torch.zeros(ams.KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    check_some_heads(c, [0, 1, kv_heads - 2, kv_heads - 1], max_q_len=count, workspace=ws)
    assert not bool(ws[:65536].any())


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("D,G,waves", [(D, G, waves) for D, G in SIZES for waves in ((4,) if D == 256 else (4, 8))])
def test_prompts(D, G, waves, window):
    # tiles of 256 rows where the table has room for 4096 keys and 512 tiles of 128 fill the chip twice
    c = Case([260, 95], [200, 70], heads=256, kv_heads=256, D=D, G=G, page=64, window=window, spare=60 if waves == 8 else 1)
    plan = plan_of(c)
    # a window of fewer than 4096 keys has tiles of 128 rows
    assert (plan["kernel"], plan["waves"]) == ("tile", 4 if window else waves) and plan["rows"] == 32 * plan["waves"], plan
    check_some_heads(c, [0, 1, 100, 255], max_q_len=200)


@pytest.mark.parametrize("D,G,kv_heads,rows,waves", [(64, 32, 64, 900, 4), (64, 64, 64, 1024, 8), (128, 128, 64, 900, 4), (128, 32, 64, 1024, 8), (256, 64, 32, 1800, 4)])
@pytest.mark.parametrize("window", [0, 4150])
def test_prompts_over_more_keys_than_one_look_up(D, G, kv_heads, rows, waves, window):
    c = Case([4300], [rows], heads=kv_heads, kv_heads=kv_heads, D=D, G=G, page=16, window=window)
    plan = plan_of(c)
    assert (plan["kernel"], plan["waves"]) == ("tile", waves), plan
    check_some_heads(c, [1, kv_heads - 1], max_q_len=rows)


@pytest.mark.parametrize("D,G,rows,tokens,waves", [(64, 32, 1, 20011, 8), (128, 64, 3, 18000, 8), (128, 128, 17, 17500, 8), (256, 32, 1, 9001, 4), (256, 128, 20, 8700, 4), (64, 64, 40, 8800, 4)])
@pytest.mark.parametrize("window", [0, 16600])
def test_rows_over_more_keys_than_one_look_up(D, G, rows, tokens, waves, window):
    # no workspace: one workgroup walks all keys, more than 64 steps to a wavefront
    c = Case([tokens], [rows], heads=1, kv_heads=1, D=D, G=G, page=16, window=window if window < tokens else 0)
    plan = plan_of(c, 0)
    assert (plan["kernel"], plan["waves"], plan["shared"]) == ("stream", waves, 0) and tokens > 64 * waves * STEP, plan
    c.check(workspace=None, max_q_len=rows)


def test_a_hint_less_call_of_drafts():
    # without max_q_len the plan has to reckon with all rows in one sequence
    lens = lengths(20, 1500, 5)
    c = Case(lens, [5] * 20, heads=16, kv_heads=8, D=128, G=32, page=64)
    known, unknown = plan_of(c), ams.ams_kv_attention_plan(dev(c.q), c.cache, c.table, c.kv_lens, 32, q_starts=c.starts)
    assert known["rows"] == 16 and "rows=64" in unknown
    c.check(max_q_len=5)
    c.check()


def test_the_plan_of_a_call_is_that_of_the_entry_point():
    table, _ = table_for([100], 64, np.random.default_rng(0))
    args = ams.ams_kv_cache(8, 2, 64, 64, 32), dev(table), dev(np.array([100], dtype=np.int32))
    q = torch.zeros((3, 4, 64), dtype=torch.float16, device="cuda")
    assert ams.ams_kv_attention_plan(q, *args, q_starts=starts_of([3])).startswith("stream rows=16 ")
    with pytest.raises(ams.AmsError):
        ams.ams_kv_attention_plan(q[:, :3], *args, q_starts=starts_of([3]))
    with pytest.raises(ams.AmsError):
        ams.ams_kv_attention_plan(q, *args, q_starts=starts_of([3]), window=-1)


@pytest.mark.parametrize("count", [1, 80])
def test_a_pool_beyond_32_bits(count):
    D, G, page, kv_heads, n = 128, 32, 1024, 8, 1100
    rng = np.random.default_rng(count)
    n_pages = (5 << 30) // (kv_heads * ams.ams_kv_block_bytes(D, page, G)) + 1
    cache = torch.empty((n_pages, kv_heads, ams.ams_kv_block_bytes(D, page, G)), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    k, v, q = (rng.standard_normal((m, h, D)).astype(np.float16) for m, h in ((n, kv_heads), (n, kv_heads), (count, 32)))
    where = dev(np.array([[n_pages - 1, n_pages // 2 + 1]], dtype=np.int32)), dev(np.array([n], dtype=np.int32))
    ams.ams_kv_write(cache, dev(k), dev(v), *where, G, q_starts=starts_of([n]))
    out = host(ams.ams_kv_attention(dev(q), cache, *where, G, q_starts=starts_of([count]), max_q_len=count, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")))
    want, _, size = O.attention(q, O.held(k, G), O.held(v, G), D**-0.5)
    ok, worst = near(out, want, size, n)
    assert ok, worst
