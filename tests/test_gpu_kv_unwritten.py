"""What the pool holds where no row was written has no effect on attention: the rest of a last tile, pages that other data used, keys
before a window.  Outputs over a pool full of something else equal those over an empty one bit for bit."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from tests.test_gpu_kv_attention import Case
from tests.test_gpu_kv_cache import SIZES, write_all

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# halves that fill the pool, scales and codes alike: the largest scale that is ever stored (10912) and the next one, whose 6-fold is no fp16
# value any more; further finite ones of both signs; the infinities and a NaN
HALVES = (0x7154, 0x7155, 0x71D0, 0x7BFF, 0xF155, 0xFBFF, 0x7C00, 0xFC00, 0x7E77)


def fill(cache, what):
    if what == "random":
        gen = torch.Generator(device="cuda").manual_seed(3)
        cache.copy_(torch.randint(0, 256, cache.shape, generator=gen, device="cuda", dtype=torch.uint8))
    elif what == "codes of 6":  # under the largest scale of all
        cache.fill_(0x77)
        D, page, G = fill.sizes
        scales = torch.full((cache.shape[0], cache.shape[1], 2 * page * (D // G)), 0x7BFF, dtype=torch.int16, device="cuda").view(torch.uint8)
        cache[:, :, page * D :] = scales
    else:
        cache.copy_(torch.full((cache.numel() // 2,), what - (what >> 15 << 16), dtype=torch.int16, device="cuda").view(torch.uint8).view(cache.shape))


def outputs(c, **more):
    lse = torch.zeros((len(c.q), c.heads), dtype=torch.float32, device="cuda")
    ws = torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")
    return c.run(workspace=ws, lse=lse, **more), lse


def same_whatever_the_pool_holds(c, page, spoil=None, **more):
    want = outputs(c, **more)
    assert bool(want[0].any()) and bool(torch.isfinite(want[0]).all())
    fill.sizes = c.D, page, c.G
    for what in (*HALVES, "random", "codes of 6"):
        fill(c.cache, what)
        if spoil is None:
            write_all(c.cache, c.table, c.seqs, c.G)
        else:
            spoil(c)
        for x, y in zip(outputs(c, **more), want):
            assert torch.equal(x, y), what if isinstance(what, str) else hex(what)


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("count", [1, 5, 11])
def test_single_rows_and_drafts(D, G, count):
    # lengths that end anywhere in a tile and in a step of two tiles
    lens = [12, 17, 31, 33, 47, 65, 100, 121]
    same_whatever_the_pool_holds(Case(lens, [count] * len(lens), heads=8, kv_heads=2, D=D, G=G, page=64), 64, max_q_len=count)


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 21)])
def test_prompts(D, G, causal, window):
    lens = [97, 90, 150, 33]
    same_whatever_the_pool_holds(Case(lens, lens, D=D, G=G, page=48, causal=causal, window=window), 48, max_q_len=150)


@pytest.mark.parametrize("D,G", [(64, 64), (128, 32), (256, 128)])
def test_long_rows_that_are_shared_out(D, G):
    same_whatever_the_pool_holds(Case([2500, 1111], [1, 1], heads=8, kv_heads=1, D=D, G=G, page=64), 64)
    same_whatever_the_pool_holds(Case([2499], [9], heads=4, kv_heads=2, D=D, G=G, page=64, window=700), 64)


@pytest.mark.parametrize("count", [1, 70])
@pytest.mark.parametrize("D,G", [(64, 32), (128, 128), (256, 64)])
def test_pages_before_the_window(D, G, count):
    # the first row sees keys from 85 (100) on: of its step's keys (its block's) the tile before belongs to no row any more
    c = Case([100 if count == 1 else 169], [count], D=D, G=G, page=16, window=15)

    def spoil(c):
        whole = c.cache.clone()
        write_all(c.cache, c.table, c.seqs, c.G)
        for page in range(5):
            at = int(c.table_host[0, page])
            c.cache[at] = whole[at]

    same_whatever_the_pool_holds(c, 16, spoil)


def test_a_pool_that_was_never_set():
    c = Case([37, 5], [1, 1], heads=2, kv_heads=1)
    want = c.run(workspace=None)
    c.cache = torch.empty_like(c.cache).copy_(torch.full_like(c.cache, 0xFF))
    ams.ams_kv_write(c.cache, *(torch.from_numpy(np.concatenate([s[i] for s in c.seqs]).view(np.int16)).cuda().view(torch.float16) for i in range(2)), c.table, c.kv_lens, c.G,
                     q_starts=torch.tensor([0, 37, 42], dtype=torch.int32, device="cuda"))
    assert torch.equal(c.run(workspace=None), want)
