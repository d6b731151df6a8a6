"""Row starts that do not ascend and stand for far more rows than a call has: nothing is done for them, whatever kernel the call gets, and the
workspace is as good as before."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from tests.test_gpu_kv_attention import Case
from tests.test_gpu_kv_cache import dev

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("hint", [1, None])
def test_more_rows_than_there_are(shared, hint):
    # every other of 512 sequences has all 4096 rows: 2^20 tiles of 64 rows (4096 of them in truth) of 4096 steps, more than 2^32 in all
    heads, D, G, page, batch, rows = 64, 64, 32, 64, 512, 4096
    cache = ams.ams_kv_cache(2, 1, D, page, G)
    table = torch.zeros((batch, 131072 // page), dtype=torch.int32, device="cuda")
    lens = torch.full((batch,), 131072, dtype=torch.int32, device="cuda")
    starts = dev(np.array([0, rows] * (batch // 2) + [0], dtype=np.int32))
    q = torch.ones((rows, heads, D), dtype=torch.float16, device="cuda")
    out = torch.full_like(q, 7.0)
    ws = torch.zeros(ams.KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda") if shared else None
    plan = ams.ams_kv_attention_plan(q, cache, table, lens, G, q_starts=starts, max_q_len=hint, workspace_bytes=ams.KV_WORKSPACE_BYTES if shared else 0)
    assert plan.split()[0] == ("stream" if hint else "tile") and plan.endswith(f"shared={int(shared and hint == 1)}")
    ams.ams_kv_attention(q, cache, table, lens, G, q_starts=starts, max_q_len=hint, workspace=ws, out=out)
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    assert ws is None or not bool(ws[:65536].any())
    c = Case([3000, 5, 1111], [1, 1, 1], heads=8, kv_heads=1)
    assert torch.equal(c.run(workspace=ws), c.run(workspace=None if ws is None else torch.zeros_like(ws)))


def test_starts_outside_of_the_rows():
    # what lies outside of [0, rows] is taken as the nearer of the two
    c = Case([60, 40, 20], [3, 2, 4], heads=2, kv_heads=1)
    want = c.run(workspace=None)
    for starts in ([-3, 3, 5, 9], [0, 3, 5, 1 << 30], [-(1 << 31), 3, 5, 9]):
        assert torch.equal(ams.ams_kv_attention(dev(c.q), c.cache, c.table, c.kv_lens, c.G, q_starts=dev(np.array(starts, dtype=np.int32))), want)
