"""Attention where scores are as large as fp16 rows can make them: a finite row has a finite result, that of the keys whose score is
the largest.  Products of powers of two, so that fp32 holds every score exactly and nothing is in doubt."""

import numpy as np
import pytest

from oracle import kv_oracle as O
from tests.test_gpu_kv_attention import Case, near
from tests.test_gpu_kv_cache import host, write_all

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(c, rng, q_size, k_size, **more):
    """q is +-q_size in all channels, a key k_size, 3/4 or 1/2 of it: scores of a few values, each of them exact."""
    n = sum(c.counts)
    c.q = (q_size * rng.choice([-1.0, 1.0], (n, c.heads, 1)) * np.ones((1, 1, c.D))).astype(np.float16)
    seqs = []
    for k, v in c.seqs:
        k = k_size * rng.choice([1.0, 0.75, 0.5], (k.shape[0], k.shape[1], 1)) * np.ones((1, 1, c.D))
        seqs.append((k.astype(np.float16), v))
    c.seqs = seqs
    for k, _ in seqs:
        assert np.array_equal(O.held(k, c.G), k.astype(np.float64))
    write_all(c.cache, c.table, c.seqs, c.G)
    lse = torch.zeros((n, c.heads), dtype=torch.float32, device="cuda")
    ws = torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")
    out = host(c.run(workspace=ws, lse=lse, softmax_scale=1.0, **more))
    want, want_lse, size = c.want(1.0)
    assert np.isfinite(want).all()
    assert np.isfinite(out).all(), (int((~np.isfinite(out)).sum()), out.size)
    ok, worst = near(out, want, size, max(c.lens))
    assert ok, worst
    got = lse.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want_lse) <= 1e-5 * (1 + np.abs(want_lse)))


# scores of 2^20 and more: up to 2^37
@pytest.mark.parametrize("q_size,k_size", [(2.0**6, 2.0**8), (2.0**9, 2.0**9), (2.0**11, 2.0**11), (2.0**13, 2.0**11), (2.0**15, 2.0**14)])
@pytest.mark.parametrize("D,G", [(64, 64), (128, 32), (256, 128)])
def test_rows_of_any_number(D, G, q_size, k_size):
    rng = np.random.default_rng(D)
    check(Case([600, 40], [1, 1], D=D, G=G, page=64), rng, q_size, k_size)
    check(Case([600, 40], [7, 7], heads=8, D=D, G=G, page=64), rng, q_size, k_size, max_q_len=7)
    check(Case([2500], [3], heads=8, kv_heads=1, D=D, G=G, page=64), rng, q_size, k_size)
    check(Case([300], [200], D=D, G=G, page=64), rng, q_size, k_size)


@pytest.mark.parametrize("count", [1, 9, 150])
@pytest.mark.parametrize("D,G", [(64, 32), (128, 128), (256, 64)])
def test_rows_of_large_random_values(D, G, count):
    # scores of some 1e9, all of them far apart: the largest one has the weight
    c = Case([400], [count], heads=4, kv_heads=2, D=D, G=G, page=64, gain=10000.0)
    c.seqs = [(np.clip(k * np.float16(1000), -60000, 60000).astype(np.float16), v) for k, v in c.seqs]
    write_all(c.cache, c.table, c.seqs, G)
    assert np.isfinite(c.q).all()
    lse = torch.zeros((count, 4), dtype=torch.float32, device="cuda")
    out = host(c.run(workspace=None, lse=lse))
    want, want_lse, size = c.want()
    assert np.isfinite(out).all()
    assert np.all(np.abs(lse.cpu().numpy() - want_lse) <= 1e-5 * (1 + np.abs(want_lse)))
    # a row whose two largest scores are nearer than what fp32 sums of D such products may be off is left out
    q, k = c.q.astype(np.float64), O.held(c.seqs[0][0], G)
    for i in range(count):
        for h in range(4):
            s = np.sort(q[i, h] @ k[: 400 - count + i + 1, h // 2].T * D**-0.5)
            if len(s) < 2 or s[-1] - s[-2] > 2.0**-20 * D * np.abs(s).max():
                assert np.all(np.abs(out[i, h] - want[i, h]) <= (2.0**-10 + 4e-5) * (np.abs(want[i, h]) + size[i, h]) + 2.0**-24), (i, h)
