"""More rows than a sequence has tokens: with `causal` the ones before its first token see no key; without it every row sees every key."""

import numpy as np
import pytest

from oracle import kv_oracle as O
from tests.test_gpu_kv_attention import Case, counts_are_zero, near, workspace  # noqa: F401  (the fixtures of that file)
from tests.test_gpu_kv_cache import host

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,G", [(64, 32), (128, 64), (256, 128)])
@pytest.mark.parametrize("lens,counts", [([3, 0, 40], [5, 2, 50]), ([70, 1, 0, 130], [200, 90, 75, 150]), ([1200, 9], [1300, 1300])])
def test_more_rows_than_tokens(lens, counts, D, G, causal):
    # up to 64 rows, more than that, and more over keys that are shared out
    c = Case(lens, counts, heads=2, kv_heads=1, D=D, G=G, causal=causal, page=64)
    lse = torch.zeros((sum(counts), 2), dtype=torch.float32, device="cuda")
    out, lse = host(c.run(lse=lse, max_q_len=max(counts))), lse.cpu().numpy().astype(np.float64)
    at = 0
    for (k, v), n in zip(c.seqs, counts):
        want, want_lse, size = O.attention(c.q[at : at + n], O.held(k, G), O.held(v, G), D**-0.5, causal)
        unseen = n - len(k) if causal else n if len(k) == 0 else 0
        assert not out[at : at + unseen].any() and np.isneginf(lse[at : at + unseen]).all() and np.isfinite(want_lse[unseen:]).all()
        ok, worst = near(out[at : at + n], want, size, len(k))
        assert ok, worst
        assert np.all(np.abs(lse[at + unseen : at + n] - want_lse[unseen:]) <= 1e-5 * (1 + np.abs(want_lse[unseen:])))
        at += n
