"""Rows that row starts beyond the call's rows leave to a sequence: rotated by the positions at which the cache's calls take them."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from tests.test_gpu_kv_cache import dev
from tests.test_gpu_rope import check, rows, turns_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# (lengths, row starts, rows): row starts count as in [0, rows], so the last sequence's rows are those that there are
CASES = [([20], [0, 10], 6), ([20, 30], [0, 2, 2**31 - 1], 5), ([9, 20], [-4, 3, 100], 7), ([20], [-(2**31), 5], 5), ([50] * 70, list(range(0, 140, 2)) + [1000], 141)]


@pytest.mark.parametrize("lens,starts,n", CASES)
def test_starts_beyond_the_rows(lens, starts, n):
    D, G, page, pages = 64, 32, 16, 5
    q, k = rows(n, 2, D), rows(n, 1, D, 1)
    kv_lens, q_starts = dev(np.array(lens, dtype=np.int32)), dev(np.array(starts, dtype=np.int32))
    at = [min(max(s, 0), n) for s in starts]
    positions = [lens[b] - at[b + 1] + r for b in range(len(lens)) for r in range(at[b], at[b + 1])]
    assert len(positions) == n
    got, got_k = ams.ams_rope(q, k, turns_of(D), kv_lens=kv_lens, q_starts=q_starts)
    check(got, q, positions, D), check(got_k, k, positions, D)
    # where the cache puts them
    table = torch.arange(len(lens) * pages, dtype=torch.int32, device="cuda").view(-1, pages)
    a, b = (ams.ams_kv_cache(len(lens) * pages, 1, D, page, G).zero_() for _ in range(2))
    ams.ams_kv_write(a, k, k, table, kv_lens, G, q_starts=q_starts)
    ams.ams_kv_write(b, k, k, table, kv_lens, G, q_starts=dev(np.array(at, dtype=np.int32)))
    assert torch.equal(a, b) and bool(a.any())
