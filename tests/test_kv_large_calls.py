"""Calls of the KV cache that would take more threads than one launch can have are refused, before anything is launched."""

import pytest

from tests.test_kv_cache import AT, DEVICE, SHAPE, calls, view

torch = pytest.importorskip("torch")


# (of the cache, rows, query heads): wavefronts of four to a workgroup; a workgroup of 256 threads for each sequence and kv head
TOO_LARGE = [(dict(q_starts=None, batch=65536, kv_heads=1024), 65536, 1024), (dict(q_starts=AT, batch=65536, kv_heads=512), 5, 512), (dict(q_starts=AT, batch=1, kv_heads=1024), 1 << 21, 1024), (dict(q_starts=AT, batch=60000, kv_heads=1000), 60000, 1000)]


@pytest.mark.parametrize("cache,rows,heads", TOO_LARGE)
def test_refused(cache, rows, heads):
    assert set(calls(view(**cache), rows=rows, heads=heads)) == {SHAPE}


def test_attention_takes_more_threads():
    """Where rows can be written and read, but not looked at in one launch."""
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    assert list(calls(view(q_starts=None, batch=65536, kv_heads=256), rows=65536, heads=256)) == [DEVICE, DEVICE, SHAPE]


def test_no_rows_are_nothing_to_do():
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    assert set(calls(view(q_starts=AT, batch=65536, kv_heads=1024), rows=0, heads=1024)) == {DEVICE}


def test_the_largest_that_are_not():
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    write, read, _ = calls(view(q_starts=None, batch=65535, kv_heads=1024), rows=65535, heads=1024)
    assert write == read == DEVICE
    assert set(calls(view(q_starts=None, batch=65536, kv_heads=255), rows=65536, heads=255)) == {DEVICE}
    assert set(calls(view(q_starts=AT, batch=1, kv_heads=1023), rows=1 << 20, heads=1023)) == {DEVICE}
