"""Writing rows into the 4-bit KV cache and reading them back, bit for bit against the definition: every size, lengths and starts
that fall anywhere in a tile, strided and unaligned rows, values at which rounding can go wrong, places that do not exist."""

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIZES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)]


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16)).cuda().view(torch.float16) if a.dtype == np.float16 else torch.from_numpy(a).cuda()


def host(t):
    return t.cpu().view(torch.int16).numpy().view(np.float16)


def bits(a):
    a = np.asarray(a, dtype=np.float16)
    return np.where(np.isnan(a), np.uint16(0x7E00), a.view(np.uint16))


def table_for(lens, page, rng, spare=1):
    """A block table with the pages of all sequences in no order, -1 where there is none, and the number of pages of the pool."""
    used = [-(-int(n) // page) for n in lens]
    order = rng.permutation(sum(used) + 2).astype(np.int32)
    table = np.full((len(lens), max(used, default=0) + spare), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at : at + n]
        at += n
    return table, sum(used) + 2


def starts_of(counts):
    return dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))


def rows_of(rng, n, heads, D):
    x = rng.standard_normal((n, heads, D)) * np.exp2(rng.integers(-3, 4, (n, heads, 1)))
    return x.astype(np.float16)


def write_all(cache, table, seqs, G):
    """Whole sequences [(k, v)] into the cache in one call."""
    lens = [len(k) for k, _ in seqs]
    k, v = (np.concatenate([s[i] for s in seqs]) for i in range(2))
    return ams.ams_kv_write(cache, dev(k), dev(v), table, dev(np.array(lens, dtype=np.int32)), G, q_starts=starts_of(lens))


@pytest.mark.parametrize("D,G", SIZES)
@pytest.mark.parametrize("page", [16, 48, 64])
def test_whole_sequences_come_back(D, G, page):
    rng = np.random.default_rng(D + G + page)
    lens, heads = [1, 0, 15, 16, 17, 2 * page + 5, 64, 33], 3
    table, n_pages = table_for(lens, page, rng)
    seqs = [(rows_of(rng, n, heads, D), rows_of(rng, n, heads, D)) for n in lens]
    cache = ams.ams_kv_cache(n_pages, heads, D, page, G)
    table = dev(table)
    write_all(cache, table, seqs, G)
    k, v = ams.ams_kv_read(cache, table, dev(np.array(lens, dtype=np.int32)), G, D, q_starts=starts_of(lens), rows=sum(lens))
    for got, i in ((k, 0), (v, 1)):
        want = O.held(np.concatenate([s[i] for s in seqs]), G)
        assert np.array_equal(bits(host(got)), bits(want))


@pytest.mark.parametrize("D,G", [(64, 32), (128, 128), (256, 64)])
def test_rows_written_in_pieces_leave_the_others_alone(D, G):
    rng = np.random.default_rng(7 * D + G)
    page, heads, n = 32, 2, 150
    table, n_pages = table_for([n, n], page, rng)
    table = dev(table)
    cache = ams.ams_kv_cache(n_pages, heads, D, page, G)
    k, v = rows_of(rng, 2 * n, heads, D).reshape(2, n, heads, D), rows_of(rng, 2 * n, heads, D).reshape(2, n, heads, D)
    at = 0
    for count in (1, 1, 2, 3, 16, 17, 5, 32, 31, 1, 40, 1):  # both sequences, some rows at a time, from every place in a tile
        at += count
        lens = dev(np.array([at, at], dtype=np.int32))
        new = [dev(x[:, at - count : at].reshape(-1, heads, D)) for x in (k, v)]
        ams.ams_kv_write(cache, *new, table, lens, G, q_starts=None if count == 1 else starts_of([count, count]))
        for back in (1, min(at, 20), at):  # the new ones, and what was there
            got = ams.ams_kv_read(cache, table, lens, G, D, q_starts=starts_of([back, back]), rows=2 * back)
            for x, y in zip(got, (k, v)):
                assert np.array_equal(bits(host(x)), bits(O.held(y[:, at - back : at], G)).reshape(2 * back, heads, D)), (at, back)


def hard_values(D, G, rng):
    """Rows at which rounding, scales or signs can go wrong."""
    half = lambda b: np.array(b, dtype=np.uint16).view(np.float16)
    rows = [np.zeros(D), np.full(D, -0.0), np.full(D, 65504.0), np.where(np.arange(D) % 2 == 0, 65504.0, -65504.0)]
    # every tie of a run whose scale is s, both signs
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, 6.0])
    for s in (1.0, 1.0009765625, 0.333251953125, 2.0**-14, 2.0**-24, 3 * 2.0**-24, 100.0):
        row = np.resize(np.concatenate([ties, -ties]) * s, D)
        row[::G] = 6.0 * s
        rows.append(row)
    rows.append(half(rng.integers(0, 0x7C00, D)).astype(np.float64))  # any finite magnitude
    rows.append(half(rng.integers(1, 40, D)).astype(np.float64))  # the smallest subnormals: scales of a few steps
    for n in range(1, 20):
        rows.append(np.full(D, n * 2.0**-24))
    for bad in (np.inf, -np.inf, np.nan):
        row = rng.standard_normal(D)
        row[D // 2] = bad
        rows.append(row)
    return np.stack(rows).astype(np.float16)


@pytest.mark.parametrize("D,G", SIZES)
def test_hard_values(D, G):
    rng = np.random.default_rng(D * G)
    k = hard_values(D, G, rng)[:, None, :]
    v = -k[::-1]
    n = len(k)
    table, n_pages = table_for([n], 16, rng)
    table, lens = dev(table), dev(np.array([n], dtype=np.int32))
    cache = ams.ams_kv_cache(n_pages, 1, D, 16, G)
    ams.ams_kv_write(cache, dev(k), dev(v), table, lens, G, q_starts=starts_of([n]))
    got = ams.ams_kv_read(cache, table, lens, G, D, q_starts=starts_of([n]), rows=n)
    for x, y in zip(got, (k, v)):
        assert np.array_equal(bits(host(x)), bits(O.held(y, G)))


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strided_and_unaligned_rows(shift):
    rng = np.random.default_rng(shift)
    D, G, page, heads, n = 128, 32, 16, 3, 37
    table, n_pages = table_for([n], page, rng)
    table, lens = dev(table), dev(np.array([n], dtype=np.int32))
    whole = torch.from_numpy(rng.standard_normal((n, 2 * heads * D + 24 + shift)).astype(np.float32)).cuda().half()
    k, v = whole[:, shift : shift + heads * D].view(n, heads, D), whole[:, shift + heads * D + 8 : shift + 2 * heads * D + 8].unflatten(1, (heads, D)).flip(1)
    cache = ams.ams_kv_cache(n_pages, heads, D, page, G)
    ams.ams_kv_write(cache, k, v, table, lens, G, q_starts=starts_of([n]))
    back = torch.full((n, 2 * heads, D + 8), 7.0, dtype=torch.float16, device="cuda").view(-1)[shift:]
    back = [torch.as_strided(back, (n - 1, heads, D), (2 * heads * (D + 8), 2 * (D + 8), 1), i * (D + 8)) for i in range(2)]
    ams.ams_kv_read(cache, table, lens, G, D, q_starts=starts_of([n - 1]), out=tuple(back))
    for x, y in zip(back, (k, v)):
        assert np.array_equal(bits(host(x.contiguous())), bits(O.held(host(y.contiguous()), G)[1:]))
    for x in back:  # nothing beside the rows
        base = x.as_strided((n - 1, 2 * heads, 8), (2 * heads * (D + 8), D + 8, 1), x.storage_offset() + D)
        assert bool((base[:, ::2] == 7.0).all())


def test_places_that_do_not_exist():
    rng = np.random.default_rng(3)
    D, G, page, heads = 64, 32, 16, 2
    cache = ams.ams_kv_cache(4, heads, D, page, G)
    before = cache.clone()
    k, v = dev(rows_of(rng, 12, heads, D)), dev(rows_of(rng, 12, heads, D))
    starts = starts_of([4, 4, 4])
    table = dev(np.array([[-1, 4], [1 << 30, -5], [0, 1]], dtype=np.int32))
    # no page of the pool; no page of the pool; a length beyond the table is the table's (rows at its end), then rows before the beginning
    ams.ams_kv_write(cache, k[:8], v[:8], table[:2], dev(np.array([20, 4], dtype=np.int32)), G, q_starts=starts_of([4, 4]))
    assert torch.equal(cache, before)
    lens = dev(np.array([20, 4, 1000], dtype=np.int32))
    ams.ams_kv_write(cache, k, v, table, lens, G, q_starts=starts)
    x, y = ams.ams_kv_read(cache, table, lens, G, D, q_starts=starts, rows=12)
    assert not bool(x[:8].any()) and not bool(y[:8].any())
    assert np.array_equal(bits(host(x[8:])), bits(O.held(host(k[8:]), G)))
    assert torch.equal(x[8:], ams.ams_kv_read(cache, table, dev(np.array([0, 0, 32], dtype=np.int32)), G, D, q_starts=starts, rows=12)[0][8:])
    # rows with a negative position: two of four, then all
    for length in (2, 0, -3):
        cache.zero_()
        lens = dev(np.array([0, 0, length], dtype=np.int32))
        ams.ams_kv_write(cache, k, v, table, lens, G, q_starts=starts)
        x, y = ams.ams_kv_read(cache, table, lens, G, D, q_starts=starts, rows=12)
        kept = max(length, 0)
        assert not bool(x[: 12 - kept].any()) and not bool(y[: 12 - kept].any())
        assert np.array_equal(bits(host(y[12 - kept :])), bits(O.held(host(v[12 - kept :]), G)))
        assert kept or not bool(cache.any())


def test_rows_that_no_sequence_has_are_left_alone():
    rng = np.random.default_rng(4)
    cache = ams.ams_kv_cache(3, 1, 64, 16, 32)
    table, lens = dev(np.array([[0], [1]], dtype=np.int32)), dev(np.array([3, 2], dtype=np.int32))
    k = dev(rows_of(rng, 9, 1, 64))
    starts = dev(np.array([2, 5, 7], dtype=np.int32))
    ams.ams_kv_write(cache, k, k, table, lens, 32, q_starts=starts)
    out = tuple(torch.full_like(k, 5.0) for _ in range(2))
    ams.ams_kv_read(cache, table, lens, 32, 64, q_starts=starts, out=out)
    assert np.array_equal(bits(host(out[0][2:7])), bits(O.held(host(k[2:7]), 32)))
    assert bool((out[0][:2] == 5).all()) and bool((out[1][7:] == 5).all())


def test_many_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, 700)
    table, n_pages = table_for(lens, 16, rng)
    seqs = [(rows_of(rng, n, 1, 64), rows_of(rng, n, 1, 64)) for n in lens]
    cache = ams.ams_kv_cache(n_pages, 1, 64, 16, 64)
    table = dev(table)
    write_all(cache, table, seqs, 64)
    k, v = ams.ams_kv_read(cache, table, dev(lens.astype(np.int32)), 64, 64, q_starts=starts_of(lens), rows=int(lens.sum()))
    assert np.array_equal(bits(host(k)), bits(O.held(np.concatenate([s[0] for s in seqs]), 64)))
    assert np.array_equal(bits(host(v)), bits(O.held(np.concatenate([s[1] for s in seqs]), 64)))


def test_a_pool_beyond_32_bits():
    rng = np.random.default_rng(6)
    D, G, page, heads = 256, 32, 1024, 8
    n_pages = (5 << 30) // (heads * ams.ams_kv_block_bytes(D, page, G)) + 1
    cache = torch.empty((n_pages, heads, ams.ams_kv_block_bytes(D, page, G)), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    table, lens = dev(np.array([[n_pages - 1, 0]], dtype=np.int32)), dev(np.array([1030], dtype=np.int32))
    k, v = rows_of(rng, 40, heads, D), rows_of(rng, 40, heads, D)
    ams.ams_kv_write(cache, dev(k), dev(v), table, lens, G, q_starts=starts_of([40]))
    x, y = ams.ams_kv_read(cache, table, lens, G, D, q_starts=starts_of([40]), rows=40)
    assert np.array_equal(bits(host(x)), bits(O.held(k, G))) and np.array_equal(bits(host(y)), bits(O.held(v, G)))


def test_nothing_to_do():
    cache = ams.ams_kv_cache(1, 1, 64, 16, 32)
    none = torch.empty((0, 1, 64), dtype=torch.float16, device="cuda")
    table, lens = torch.zeros((0, 1), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    ams.ams_kv_write(cache, none, none, table, lens, 32)
    assert ams.ams_kv_read(cache, table, lens, 32, 64)[0].shape == (0, 1, 64)
    assert not bool(cache.any())
