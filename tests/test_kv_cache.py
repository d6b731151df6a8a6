"""What the entry points of the 4-bit KV cache refuse, without a GPU: the C ABI's checks come before it looks at the device, the
binding's before it calls; and the sizes of a block."""

import ctypes

import numpy as np
import pytest

import paper_2510_16045_amd as ams
from oracle import kv_oracle as O

torch = pytest.importorskip("torch")

OK, SHAPE, NULL, ALIGN, DEVICE = 0, -2, -3, -4, -7
AT = 1 << 20  # an address that nothing reads: every call here is refused, or ends where no gfx950 is found or nothing is to be done


@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("page", [16, 48, 1024])
def test_block_bytes(D, G, page):
    assert ams.ams_kv_block_bytes(D, page, G) == page * 2 * (D // 2 + 2 * (D // G))
    assert ams.ams_kv_cache(3, 2, D, page, G, device="cpu").shape == (3, 2, ams.ams_kv_block_bytes(D, page, G))


@pytest.mark.parametrize("D,page,G", [(32, 16, 32), (96, 16, 32), (512, 16, 32), (128, 8, 32), (128, 40, 32), (128, 0, 32), (128, 1040, 32), (128, 16, 16), (128, 16, 256), (64, 16, 128), (128, 16, 0), (0, 16, 32)])
def test_sizes_that_there_are_no_kernels_for(D, page, G):
    with pytest.raises(ams.AmsError, match="shape"):
        ams.ams_kv_block_bytes(D, page, G)


def view(**but):
    fields = dict(pages=AT, block_table=AT, kv_lens=AT, q_starts=AT, n_pages=4, table_stride=3, table_width=3, batch=2, kv_heads=2, head_dim=128, page_size=16, scale_group=32)
    return ams._KvCache(**{**fields, **but})


def calls(c, rows=5, heads=4, k=AT, scale=1.0, causal=1, window=0, most=0, ws=AT, lse=None):
    lib = ams.load_library()
    c = ctypes.byref(c) if c is not None else None
    yield lib.ams_kv_write(c, k, AT, rows, 256, 128, 256, 128, None)
    yield lib.ams_kv_read(c, k, AT, rows, 256, 128, 256, 128, None)
    yield lib.ams_kv_attention(c, k, AT, lse, rows, heads, 512, 128, 512, 128, heads, scale, causal, window, most, ws, 1 << 20, None)


@pytest.mark.parametrize("but", [
    dict(head_dim=96), dict(page_size=24), dict(scale_group=48), dict(kv_heads=0), dict(kv_heads=1025), dict(n_pages=0), dict(n_pages=1 << 31), dict(batch=-1), dict(batch=65537), dict(table_width=0),
    dict(table_stride=-1), dict(table_width=1 << 28), dict(q_starts=None),
])
def test_caches_that_are_refused(but):
    assert set(calls(view(**but))) == {SHAPE}


def test_pointers_that_are_refused():
    assert set(calls(None)) == {NULL}
    for name in ("pages", "block_table", "kv_lens"):
        assert set(calls(view(**{name: None}))) == {NULL}
    assert set(calls(view(), k=None)) == {NULL}
    for name, off in (("pages", 8), ("block_table", 2), ("kv_lens", 1), ("q_starts", 2)):
        assert set(calls(view(**{name: AT + off}))) == {ALIGN}
    assert set(calls(view(), k=AT + 1)) == {ALIGN}
    assert list(calls(view(), ws=AT + 8))[2] == ALIGN and list(calls(view(), lse=AT + 2))[2] == ALIGN


def test_rows_and_arguments_that_are_refused():
    assert set(calls(view(), rows=-1)) == {SHAPE} and set(calls(view(), rows=(1 << 28) + 1)) == {SHAPE}
    for bad in (dict(heads=3), dict(heads=0), dict(heads=1026), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(causal=0, window=4), dict(most=-1),
                dict(rows=1 << 28)):
        assert list(calls(view(), **bad))[2] == SHAPE, bad


def test_no_other_gpu_and_no_cpu():
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    assert set(calls(view())) == {DEVICE}


def test_workspace_of_any_call_is_within_the_bound():
    lib, size = ams.load_library(), ctypes.c_size_t()
    for D, G in ((64, 32), (128, 32), (256, 128)):
        for kv_heads in (1, 3, 8, 40, 300, 1024):
            for group in (1, 2, 7, 16, 64):
                for rows, starts in ((2, None), (2, AT), (5, AT), (40, AT), (5000, AT)):
                    if kv_heads * group > 1024:
                        continue
                    for most in (0, 1, 7, 100000):
                        c = view(kv_heads=kv_heads, head_dim=D, scale_group=G, q_starts=starts, table_width=20000)
                        assert lib.ams_kv_attention_workspace_bytes(ctypes.byref(c), rows, kv_heads * group, most, ctypes.byref(size)) == OK
                        assert size.value <= ams.KV_WORKSPACE_BYTES
    assert lib.ams_kv_attention_workspace_bytes(ctypes.byref(view()), 5, 3, 0, ctypes.byref(size)) == SHAPE
    assert lib.ams_kv_attention_workspace_bytes(ctypes.byref(view()), 5, 4, 0, None) == NULL


def tensors():
    return dict(
        cache=ams.ams_kv_cache(4, 2, 128, 16, 32, device="cpu"), k=torch.zeros((3, 2, 128), dtype=torch.float16), v=torch.zeros((3, 2, 128), dtype=torch.float16),
        q=torch.zeros((3, 4, 128), dtype=torch.float16), block_table=torch.zeros((3, 2), dtype=torch.int32), kv_lens=torch.ones(3, dtype=torch.int32),
    )


def refused(error, match, **but):
    t = {**tensors(), **but}
    q, rest = t.pop("q"), {n: t[n] for n in ("block_table", "kv_lens", "q_starts") if n in t}
    for call in (
        lambda: ams.ams_kv_write(t["cache"], t["k"], t["v"], **rest),
        lambda: ams.ams_kv_read(t["cache"], **rest, out=(t["k"], t["v"])),
        lambda: ams.ams_kv_attention(q, t["cache"], **rest),
    ):
        with pytest.raises(error, match=match):
            call()


def test_what_the_binding_refuses():
    z = torch.zeros
    refused(ValueError, "CUDA")  # tensors of the host
    refused(ValueError, "expected cache", cache=z(4, dtype=torch.uint8))
    refused(ValueError, "expected cache", block_table=z(3, dtype=torch.int32))
    refused(ValueError, "sequences", kv_lens=z(2, dtype=torch.int32))
    refused(ValueError, "q_starts must", q_starts=z(3, dtype=torch.int32))
    refused(ValueError, "whole number", cache=z((4, 2, 1000), dtype=torch.uint8))
    refused(TypeError, "int32", block_table=z((3, 2), dtype=torch.int64))
    with pytest.raises(ValueError, match="rows or out"):
        ams.ams_kv_read(*(tensors()[n] for n in ("cache", "block_table", "kv_lens")), q_starts=z(4, dtype=torch.int32))


@pytest.mark.gpu
def test_what_the_binding_refuses_on_the_gpu():
    t = {n: x.cuda() for n, x in tensors().items()}
    z = lambda *s, **k: torch.zeros(*s, **{"dtype": torch.float16, "device": "cuda", **k})  # noqa: E731
    where = (t["block_table"], t["kv_lens"])
    for bad, error in (
        (z(3, 2, 64), ValueError), (z(3, 3, 128), ValueError), (z(2, 2, 128), ValueError), (z(3, 256), ValueError), (z(3, 2, 128, dtype=torch.float32), TypeError), (z(3, 2, 256)[:, :, ::2], ValueError),
        (z(3, 2, 128).cpu(), ValueError),
    ):
        with pytest.raises(error):
            ams.ams_kv_write(t["cache"], t["k"], bad, *where)
        with pytest.raises(error):
            ams.ams_kv_read(t["cache"], *where, out=(t["k"], bad))
    attention = lambda **k: ams.ams_kv_attention(**{**dict(q=t["q"], cache=t["cache"], block_table=t["block_table"], kv_lens=t["kv_lens"]), **k})  # noqa: E731
    for error, bad in (
        (ValueError, dict(q=z(3, 512))), (ValueError, dict(out=z(2, 4, 128))), (ValueError, dict(out=z(3, 4, 64))), (TypeError, dict(out=z(3, 4, 128, dtype=torch.bfloat16))), (ValueError, dict(lse=z(3, 2))),
        (TypeError, dict(lse=z(3, 4))), (TypeError, dict(workspace=z(64))), (ams.AmsError, dict(q=z(3, 3, 128))), (ams.AmsError, dict(softmax_scale=0.0)), (ams.AmsError, dict(window=3, causal=False)),
        (ams.AmsError, dict(scale_group=48)), (ValueError, dict(cache=t["cache"][:, :, ::2])), (TypeError, dict(kv_lens=t["kv_lens"].long())), (ValueError, dict(kv_lens=t["kv_lens"].cpu())),
        (ams.AmsError, dict(q=z(2, 4, 128))),
    ):
        with pytest.raises(error):
            attention(**bad)
    attention()
    torch.cuda.synchronize()


def test_the_oracle_rounds_as_the_definition_says():
    # scale 1: ties to the even code, saturation, signs; a run of zeros; a run that holds an inf
    x = np.array([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 0.2501, 0.7499] + [0] * 19, dtype=np.float16)  # the last two are ties once they are fp16
    y = O.held(x[None], 32)[0]
    assert list(y[:13]) == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -4, 0, 1]
    assert list(O.held(np.array([[6, 0.2505, 0.749] + [0] * 29], dtype=np.float16), 32)[0, :3]) == [6, 0.5, 0.5]
    assert np.signbit(y[8]) and not np.signbit(y[20])
    assert not O.held(np.zeros((1, 64), np.float16), 32).any()
    z = np.ones((1, 64), np.float16)
    z[0, 40] = np.inf
    assert np.isnan(O.held(z, 32)[0, 32:]).all() and np.isfinite(O.held(z, 32)[0, :32]).all()
    assert np.isfinite(O.held(np.full((1, 32), 65504, np.float16), 32)).all()
    # softmax over two keys, one masked for the first row
    k, v = np.zeros((2, 1, 32)), np.stack([np.ones((1, 32)), 3 * np.ones((1, 32))])
    out, lse, _ = O.attention(np.zeros((2, 1, 32), np.float16), k, v, 1.0)
    assert np.allclose(out[:, 0, 0], [1, 2]) and np.allclose(lse[:, 0], [0, np.log(2)])
