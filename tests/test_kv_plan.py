"""Which kernel and launch shape ams_kv_attention gives a call (host only): a workspace never leaves a call with much fewer workgroups than it
has without one, as far as they fit on the chip."""

import ctypes

import pytest

import paper_2510_16045_amd as ams
from tests.test_kv_cache import AT, NULL, OK, SHAPE, view


def plan(c, rows, heads, window=0, most=0, workspace=ams.KV_WORKSPACE_BYTES):
    text = ctypes.create_string_buffer(256)
    assert ams.load_library().ams_kv_attention_plan(ctypes.byref(c), rows, heads, window, most, workspace, text, len(text)) == OK
    kernel, *pairs = text.value.decode().split()
    return dict(kernel=kernel, **{name: int(value) for name, value in (x.split("=") for x in pairs)})


def test_what_is_refused():
    lib, text = ams.load_library(), ctypes.create_string_buffer(256)
    ask = lambda c, rows=5, heads=4, window=0, most=0, to=text, n=256: lib.ams_kv_attention_plan(ctypes.byref(c), rows, heads, window, most, 0, to, n)  # noqa: E731
    assert ask(view()) == OK and text.value.split()[0] in (b"stream", b"tile")
    assert ask(view(), n=4) == OK and len(text.value) == 3
    assert ask(view(), to=None) == ask(view(), n=0) == ask(view(pages=None)) == NULL
    assert ask(view(), heads=3) == ask(view(), window=-1) == ask(view(), most=-1) == ask(view(), rows=1 << 28) == ask(view(head_dim=96)) == SHAPE


@pytest.mark.parametrize("D,G", [(64, 32), (128, 32), (256, 64)])
@pytest.mark.parametrize("heads,kv_heads", [(32, 8), (64, 8), (28, 4), (16, 16), (12, 1)])
def test_a_workspace_takes_no_workgroups_away(D, G, heads, kv_heads):
    shared = set()
    for batch in (1, 2, 7, 32, 64, 300):
        for rows, starts in ((batch, None), (5 * batch, AT), (60 * batch, AT)):
            for width in (20, 100, 8192):
                c = view(batch=batch, kv_heads=kv_heads, head_dim=D, scale_group=G, q_starts=starts, table_width=width, page_size=16)
                ask = lambda size: plan(c, rows, heads, most=rows // batch, workspace=size)  # noqa: E731
                without, ample = ask(0), ask(ams.KV_WORKSPACE_BYTES)
                assert not without["shared"]
                for size in (16, 65536, 100000, 200000, 400000, 1 << 20, 3 << 20, 10 << 20, ams.KV_WORKSPACE_BYTES):
                    got = ask(size)
                    if got["shared"]:
                        assert 8 * got["workgroups"] >= 7 * min(without["workgroups"], ample["workgroups"]), (batch, rows, width, size, got, without)
                    else:
                        assert got == without
                    shared.add(got["shared"])
    assert shared == {0, 1}
