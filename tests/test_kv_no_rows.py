"""What the host says of an attention call without rows: nothing is used, nothing ends the process."""

import ctypes

import pytest

import paper_2510_16045_amd as ams
from tests.test_kv_cache import AT, OK, view
from tests.test_kv_plan import plan


@pytest.mark.parametrize("D,G", [(64, 32), (128, 128), (256, 64)])
@pytest.mark.parametrize("batch", [0, 1, 300])
@pytest.mark.parametrize("width", [1, 20000])
def test_no_rows(D, G, batch, width):
    c, size = view(q_starts=AT, batch=batch, head_dim=D, scale_group=G, table_width=width), ctypes.c_size_t(1)
    for most in (0, 1, 500):
        assert ams.load_library().ams_kv_attention_workspace_bytes(ctypes.byref(c), 0, 4, most, ctypes.byref(size)) == OK and size.value == 0
        for workspace in (0, 1 << 20, ams.KV_WORKSPACE_BYTES):
            assert plan(c, 0, 4, most=most, workspace=workspace)["shared"] == 0
