"""Log probabilities: what is refused before anything is launched."""

import ctypes
import math

import pytest

import paper_2510_16045_amd as ams

torch = pytest.importorskip("torch")

NULL, SHAPE, ALIGN = -3, -2, -4


def call(logits=0x1000, kind=0, rows=4, vocab=100, stride=100, tokens=0x1000, temperature=1.0, top=2, logprob=0x1000, rank=0x1000, entropy=0x1000, values=0x1000, indexes=0x1000, workspace=None, size=0):
    """ams_logprobs with addresses that are never used: what is refused is refused before anything is launched."""
    return ams.load_library().ams_logprobs(logits, kind, rows, vocab, stride, tokens, temperature, top, logprob, rank, entropy, values, indexes, workspace, size, None)


@pytest.mark.parametrize(
    "more,code",
    [
        (dict(kind=2), SHAPE), (dict(kind=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 28) + 1), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=(1 << 28) + 1), SHAPE), (dict(top=-1), SHAPE),
        (dict(top=65), SHAPE), (dict(temperature=0.0), SHAPE), (dict(temperature=-1.0), SHAPE), (dict(temperature=math.nan), SHAPE), (dict(temperature=math.inf), SHAPE), (dict(logits=None), NULL),
        (dict(tokens=None), NULL), (dict(tokens=None, logprob=None), NULL), (dict(values=None), NULL), (dict(indexes=None), NULL), (dict(logits=0x1001), ALIGN), (dict(kind=1, logits=0x1002), ALIGN),
        (dict(tokens=0x1002), ALIGN), (dict(logprob=0x1002), ALIGN), (dict(rank=0x1001), ALIGN), (dict(entropy=0x1002), ALIGN), (dict(values=0x1002), ALIGN), (dict(indexes=0x1002), ALIGN),
        (dict(workspace=0x1008, size=1 << 20), ALIGN),
    ],
)
def test_refused(more, code):
    assert call(**more) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")
def test_no_gpu():
    assert call() == -7


def test_workspace_bytes():
    lib, size = ams.load_library(), ctypes.c_size_t(1)
    assert lib.ams_logprobs_workspace_bytes(0, 4, 100, 2, None) == NULL
    assert lib.ams_logprobs_workspace_bytes(0, 4, 0, 2, ctypes.byref(size)) == SHAPE
    for rows in (0, 1, 7, 32, 300, 5000, 1 << 28):
        for kind in (0, 1):
            for top in (0, 1, 20, 64):
                assert lib.ams_logprobs_workspace_bytes(kind, rows, 128256, top, ctypes.byref(size)) == 0
                assert size.value <= ams.KV_WORKSPACE_BYTES
                if rows in (1, 7, 32):
                    assert size.value > 0
                if rows in (0, 5000, 1 << 28):
                    assert size.value == 0


def test_python_refusals():
    x = torch.zeros((3, 50), dtype=torch.float16)
    for bad in (x[0], x.unsqueeze(0)):
        with pytest.raises(ValueError):
            ams.ams_logprobs(bad)
    with pytest.raises(TypeError):
        ams.ams_logprobs(x.to(torch.bfloat16))
    with pytest.raises(ValueError):
        ams.ams_logprobs(x)  # not on a GPU
