"""Inputs whose rows lie further apart than the library takes (CPU only: the calls into
the library are caught, and what they would read is compared with the tensors)."""
import contextlib
import re

import pytest
import torch

import paper_2607_10071_amd as fb
from paper_2607_10071_amd import block
from test_linear_abi import HEADER

FAR = (1 << 20) + 3   # elements from one row to the next
K, N = 5, 4


class Device(torch.Tensor):
    """A host tensor that says it is on the device."""

    is_cuda = property(lambda self: True)


def tensor(t):
    return t.as_subclass(Device)


def far(rows, width, seed=0):
    """Rows at stride FAR, of which the first and the last hold numbers."""
    t = torch.empty((rows - 1) * FAR + width)
    view = t.as_strided((rows, width), (FAR, 1))
    view.copy_(torch.randn(rows, width, generator=torch.Generator().manual_seed(seed)))
    return tensor(view)


def near(rows, width, seed=0):
    return tensor(torch.randn(rows, width, generator=torch.Generator().manual_seed(seed)))


@pytest.fixture
def calls(monkeypatch):
    made = []

    def packed_call(name, kinds):
        return lambda *args: made.append((name, args)) or 0

    monkeypatch.setattr(block, "_packed_call", packed_call)
    monkeypatch.setattr(block, "_stream_handle", lambda stream, dev: 0)
    monkeypatch.setattr(block, "_on_device", lambda dev: contextlib.nullcontext())
    if hasattr(block, "_on_stream"):
        monkeypatch.setattr(block, "_on_stream", lambda dev, s: contextlib.nullcontext())
    for need in ("_linear_need", "_linear_backward_need", "_norm_need"):
        monkeypatch.setattr(block, need, lambda *a: 0)
    return made


def test_the_limit_is_the_headers():
    limit = int(re.search(r"FLASHBLOCK_LD_MAX (\d+)", open(HEADER).read())[1])
    assert block.LD_MAX == limit < FAR


def strides(pack, args, n):
    return pack.unpack(args[0])[1:n]


def test_linear_forward(calls):
    x, w, r = far(3, K), far(N, K, 1), far(3, N, 2)
    fb.linear_forward(x, w, residual=r)
    (_, args), = calls
    assert strides(block._PACK_LINEAR, args, 6) == (K, K, N, N, N)
    # what is near stays where it is
    x = near(3, K)
    fb.linear_forward(x, w)
    assert calls[1][1][1] == x.data_ptr()


def test_linear_backward(calls):
    g, x, w, pre = far(3, N), far(3, K), far(N, K), far(3, N)
    fb.linear_backward(g, x, w, pre, "relu")
    assert strides(block._PACK_LINEAR, calls[0][1], 6) == (K, K, N, N, N)


def test_norm_forward(calls):
    x, r = far(3, K), far(3, K, 1)
    y, s = fb.norm_forward(x, residual=r)
    assert strides(block._PACK_NORM, calls[0][1], 5) == (K, K, K, K)
    y, s = fb.norm_forward(x)
    assert s is x and strides(block._PACK_NORM, calls[1][1], 5) == (K, K, K, K)


def test_norm_backward(calls):
    t = [far(3, K, i) for i in range(4)]
    fb.norm_backward(*t, want=("x", "residual"))
    assert strides(block._PACK_NORM, calls[0][1], 5) == (K, K, K, K)


def test_gradients_that_autograd_hands_over():
    t = far(3, K)
    got, ld = block._as_rows(t, K)
    assert ld == K and got.is_contiguous() and torch.equal(got, t)


def test_outputs_and_prepared_calls_are_not_copied(calls):
    """An output is written where it is (the library refuses it); a prepared call reads its
    tensors anew each time."""
    x, w, out = near(3, K), near(N, K), far(3, N)
    fb.linear_forward(x, w, residual=out, out=out)
    assert strides(block._PACK_LINEAR, calls[0][1], 6) == (K, K, FAR, FAR, N)
    assert calls[0][1][4] == calls[0][1][5] == out.data_ptr()
    with pytest.raises(ValueError, match="prepared"):
        fb.prepare_linear_forward(far(3, K), w, out=near(3, N))
    with pytest.raises(ValueError, match="prepared"):
        fb.prepare_norm_forward(far(3, K), out=near(3, K))
    stream = far(3, K)
    fb.norm_forward(x, residual=stream, out_s=stream)
    assert strides(block._PACK_NORM, calls[1][1], 5) == (K, FAR, FAR, K)
