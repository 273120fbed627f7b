"""Calls of the encoder block's operators with more workgroups than one row of a grid
takes (2^32 threads): the same rows, bit for bit, as calls of a part of them."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


def rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


@pytest.fixture
def gen(device):
    yield torch.Generator(device=device).manual_seed(1)
    torch.cuda.empty_cache()


def test_norm_forward(fb, gen):
    """32 rows a workgroup of 256 threads."""
    M, C = (1 << 29) + 37, 2
    x = rand(gen, M, C)
    y, s = fb.norm_forward(x, scale=0.5)
    for a, b in ((0, 1 << 28), (1 << 28, M)):
        y2, s2 = fb.norm_forward(x[a:b], scale=0.5)
        assert torch.equal(y[a:b], y2) and torch.equal(s[a:b], s2)


def test_linear_forward(fb, gen):
    """64 rows a workgroup of 256 threads."""
    M = (1 << 30) + 70
    x, w = rand(gen, M, 1), rand(gen, 1, 1)
    out = fb.linear_forward(x, w)
    step = 1 << 28
    for a in range(0, M, step):
        assert torch.equal(out[a:a + step], (x[a:a + step].float() * w.float()).to(torch.bfloat16))


@pytest.mark.parametrize("M,C", [((1 << 24) + 5, 8), ((1 << 16) + 16, 4096)])
def test_norm_backward_of_many_samples(fb, gen, M, C):
    """A workgroup for each sample, and for each 16 channels of its gate's gradient."""
    x, gate, gy = (rand(gen, M, C) for _ in range(3))
    _, s = fb.norm_forward(x, gate=gate)
    got = fb.norm_backward(gy, None, x, s, gate=gate, want=("x", "gate"))
    for a, b in ((0, M // 2), (M // 2, M)):
        part = fb.norm_backward(gy[a:b], None, x[a:b], s[a:b], gate=gate[a:b], want=("x", "gate"))
        assert torch.equal(got["x"][a:b], part["x"]) and torch.equal(got["gate"][a:b], part["gate"])
