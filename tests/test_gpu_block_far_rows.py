"""The encoder block's operators on inputs whose rows lie more than 2^20 elements apart
(the last token of each of a batch of sequences, say): the same as on copies of them."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

B, T, C, N = 5, 300, 4096, 72   # rows 1228800 elements apart


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


@pytest.fixture
def rand(device):
    gen = torch.Generator(device=device).manual_seed(3)
    return lambda *s: torch.randn(s, generator=gen, device=device, dtype=torch.bfloat16)


def apart(t):
    """t's rows FAR from each other."""
    far = torch.empty(t.shape[0], 1 << 21, dtype=t.dtype, device=t.device)[:, 7:7 + t.shape[1]]
    far.copy_(t)
    return far


def test_linear(fb, rand):
    hidden, w, b, r = rand(B, T, C), rand(N, C), rand(N), rand(B, N)
    x = hidden[:, -1]
    want = fb.linear_forward(x.contiguous(), w, b, "silu", r)
    assert torch.equal(fb.linear_forward(x, apart(w), b, "silu", apart(r)), want)
    pre, g = rand(B, N), rand(B, N)
    want = fb.linear_backward(g, x.contiguous(), w, pre, "silu")
    got = fb.linear_backward(apart(g), x, apart(w), apart(pre), "silu")
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_norm(fb, rand):
    hidden, w, r, gy, gs = rand(B, T, C), rand(C), rand(B, C), rand(B, C), rand(B, C)
    x = hidden[:, -1]
    y, s = fb.norm_forward(x.contiguous(), w, None, r, post_norm="rms")
    y2, s2 = fb.norm_forward(x, w, None, apart(r), post_norm="rms")
    assert torch.equal(y, y2) and torch.equal(s, s2)
    kw = dict(weight=w, post_norm="rms", want=("x", "residual", "weight"))
    want = fb.norm_backward(gy, gs, x.contiguous(), s, **kw)
    got = fb.norm_backward(apart(gy), apart(gs), x, apart(s), **kw)
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_autograd(fb, rand):
    hidden, w, v = rand(B, T, C).requires_grad_(), rand(N, C).requires_grad_(), rand(N).requires_grad_()
    g = rand(B, T, N)

    def step(x, into):
        y, _ = fb.norm_autograd(fb.linear_autograd(x, w, None, "gelu"), v)
        return torch.autograd.grad(y, [hidden, w, v], into)

    far = apart(g[:, -1])
    got, want = step(hidden[:, -1], far), step(hidden[:, -1].contiguous(), g[:, -1].contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_another_stream(fb, rand):
    """The copy is made in the order of the call's stream: values that this stream alone has
    written so far are the ones that count."""
    x, w = apart(rand(40, C)), rand(N, C)
    big = torch.randn(4096, 4096, device="cuda")
    new = rand(40, C)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for handle in (side, side.cuda_stream):
        out = torch.empty(40, N, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(10):
                big @ big
            x.copy_(new)
        fb.linear_forward(x, w, out=out, stream=handle)
        torch.cuda.synchronize()
        assert torch.equal(out, fb.linear_forward(new, w))
        new = rand(40, C)
        torch.cuda.synchronize()


def test_what_is_not_copied(fb, rand):
    x, w = rand(B, C), rand(N, C)
    out = apart(rand(B, N))
    with pytest.raises(fb.FlashBevError):
        fb.linear_forward(x, w, out=out)
    with pytest.raises(fb.FlashBevError):
        fb.norm_forward(x, out=apart(x))
    with pytest.raises(ValueError):
        fb.prepare_linear_forward(apart(x), w, out=rand(B, N))
