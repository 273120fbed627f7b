"""The gradients of the encoder block's operators under hooks on saved tensors that give
back slices of wider buffers: the same as without hooks."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


def wide_there(t):
    n = t.shape[-1]
    if t.dim() == 1:
        view = torch.full((2 * n,), 99.0, dtype=t.dtype, device=t.device)[::2]
    else:
        view = torch.full((*t.shape[:-1], n + 11), 99.0, dtype=t.dtype, device=t.device)[..., 3:n + 3]
    view.copy_(t)
    return view


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M,K,N", [(50, 40, 64), (600, 256, 256), (130, 33, 71)])
def test_linear(fb, device, M, K, N, act):
    gen = torch.Generator().manual_seed(M)
    for dtype in (torch.float32, torch.bfloat16):
        x, w, b = (torch.randn(s, generator=gen).to(dtype).to(device).requires_grad_()
                   for s in ((M, K), (N, K), (N,)))
        g = torch.randn(M, N, generator=gen).to(dtype).to(device)

        def step():
            return torch.autograd.grad(fb.linear_autograd(x, w, b, act), [x, w, b], g)

        want = step()
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wide_there):
            got = step()
        assert torch.equal(got[2], want[2])
        # other strides may take another kernel: the same sum of n terms in another order,
        # each order off by at most (n + 2) 2^-24 of the terms' magnitude, and each sum
        # rounded; a slope is at most 1.13
        d = 1.13 * g.double().abs()
        for a, c, n, mag in ((got[0], want[0], N, d @ w.detach().double().abs()),
                             (got[1], want[1], M, d.t() @ x.detach().double().abs())):
            e = (n + 2) * 2.0 ** -24 * mag
            lim = 2 * e + torch.finfo(dtype).eps * (c.double().abs() + 2 * e)
            assert ((a.double() - c.double()).abs() <= lim).all()


@pytest.mark.parametrize("samples", [False, True])
@pytest.mark.parametrize("C", [40, 256, 771])
def test_norm(fb, device, C, samples):
    gen = torch.Generator().manual_seed(C)
    make = lambda *s: torch.randn(s, generator=gen).to(device).requires_grad_()
    x, r, gate = make(3, 20, C), make(3, 20, C), make(*((3, C) if samples else (C,)))
    w, b, pw, pb = (make(C) for _ in range(4))
    leaves = [x, r, gate, w, b, pw, pb]
    gy, gs = torch.randn(2, 3, 20, C, generator=gen).to(device)

    def step():
        y, s = fb.norm_autograd(x, w, b, r, gate, 0.5, "layer", "rms", pw, pb)
        return torch.autograd.grad([y, s], leaves, [gy, gs])

    want = step()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wide_there):
        got = step()
    assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_what_was_not_saved_is_refused(fb, device):
    """Host copies, other types and sizes, before anything is enqueued."""
    x = torch.randn(8, 16, device=device, requires_grad=True)
    w = torch.randn(24, 16, device=device, requires_grad=True)
    for bad in (lambda t: t.cpu(), lambda t: t.half(), lambda t: t[:-1]):
        for call in (lambda: fb.linear_autograd(x, w, None, "silu"),
                     lambda: fb.norm_autograd(x, None, None, x.detach())[0]):
            with torch.autograd.graph.saved_tensors_hooks(lambda t: t, bad):
                out = call()
            with pytest.raises(ValueError, match="was saved as"):
                out.sum().backward()
