"""What the encoder block's gradients read when hooks on saved tensors give back other
tensors than were saved (CPU only: the calls into the library are caught, and what they
would read at the addresses and strides they are given is compared with what was saved)."""
import ctypes

import pytest
import torch

from paper_2607_10071_amd import block

M, K, N, C = 6, 10, 7, 9
CPU = torch.device("cpu")


def wide(t):
    """The same values as a column slice of a wider buffer; a vector as every second
    element of a longer one."""
    if t.dim() == 1:
        big = torch.full((2 * t.numel(),), 99.0, dtype=t.dtype)
        view = big[::2]
    else:
        big = torch.full((*t.shape[:-1], t.shape[-1] + 5), 99.0, dtype=t.dtype)
        view = big[..., 2:-3]
    view.copy_(t)
    return view


def read(t, ld, rows, width):
    """What a kernel reads of `rows` rows at stride `ld` from t's address."""
    return torch.as_strided(t, (rows, width), (ld, 1), t.storage_offset()).clone()


@pytest.fixture
def caught(monkeypatch):
    """The arguments of the gradients' calls; the forwards give zeros."""
    calls = []

    def linear_forward(x, weight, bias, activation, residual, scale, out, out_dtype, pre, stream):
        rows = x.numel() // K
        if pre is not None:
            pre.copy_(torch.arange(rows * N).reshape(pre.shape))
        return (torch.zeros(*x.shape[:-1], N),
                (rows, K, K, K, N, 0, 0, block._act_code(activation), scale, CPU))

    def linear_gradients(sizes, g, ldo, x, weight, pre, ldp, gx, ldgx, gw, ldgw, gb, stream):
        rows = sizes[0]
        calls.append({"grad": read(g, ldo, rows, N), "x": read(x, sizes[1], rows, K),
                      "weight": read(weight, sizes[2], N, K),
                      "pre": None if pre is None else read(pre, ldp, rows, N)})

    def norm_forward(x, weight, bias, residual, gate, scale, norm, post_norm, post_weight, post_bias,
                     eps, out, out_s, stream):
        rows = x.numel() // C
        s = torch.arange(float(x.numel())).reshape(x.shape)
        return torch.zeros_like(x), s, (rows, C, C, 1 if gate is None or gate.dim() == 1 else
                                        gate.shape[0], C, (), CPU)

    def norm_gradients(sizes, gy, ldgy, gs, ldgs, x, s, gate, vectors, pdt, want, stream):
        rows = sizes[0]
        at = block._PACK_VECTORS.unpack(vectors)
        n = (0 if gate is None else gate.numel(), C, 0, C, C)
        vec = [torch.tensor((ctypes.c_float * k).from_address(a)) if a else None for a, k in zip(at, n)]
        calls.append({"x": read(x, sizes[1], rows, C), "s": read(s, sizes[2], rows, C),
                      **dict(zip(("gate", "weight", "bias", "post_weight", "post_bias"), vec))})
        return {}

    for name, fn in (("_linear_forward", linear_forward), ("_linear_gradients", linear_gradients),
                     ("_norm_forward", norm_forward), ("_norm_gradients", norm_gradients)):
        monkeypatch.setattr(block, name, fn)
    return calls


def leaf(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).requires_grad_()


def linear_pass(unpack, act):
    x, w = leaf(2, M // 2, K), leaf(N, K, seed=1)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        out = block._autograd_functions()["linear"].apply(x, w, None, None, act, 1.0, None)
    out.sum().backward()
    return {"x": x.detach().reshape(M, K), "weight": w.detach(),
            "pre": torch.arange(float(M * N)).reshape(M, N) if act != "none" else None}


def norm_pass(unpack, samples):
    x, res = leaf(2, M // 2, C), leaf(2, M // 2, C, seed=1)
    v = {k: leaf(C, seed=2 + i) for i, k in enumerate(("weight", "bias", "post_weight", "post_bias"))}
    gate = leaf(*((2, C) if samples else (C,)), seed=9)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        y, s = block._autograd_functions()["norm"].apply(x, res, gate, v["weight"], v["bias"],
                                                         v["post_weight"], v["post_bias"], 1.0, "layer",
                                                         "layer", 1e-5)
    (y.sum() + s.sum()).backward()
    return {"x": x.detach().reshape(M, C), "s": torch.arange(float(M * C)).reshape(M, C),
            "gate": gate.detach().reshape(-1), "weight": v["weight"].detach(),
            "post_weight": v["post_weight"].detach(), "post_bias": v["post_bias"].detach()}


def same(call, want):
    for k, t in want.items():
        assert (call[k] is None) == (t is None) and (t is None or torch.equal(call[k], t)), k


@pytest.mark.parametrize("unpack", [lambda t: t, wide], ids=["as saved", "wide"])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_a_linears_gradients_go_by_the_strides_they_get(caught, act, unpack):
    want = linear_pass(unpack, act)
    same(caught[0], want)


@pytest.mark.parametrize("unpack", [lambda t: t, wide], ids=["as saved", "wide"])
@pytest.mark.parametrize("samples", [False, True])
def test_a_norms_gradients_go_by_the_strides_they_get(caught, samples, unpack):
    want = norm_pass(unpack, samples)
    same(caught[0], want)


BAD = {"type": lambda t: t.double(), "fewer rows": lambda t: t[:-1], "place": lambda t: t.to("meta")}


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("which", range(3))
def test_a_linears_saved_tensors_must_be_what_was_saved(caught, bad, which):
    """x, weight and the sums before the activation, one at a time: another type, size
    or device is refused, with no call."""
    n = iter(range(3))
    with pytest.raises(ValueError, match="was saved as"):
        linear_pass(lambda t: BAD[bad](t) if next(n) == which else t, "gelu")
    assert not caught


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("which", range(6))
def test_a_norms_saved_tensors_must_be_what_was_saved(caught, bad, which):
    n = iter(range(6))
    with pytest.raises(ValueError, match="was saved as"):
        norm_pass(lambda t: BAD[bad](t) if next(n) == which else t, True)
    assert not caught
