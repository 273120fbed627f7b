"""The encoder block's operators in plain float64 torch, with bounds on how far a
result with float32 sums and one final rounding may be off.

u(t) is half a unit in the last place relative to the value (bf16 2^-8, fp16
2^-11, float32 2^-24); a float32 sum of n terms in any order is off by at most
about n 2^-24 times the sum of their magnitudes.
"""
import math

import torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F32 = 2.0 ** -24


def u(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half the spacing of the subnormals: the rounding of values near zero."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def act(name, v):
    if name == "relu":
        return v.clamp(min=0)
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    return v


def slope(name, v):
    if name == "relu":
        return (v > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(v / math.sqrt(2))) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (v + 0.044715 * v ** 3))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * c * (1 + 3 * 0.044715 * v * v)
    if name == "silu":
        p = 1 / (1 + torch.exp(-v))
        return p * (1 + v * (1 - p))
    return torch.ones_like(v)


def linear(x, w, b, name, res, scale):
    """(out, pre) in float64 and the bounds of their float32 values before the final
    rounding."""
    x, w = x.double(), w.double()
    K = x.shape[-1]
    pre, mag = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        pre, mag = pre + b.double(), mag + b.double().abs()
    e_pre = (K + 2) * F32 * mag
    out = scale * act(name, pre)
    # an activation's slope is at most 1.13; its own evaluation is off by a few
    # float32 roundings of values up to |pre| + 1
    e = abs(scale) * (1.13 * e_pre + (16 * F32 * (pre.abs() + 1) if name != "none" else 0))
    e = e + 2 * F32 * out.abs()
    if res is not None:
        out = out + res.double()
        e = e + F32 * (out.abs() + res.double().abs())
    return out, pre, e, e_pre


def close(got, want, err):
    """got against want, off by at most err before the rounding to got's type."""
    g = got.double().cpu()
    lim = err + u(got.dtype) * (want.abs() + err) + tiny(got.dtype)
    bad = ~((g - want).abs() <= lim) & ~(g == want)
    assert not bad.any(), (
        f"{int(bad.sum())} of {bad.numel()} off, worst "
        f"{float(((g - want).abs() / lim)[bad].max()):.3g} times the bound, first at "
        f"{bad.nonzero()[0].tolist()}: {float(g[bad][0]):.9g} for {float(want[bad][0]):.9g}")


def linear_grads(g, x, w, pre, name, scale, dtype, formed):
    """Gradients in float64 and their bounds; `pre` is what the backward is given,
    `formed`: d is rounded to `dtype` before the products."""
    g, x, w = g.double(), x.double(), w.double()
    s = slope(name, pre.double()) if name != "none" else torch.ones_like(g)
    d = scale * g * s
    e32 = (24 * F32 * (scale * g).abs() if name != "none" else 2 * F32 * d.abs())
    ed = e32 + ((u(dtype) * (d.abs() + e32) + tiny(dtype)) if formed else 0)
    M, N = g.shape
    dm = d.abs() + ed
    out = {"x": (d @ w, ed @ w.abs() + (N + 4) * F32 * (dm @ w.abs())),
           "weight": (d.t() @ x, ed.t() @ x.abs() + (M + 4) * F32 * (dm.t() @ x.abs())),
           "bias": (d.sum(0), (e32 + (M + 4) * F32 * dm).sum(0))}
    return out
