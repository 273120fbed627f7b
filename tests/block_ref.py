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
        # (1 + erf(x) cancels for negative x, in float64 too)
        return 0.5 * v * torch.erfc(-v / math.sqrt(2))
    if name == "gelu_tanh":   # (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
        return v / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    return v


def slope(name, v):
    if name == "relu":
        return (v > 0).double()
    if name == "gelu":
        return 0.5 * torch.erfc(-v / math.sqrt(2)) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
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


# ---- norms -----------------------------------------------------------------------------------

# A row's sums: 16 terms in a lane, then at most six lane exchanges and 16
# wavefronts, plus the roundings of the terms themselves.
DEPTH = 48


def stats(v, kind, eps):
    """(vhat, r, bound of vhat's float32 value, relative bound of r's)."""
    v = v.double()
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[..., :1])
    em = DEPTH * F32 * v.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    d = v - mean
    var = (d * d).mean(-1, keepdim=True) + eps
    r = 1 / torch.sqrt(var)
    # the mean's error is second order in the variance: sum d is 0
    dr = (DEPTH / 2 + 4) * F32 + (em * em + 2 * em * DEPTH * F32 * d.abs().mean(-1, keepdim=True)) / var
    return d * r, r, r * (em + F32 * d.abs()) + (d * r).abs() * (dr + 2 * F32), dr


def normed(v, kind, eps, weight, bias):
    """(N(v) weight + bias, bound)."""
    h, _, e, _ = stats(v, kind, eps)
    if weight is not None:
        h, e = h * weight.double(), e * weight.double().abs()
    e = e + 3 * F32 * h.abs()
    if bias is not None:
        h = h + bias.double()
        e = e + F32 * (bias.double().abs() + h.abs())
    return h, e


def stream(x, residual, gate, scale, kind, pw, pb, eps):
    """(s before its rounding, bound, u, bound of u)."""
    u, eu = (normed(x, kind, eps, pw, pb) if kind else (x.double(), torch.zeros_like(x.double())))
    f = factor(gate, scale, x)
    s = f * u
    e = f.abs() * eu + 3 * F32 * s.abs()
    if residual is not None:
        s = s + residual.double()
        e = e + 2 * F32 * s.abs()
    return s, e, u, eu


def factor(gate, scale, x):
    """scale * gate over x's rows [M, C]."""
    if gate is None:
        return torch.full_like(x.double(), scale)
    g = gate.double()
    if g.dim() == 2:
        g = g.repeat_interleave(x.shape[0] // g.shape[0], 0)
    return scale * g.expand(x.shape)


def norm_grad(h, eh, v, kind, eps):
    """r (h - mean(h) - vhat mean(h vhat)) and its bound, `eh` that of h."""
    vh, r, ev, dr = stats(v, kind, eps)
    m1 = h.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(r)
    m2 = (h * vh).mean(-1, keepdim=True)
    out = r * (h - m1 - vh * m2)
    a = h.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(r)
    b = (h * vh).abs().mean(-1, keepdim=True)
    am = eh.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(r)
    e = r * (eh + am + vh.abs() * (eh * vh.abs()).mean(-1, keepdim=True)
             + ev * b + vh.abs() * (h.abs() * ev).mean(-1, keepdim=True)
             + DEPTH * F32 * (h.abs() + a + vh.abs() * b))
    return out, e + out.abs() * dr + 4 * F32 * r * (h.abs() + a + vh.abs() * b)


def norm_grads(gy, gs, x, s, gate, scale, norm, weight, post, pw, pb, eps):
    """{name: (gradient, bound)} of rows [M, C]."""
    M = x.shape[0]
    zero = torch.zeros_like(x.double())
    ds, eds = (gs.double() if gs is not None else zero), zero
    out = {}
    if norm and gy is not None:
        g = gy.double()
        h = g * (weight.double() if weight is not None else 1.0)
        t, e = norm_grad(h, F32 * h.abs(), s, norm, eps)
        sh, _, es, _ = stats(s, norm, eps)
        out["weight"] = total(g * sh, g.abs() * es, M)
        out["bias"] = total(g, zero, M)
        ds = ds + t
        eds = e + 2 * F32 * (ds.abs() + t.abs())
    out["residual"] = (ds, eds)
    f = factor(gate, scale, x)
    du = f * ds
    edu = f.abs() * eds + 3 * F32 * du.abs()
    u, eu = normed(x, post, eps, pw, pb) if post else (x.double(), zero)
    dg, edg = scale * ds * u, abs(scale) * (eds * u.abs() + ds.abs() * eu + eds * eu)
    G = gate.shape[0] if gate is not None and gate.dim() == 2 else 0
    if G:
        parts = [total(a, b, M // G) for a, b in zip(dg.chunk(G), edg.chunk(G))]
        out["gate"] = tuple(torch.stack(p) for p in zip(*parts))
    else:
        out["gate"] = total(dg, edg, M)
    if post:
        xh, _, ex, _ = stats(x, post, eps)
        out["post_weight"] = total(du * xh, edu * xh.abs() + du.abs() * ex, M)
        out["post_bias"] = total(du, edu, M)
        h = pw.double() if pw is not None else 1.0
        out["x"] = norm_grad(du * h, edu * abs(h) + F32 * (du * h).abs(), x, post, eps)
    else:
        out["x"] = (du, edu)
    return out


def total(v, e, n):
    """A sum over rows in float32 and its bound."""
    return v.sum(0), e.sum(0) + (n + 24) * F32 * (v.abs() + e).sum(0)
