"""The norms around a block on the GPU against float64, over odd widths, types,
strides, gates and residuals; their gradients against the formulas' and against
differences."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

import block_ref as ref  # noqa: E402

TYPES = [("f32", "f32", "f32"), ("f16", "f16", "f16"), ("bf16", "bf16", "bf16"),
         ("bf16", "f32", "bf16"), ("f16", "f32", "f32"), ("bf16", "bf16", "f32")]
SIZES = [(1, 1), (1, 8), (2, 7), (70, 9), (3, 33), (5, 64), (7, 65), (530, 32), (17, 99), (33, 128),
         (9, 255), (301, 256), (5, 257), (4, 512), (6, 771), (5, 1024), (3, 1031), (3, 2048), (2, 2500),
         (3, 4096), (2, 5001), (2, 8192), (3, 8200), (2, 16384)]
NAMES = ("x", "residual", "gate", "weight", "bias", "post_weight", "post_bias")


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


def make(seed, M, C, types, kind="layer", post=None, residual=True, gate="channel", affine=True, G=1,
         mean=0.25):
    dt, sdt, pdt = (ref.DTYPES[t] for t in types)
    gen = torch.Generator().manual_seed(seed)

    def rand(*shape, dtype, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen) * std + mean).to(dtype)

    t = dict.fromkeys(NAMES)
    t["x"] = rand(M, C, dtype=dt, std=1.5, mean=mean)
    if residual:
        t["residual"] = rand(M, C, dtype=sdt, mean=mean)
    if gate:
        t["gate"] = rand(*((G, C) if gate == "sample" else (C,)), dtype=pdt, std=0.3, mean=0.5)
    if affine:
        t["weight"] = rand(C, dtype=pdt, std=0.1, mean=1.0)
        if kind == "layer":
            t["bias"] = rand(C, dtype=pdt, std=0.1)
        if post:
            t["post_weight"] = rand(C, dtype=pdt, std=0.1, mean=1.0)
            t["post_bias"] = rand(C, dtype=pdt, std=0.1)
    gy = rand(M, C, dtype=dt)
    gs = rand(M, C, dtype=sdt if residual else dt)
    return t, gy, gs


def on(t):
    return {k: None if v is None else v.to("cuda") for k, v in t.items()}


def grouped(t, G):
    """[M, C] tensors as [G, M / G, C]."""
    return {k: v.reshape(G, -1, v.shape[-1]) if k in ("x", "residual") and v is not None else v
            for k, v in t.items()}


def check_forward(fb, t, kind, post, scale, eps, G=1):
    d = grouped(on(t), G) if t["gate"] is not None and t["gate"].dim() == 2 else on(t)
    y, s = fb.norm_forward(d["x"], d["weight"], d["bias"], d["residual"], d["gate"], scale, kind, post,
                           d["post_weight"], d["post_bias"], eps)
    want, e, _, _ = ref.stream(t["x"], t["residual"], t["gate"], scale, post, t["post_weight"],
                               t["post_bias"], eps)
    s2 = s.reshape(t["x"].shape)
    ref.close(s2, want, e)
    if kind:
        # the norm reads s as stored
        ref.close(y.reshape(t["x"].shape), *ref.normed(s2.cpu(), kind, eps, t["weight"], t["bias"]))
    else:
        assert y is None
    return y, s


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("M,C", SIZES)
def test_forward_sizes(fb, device, M, C, types):
    t, _, _ = make(M + C, M, C, types)
    check_forward(fb, t, "layer", None, 0.5, 1e-5)
    t, _, _ = make(M + C, M, C, types, "rms", "layer", gate=None)
    check_forward(fb, t, "rms", "layer", 1.0, 1e-6)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("kind,post", [("layer", None), ("rms", None), ("layer", "layer"), ("rms", "rms"),
                                       (None, "rms"), (None, "layer"), ("layer", "rms")])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("gate,G", [(None, 1), ("channel", 1), ("sample", 1), ("sample", 6)])
def test_forward_forms(fb, device, types, kind, post, residual, gate, G):
    for affine in (True, False):
        t, _, _ = make(3, 42, 72, types, kind or "layer", post, residual, gate, affine, G)
        if not kind:
            t["weight"] = t["bias"] = None
        check_forward(fb, t, kind, post, -0.75, 1e-5, G)


def test_forward_without_anything_to_add(fb, device):
    """s is x itself."""
    t, _, _ = make(1, 9, 40, ("bf16",) * 3, residual=False, gate=None)
    d = on(t)
    y, s = fb.norm_forward(d["x"], d["weight"], d["bias"])
    assert s is d["x"]
    ref.close(y, *ref.normed(t["x"], "layer", 1e-5, t["weight"], t["bias"]))
    into = torch.empty_like(d["x"])
    y2, s2 = fb.norm_forward(d["x"], d["weight"], d["bias"], out_s=into)
    assert s2 is into and torch.equal(into, d["x"]) and torch.equal(y, y2)


@pytest.mark.parametrize("C", [33, 256, 771])
def test_forward_strides(fb, device, C):
    """Rows inside wider tensors, what lies around the outputs left as it was; the
    residual in place."""
    t, _, _ = make(2, 13, C, ("bf16", "f32", "bf16"))
    d = on(t)
    y0, s0 = fb.norm_forward(d["x"], d["weight"], d["bias"], d["residual"], d["gate"])

    def inside(v, before, after):
        big = torch.full((v.shape[0] + 2, before + v.shape[1] + after), 7.0, dtype=v.dtype, device=device)
        view = big[1:-1, before:before + v.shape[1]]
        view.copy_(v)
        return big, view

    _, x = inside(d["x"], 3, 4)
    bs, s = inside(d["residual"], 1, 2)
    by, y = inside(torch.zeros_like(d["x"]), 5, 1)
    ry, rs = fb.norm_forward(x, d["weight"], d["bias"], s, d["gate"], out=y, out_s=s)
    assert ry is y and rs is s and torch.equal(y, y0) and torch.equal(s, s0)
    for big, lo in ((bs, 1), (by, 5)):
        keep = torch.ones_like(big, dtype=torch.bool)
        keep[1:-1, lo:lo + C] = False
        assert (big[keep] == 7).all()


def test_forward_far_means_and_constant_rows(fb, device):
    """Rows far from zero keep their small differences (the variance sums squared
    differences from the mean); rows without any come out as the bias."""
    t, _, _ = make(5, 20, 200, ("f32",) * 3, residual=False, gate=None, mean=1000.0)
    t["x"][3] = 12.5
    t["x"][4] = 0.0
    check_forward(fb, t, "layer", None, 1.0, 1e-5)
    check_forward(fb, t, "rms", None, 1.0, 1e-5)
    d = on(t)
    y, _ = fb.norm_forward(d["x"], d["weight"], d["bias"])
    assert torch.equal(y[4], d["bias"]) and torch.equal(y[3], d["bias"])


def test_nan_and_infinity_stay_in_their_rows(fb, device):
    for C in (33, 128, 1000, 4100):
        t, gy, gs = make(6, 37, C, ("bf16",) * 3, post="rms")
        d = on(t)
        kw = dict(gate=d["gate"], norm="layer", post_norm="rms", post_weight=d["post_weight"],
                  post_bias=d["post_bias"])
        y0, s0 = fb.norm_forward(d["x"], d["weight"], d["bias"], d["residual"], **kw)
        gy, gs = gy.cuda(), gs.cuda()
        b0 = fb.norm_backward(gy, gs, d["x"], s0, d["weight"], want=("x", "residual"), **kw)
        d["x"][5, C // 2] = float("nan")
        d["residual"][11, 0] = float("inf")
        y, s = fb.norm_forward(d["x"], d["weight"], d["bias"], d["residual"], **kw)
        b = fb.norm_backward(gy, gs, d["x"], s, d["weight"], want=("x", "residual"), **kw)
        keep = torch.ones(37, dtype=torch.bool, device=device)
        keep[5] = keep[11] = False
        assert torch.equal(y[keep], y0[keep]) and torch.equal(s[keep], s0[keep])
        assert all(torch.equal(b[k][keep], b0[k][keep]) for k in b)
        assert y[5].isnan().all() and y[11].isnan().all()


def check_backward(fb, t, gy, gs, kind, post, scale, eps, G=1, drop=()):
    d = grouped(on(t), G) if t["gate"] is not None and t["gate"].dim() == 2 else on(t)
    _, s = fb.norm_forward(d["x"], d["weight"], d["bias"], d["residual"], d["gate"], scale, kind, post,
                           d["post_weight"], d["post_bias"], eps)
    shape = d["x"].shape
    gy = None if "y" in drop or not kind else gy
    gs = None if "s" in drop else gs
    want = [k for k in NAMES if t[k] is not None]
    args = [None if g is None else g.cuda().reshape(shape) for g in (gy, gs)]
    kw = dict(weight=d["weight"], gate=d["gate"], scale=scale, norm=kind, post_norm=post,
              post_weight=d["post_weight"], post_bias=d["post_bias"], eps=eps)
    got = fb.norm_backward(*args, d["x"], s, want=want, **kw)
    exact = ref.norm_grads(gy, gs, t["x"], s.reshape(t["x"].shape).cpu(), t["gate"], scale, kind,
                           t["weight"], post, t["post_weight"], t["post_bias"], eps)
    for k in want:
        if k in ("weight", "bias") and gy is None:
            assert (got[k] == 0).all()
            continue
        assert got[k].dtype == (s.dtype if k == "residual" else t[k].dtype)
        v, e = exact[k]
        ref.close(got[k].reshape(v.shape), v, e)
    again = fb.norm_backward(*args, d["x"], s, want=want, **kw)
    assert all(torch.equal(got[k], again[k]) for k in got)
    for k in want:   # one at a time
        one = fb.norm_backward(*args, d["x"], s, want=(k,), **kw)
        assert list(one) == [k] and torch.equal(one[k], got[k])


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("M,C", SIZES + [(5000, 40)])
def test_backward_sizes(fb, device, M, C, types):
    t, gy, gs = make(M + C, M, C, types)
    check_backward(fb, t, gy, gs, "layer", None, 0.5, 1e-5)
    t, gy, gs = make(M + C, M, C, types, "rms", "layer", gate="sample")
    check_backward(fb, t, gy, gs, "rms", "layer", 1.0, 1e-6)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("kind,post", [("layer", None), ("rms", None), ("layer", "layer"), ("rms", "rms"),
                                       (None, "rms"), (None, "layer"), ("layer", "rms")])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("gate,G", [(None, 1), ("channel", 1), ("sample", 6)])
def test_backward_forms(fb, device, types, kind, post, residual, gate, G):
    for affine, drop in ((True, ()), (False, ()), (True, ("y",)), (True, ("s",))):
        if len(drop) and not kind and "s" in drop:
            continue
        t, gy, gs = make(3, 42, 72, types, kind or "layer", post, residual, gate, affine, G)
        if not kind:
            t["weight"] = t["bias"] = None
        check_backward(fb, t, gy, gs, kind, post, -0.75, 1e-5, G, drop)


@pytest.mark.parametrize("kind,post", [("layer", "rms"), ("rms", "layer")])
def test_backward_against_differences(fb, device, kind, post):
    """<grad, v> against (L(+h v) - L(-h v)) / 2h in float32, L = <y, gy> + <s, gs>,
    for h and 2 h: the difference quotient's error is c h^2 + r / h with r the
    rounding of the two L (48 + 8 roundings of its terms' magnitude), so the two
    quotients bound c from their difference, 3 c h^2 up to roundings; the next
    term, of order h^4, is taken as a quarter of it again."""
    t, gy, gs = make(8, 11, 48, ("f32",) * 3, "layer", post, True, "channel")
    d = on(t)
    gy, gs = gy.cuda(), gs.cuda()
    h, eps, scale = 2.0 ** -6, 1e-3, 0.5

    def forward(a):
        return fb.norm_forward(a["x"], a["weight"], a["bias"], a["residual"], a["gate"], scale, kind, post,
                               a["post_weight"], a["post_bias"], eps)

    y, s = forward(d)
    grads = fb.norm_backward(gy, gs, d["x"], s, d["weight"], d["gate"], scale, kind, post,
                             d["post_weight"], d["post_bias"], eps, want=NAMES)
    gen = torch.Generator().manual_seed(2)
    mag = float((gy.double() * y.double()).abs().sum() + (gs.double() * s.double()).abs().sum()
                + gy.double().abs().sum() * 4 + gs.double().abs().sum() * 4)
    for k in NAMES:
        v = torch.randn(d[k].shape, generator=gen).cuda()

        def loss(step):
            yy, ss = forward({**d, k: d[k] + step * v})
            return float((yy.double() * gy.double()).sum() + (ss.double() * gs.double()).sum())

        num = (loss(h) - loss(-h)) / (2 * h)
        wide = (loss(2 * h) - loss(-2 * h)) / (4 * h)
        ana = float((grads[k].double() * v.double()).sum())
        rounding = 56 * ref.F32 * mag / h
        trunc = (abs(wide - num) + 1.5 * rounding) / 3 * 1.25
        assert trunc < 0.05 * max(1.0, float((grads[k].double() * v.double()).abs().sum()))
        assert abs(num - ana) <= trunc + rounding, (k, num, ana, trunc, rounding)


@pytest.mark.parametrize("types", [("f32",) * 3, ("bf16", "f32", "bf16")], ids="-".join)
@pytest.mark.parametrize("post", [None, "layer"])
def test_autograd_is_the_explicit_calls(fb, device, types, post):
    t, gy, gs = make(4, 60, 56, types, "layer", post, True, "sample", True, 3)
    d = grouped(on(t), 3)
    leaves = {k: v.clone().requires_grad_() for k, v in d.items() if v is not None}
    args = {k: leaves.get(k) for k in NAMES}
    y, s = fb.norm_autograd(args["x"], args["weight"], args["bias"], args["residual"], args["gate"], 0.5,
                            "layer", post, args["post_weight"], args["post_bias"])
    y0, s0 = fb.norm_forward(d["x"], d["weight"], d["bias"], d["residual"], d["gate"], 0.5, "layer", post,
                             d["post_weight"], d["post_bias"])
    assert torch.equal(y.detach(), y0) and torch.equal(s.detach(), s0)
    gy, gs = gy.cuda().reshape(y.shape), gs.cuda().reshape(s.shape)
    kw = dict(gate=d["gate"], scale=0.5, post_norm=post, post_weight=d["post_weight"],
              post_bias=d["post_bias"], want=list(leaves))
    for a, b in ((gy, gs), (gy, None), (None, gs)):
        outs, into = zip(*[(o, g) for o, g in ((y, a), (s, b)) if g is not None])
        got = torch.autograd.grad(outs, list(leaves.values()), into, retain_graph=True, allow_unused=True)
        want = fb.norm_backward(a, b, d["x"], s0, d["weight"], **kw)
        assert all(torch.equal(g, want[k]) for g, k in zip(got, leaves))
    # a norm alone: s is x
    x = d["x"].clone().requires_grad_()
    y, s = fb.norm_autograd(x, d["weight"], d["bias"])
    assert s is x
    (g,) = torch.autograd.grad(y.sum(), x)
    want = fb.norm_backward(torch.ones_like(y), None, d["x"], d["x"], d["weight"])
    assert torch.equal(g, want["x"])


def test_empty(fb, device):
    for dt in ref.DTYPES.values():
        for M, C in ((0, 8), (0, 0), (3, 0)):
            x = torch.ones(M, C, dtype=dt, device=device)
            w = torch.ones(C, dtype=dt, device=device)
            y, s = fb.norm_forward(x, w, w, x, w)
            assert y.shape == s.shape == x.shape
            r = fb.norm_backward(y, s, x, s, w, w, want=NAMES[:5])
            assert r["x"].shape == x.shape and (r["weight"] == 0).all() and (r["gate"] == 0).all()


def test_rows_past_32_bits(fb, device):
    """x, s and y past 2^32 bytes: the last rows are their own norms."""
    M, C = (1 << 21) + 3, 1032
    x = torch.zeros(M, C, dtype=torch.bfloat16, device=device)
    x[-3:] = torch.randn(3, C, device=device).to(torch.bfloat16)
    w = torch.randn(C, device=device).to(torch.bfloat16)
    y, s = fb.norm_forward(x, w, None, None, w, norm="rms")
    y2, s2 = fb.norm_forward(x[-3:], w, None, None, w, norm="rms")
    assert torch.equal(y[-3:], y2) and torch.equal(s[-3:], s2) and (y[:-3] == 0).all()
    r = fb.norm_backward(y, None, x, s, w, w, norm="rms", want=("x",))
    r2 = fb.norm_backward(y2, None, x[-3:], s2, w, w, norm="rms", want=("x",))
    assert torch.equal(r["x"][-3:], r2["x"]) and (r["x"][:-3] == 0).all()
