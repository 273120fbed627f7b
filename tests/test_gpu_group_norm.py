"""Group norm with an activation on the GPU against float64."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2607_10071_amd as fb

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)]
IDS = ["f32", "f16", "bf16", "f16_f32", "bf16_f32"]


def make(N, R, C, dtype, pdt, seed=0, mean=0.5, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 13 * R + C)
    x = (torch.randn((N, R, C), generator=g, device="cuda") * std
         + mean * torch.randn((C,), generator=g, device="cuda")).to(dtype)
    w = (1 + 0.2 * torch.randn(C, generator=g, device="cuda")).to(pdt)
    b = (0.3 * torch.randn(C, generator=g, device="cuda")).to(pdt)
    gy = torch.randn((N, R, C), generator=g, device="cuda").to(dtype)
    return x, w, b, gy


def check_all(x, groups, w, b, gy, act, eps=1e-5):
    N, C = x.shape[0], x.shape[-1]
    leaves = {n: t.detach().double().requires_grad_() for n, t in (("x", x), ("weight", w), ("bias", b)) if t is not None}
    y = ref.group_norm(leaves["x"], groups, leaves.get("weight"), leaves.get("bias"), act, eps)
    stats = torch.empty((N, groups, 2), device="cuda")
    out = fb.group_norm_forward(x, groups, w, b, act, eps, stats=stats)
    t = leaves["x"].detach().reshape(N, -1, groups, C // groups)
    mean, var = t.mean((1, 3)), t.var((1, 3), correction=0)
    rstd = (var + eps).rsqrt()
    # A mean is kept from a value of its group, x[0] of the first channel: joins of some 16 roundings
    # relative to the differences from it, and one to add it.  A join's d^2 has 2 d times the means'
    # errors, so the variance's relative error is 2 e / spread and rstd's half of that, next to some
    # 40 roundings.  xhat: a difference rounded once, relative to x and the mean; the factors have some
    # 6 roundings, an activation 1e-6 of its argument's size (slopes reach 1.13) and more
    size = t.abs().amax((1, 3))
    e_from = 16 * ref.U32 * (t - t[:, :1, :, :1]).abs().mean((1, 3))
    e_mean = e_from + ref.U32 * mean.abs()
    e_rstd = 40 * ref.U32 * rstd + rstd ** 2 * e_from
    assert ((stats[..., 0].double() - mean).abs() <= e_mean + 1e-30).all()
    n = t.shape[1] * t.shape[3]
    assert ((stats[..., 1].double() - rstd).abs() <= e_rstd + 1e-30).all()
    per = C // groups
    wide = lambda s: s.repeat_interleave(per, -1).reshape(N, *([1] * (x.dim() - 2)), C)   # noqa: E731
    xhat = (leaves["x"].detach() - wide(mean)) * wide(rstd)
    aw = w.double().abs() if w is not None else torch.ones(C, device="cuda", dtype=torch.float64)
    ab = b.double().abs() if b is not None else torch.zeros(C, device="cuda", dtype=torch.float64)
    e_hat = wide(rstd * (e_mean + 2 * ref.U32 * size)) + xhat.abs() * (48 * ref.U32 + wide(rstd * e_from))
    e_pre = e_hat * aw + (xhat.abs() * aw + ab) * 6 * ref.U32
    e_y = 1.13 * e_pre + (0 if act == "none" else 1e-6) * (xhat.abs() * aw + ab) + ref.half(x.dtype) * y.detach().abs()
    ref.check(out, y.detach(), e_y + ref._floor(x.dtype), "y")
    names = list(leaves)
    grads = dict(zip(names, torch.autograd.grad(y, list(leaves.values()), gy.double())))
    got = fb.group_norm_backward(gy, x, stats, groups, w, b, act, want=names)
    # d = gy act'(pre): slopes change by at most 1.6 times pre's error and have 2e-6 of their own; relu's
    # steps where pre changes its sign
    pre = xhat * (w.double() if w is not None else 1) + (b.double() if b is not None else 0)
    e_d = gy.double().abs() * ((pre.abs() <= e_pre).double() if act == "relu" else
                               0.0 if act == "none" else 1.6 * e_pre + 2e-6)
    d = gy.double().abs() * 1.13
    fold = lambda v: v.reshape(N, -1, groups, per).mean((1, 3))   # noqa: E731
    rows = 64 + math.sqrt(n)   # of a sum's roundings, in float32 over lanes, chunks and joins
    m1, e1 = fold(d * aw), fold(e_d * aw) + rows * ref.U32 * fold(d * aw)
    m2, e2 = fold(d * aw * xhat.abs()), fold(e_d * aw * xhat.abs() + d * aw * e_hat) + rows * ref.U32 * fold(d * aw * xhat.abs())
    e_x = wide(rstd) * (e_d * aw + wide(e1) + xhat.abs() * wide(e2) + e_hat * wide(m2)
                        + 60 * ref.U32 * (d * aw + wide(m1) + xhat.abs() * wide(m2)))
    ref.check(got["x"], grads["x"], e_x + ref.half(x.dtype) * grads["x"].abs() + ref._floor(x.dtype), "grad_x")
    flat = lambda v: v.reshape(-1, C).sum(0)   # noqa: E731
    rows = 64 + math.sqrt(N * t.shape[1])
    if w is not None:
        e = flat(e_d * xhat.abs() + d * e_hat) + rows * ref.U32 * flat(d * xhat.abs())
        ref.check(got["weight"], grads["weight"], e + ref.half(w.dtype) * grads["weight"].abs() + ref._floor(w.dtype), "grad_weight")
    if b is not None:
        e = flat(e_d) + rows * ref.U32 * flat(d)
        ref.check(got["bias"], grads["bias"], e + ref.half(b.dtype) * grads["bias"].abs() + ref._floor(b.dtype), "grad_bias")
    return out, got


SHAPES = [
    # N, R, C, groups: by one workgroup for a slice, by chunks, over several slices of columns
    (1, 1, 1, 1), (1, 1, 32, 8), (2, 7, 12, 3), (3, 64, 32, 8), (1, 529, 256, 32), (2, 1000, 8, 2), (1, 5000, 1, 1),
    (1, 3000, 256, 1), (2, 777, 330, 30), (6, 2000, 64, 16), (1, 300, 4099, 1), (1, 200, 4096, 2), (1, 3, 16384, 16384),
    (1, 2, 16384, 1), (2, 150, 2400, 5), (1, 20011, 7, 7), (5, 33, 1027, 13),
]


@pytest.mark.parametrize("dtype,pdt", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(shape, dtype, pdt):
    N, R, C, groups = shape
    x, w, b, gy = make(N, R, C, dtype, pdt)
    check_all(x, groups, w, b, gy, "silu")


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R", [50, 4000])
def test_activations(act, dtype, R):
    x, w, b, gy = make(2, R, 96, dtype, dtype, seed=1)
    check_all(x, 12, w, b, gy, act)
    check_all(x, 12, None, None, gy, act)
    check_all(x, 12, w, None, gy, act)
    check_all(x, 12, None, b, gy, act)


@pytest.mark.parametrize("R", [60, 9000])
def test_offsets_far_above_the_spread(R):
    """Means 1e4 times the spread: differences from means lose no digits of the spread."""
    x, w, b, gy = make(2, R, 64, F32, F32, mean=0.0)
    x = x + 1e4
    check_all(x, 8, w, b, gy, "none")
    x[:, : R // 2] += 100.0
    check_all(x, 8, w, b, gy, "none")


@pytest.mark.parametrize("R", [40, 6000])
def test_constant_groups(R):
    x = torch.full((1, R, 64), 3.25, device="cuda", dtype=BF16)
    w, b = torch.ones(64, device="cuda", dtype=BF16), torch.full((64,), 0.5, device="cuda", dtype=BF16)
    out = fb.group_norm_forward(x, 8, w, b)
    assert (out == 0.5).all()


@pytest.mark.parametrize("R", [40, 6000])
def test_nan_stays_in_its_group(R):
    x, w, b, gy = make(2, R, 64, BF16, F32)
    clean = fb.group_norm_forward(x, 8, w, b)
    x = x.clone()
    x[1, R // 2, 13] = math.nan
    out = fb.group_norm_forward(x, 8, w, b)
    assert torch.equal(out[0], clean[0]) and out[1, :, 8:16].isnan().all()
    keep = [c for c in range(64) if not 8 <= c < 16]
    assert torch.equal(out[1][:, keep], clean[1][:, keep])


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("R", [6, 90])
def test_strides_and_maps(dtype, R):
    g = torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn((2, R, 11, 200), generator=g, device="cuda").to(dtype)
    x = wide[..., 3:93]
    w, b = torch.rand(90, generator=g, device="cuda"), torch.rand(90, generator=g, device="cuda")
    gy = torch.randn((2, R, 11, 100), generator=g, device="cuda").to(dtype)[..., 7:97]
    out, got = check_all(x, 9, w, b, gy, "relu")
    again, more = check_all(x.contiguous(), 9, w, b, gy.contiguous(), "relu")
    assert torch.equal(out, again) and all(torch.equal(got[n], more[n]) for n in got)
    room = torch.full((2, R, 11, 120), 5.0, device="cuda", dtype=dtype)
    fb.group_norm_forward(x, 9, w, b, "relu", out=room[..., 5:95])
    assert torch.equal(room[..., 5:95], out)
    room[..., 5:95] = 5.0
    assert (room == 5.0).all()


def test_far_rows():
    base = torch.randn((1 << 20) * 4 + 300, device="cuda")
    x = base.as_strided((1, 4, 64), (1, (1 << 20) + 40, 1))
    assert torch.equal(fb.group_norm_forward(x, 8), fb.group_norm_forward(x.contiguous(), 8))
    with pytest.raises(ValueError, match="elements apart"):
        fb.prepare_group_norm_forward(x, 8, out=torch.empty((1, 4, 64), device="cuda"))


def test_empty():
    for shape in ((0, 5, 8), (2, 0, 8)):
        x = torch.zeros(shape, device="cuda")
        w = torch.ones(8, device="cuda")
        assert fb.group_norm_forward(x, 2, w).shape == shape
        r = fb.group_norm_backward(x, x, torch.zeros((shape[0], 2, 2), device="cuda"), 2, w, None, want=("x", "weight", "bias"))
        assert r["x"].shape == shape and (r["weight"] == 0).all() and (r["bias"] == 0).all()


@pytest.mark.parametrize("dtype,pdt", TYPES, ids=IDS)
def test_autograd(dtype, pdt):
    x, w, b, gy = make(3, 700, 48, dtype, pdt)
    leaves = [t.requires_grad_() for t in (x, w, b)]
    out = fb.group_norm_autograd(x, 6, w, b, "gelu")
    got = torch.autograd.grad(out, leaves, gy)
    _, want = check_all(x.detach(), 6, w.detach(), b.detach(), gy, "gelu")
    for n, t in zip(("x", "weight", "bias"), got):
        assert torch.equal(t, want[n]), n
    (gw,) = torch.autograd.grad(fb.group_norm_autograd(x.detach(), 6, w, None, "gelu"), [w], gy)
    assert gw.dtype == pdt and gw.shape == w.shape
    (gx,) = torch.autograd.grad(fb.group_norm_autograd(x, 6, activation="none").float().sum(), [x])
    # the gradient of a sum is zero: what is left are roundings of the terms 1 and of means of them
    assert gx.double().abs().max() <= 1e-4


def test_same_bits_again_and_on_another_stream():
    x, w, b, gy = make(4, 3000, 256, BF16, F32)
    stats = torch.empty((4, 32, 2), device="cuda")
    first = fb.group_norm_forward(x, 32, w, b, "silu", stats=stats)
    grads = fb.group_norm_backward(gy, x, stats, 32, w, b, "silu", want=("x", "weight", "bias"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = fb.group_norm_forward(x, 32, w, b, "silu")
        more = fb.group_norm_backward(gy, x, stats, 32, w, b, "silu", want=("x", "weight", "bias"))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again) and all(torch.equal(grads[n], more[n]) for n in grads)
    out = torch.empty_like(x)
    call = fb.prepare_group_norm_forward(x, 32, w, b, "silu", out=out)
    call()
    call()
    assert torch.equal(out, first)


@pytest.mark.parametrize("groups", [1, 3])
def test_no_channels(groups):
    x = torch.zeros((2, 100, 0), device="cuda", requires_grad=True)
    out = torch.full_like(x, 3.0)
    assert fb.group_norm_forward(x.detach(), groups).shape == x.shape
    fb.prepare_group_norm_forward(x.detach(), groups, out=out.detach())()
    w = torch.zeros(0, device="cuda", requires_grad=True)
    y = fb.group_norm_autograd(x, groups, w, w, "silu")
    got = torch.autograd.grad(y, [x, w], torch.zeros_like(x))
    assert y.shape == x.shape and got[0].shape == x.shape and got[1].shape == w.shape
    for shape in ((0, 5, 8), (2, 0, 8), (2, 5, 0)):   # the gradient of x alone
        x = torch.zeros(shape, device="cuda", requires_grad=True)
        (gx,) = torch.autograd.grad(fb.group_norm_autograd(x, 1), [x], torch.zeros_like(x))
        assert gx.shape == shape


@pytest.mark.parametrize("R", [60, 5000, 60000])
@pytest.mark.parametrize("where", [0, 0.3, 0.5, 1])
def test_one_value_far_from_the_others(where, R):
    """One position 1e5 spreads away, the first, middle and last one too: means lose no digits by it."""
    x, w, b, gy = make(2, R, 64, F32, F32, mean=0.0)
    x[:, int(where * (R - 1))] += 1e5
    stats = torch.empty((2, 8, 2), device="cuda")
    out = fb.group_norm_forward(x, 8, w, b, stats=stats)
    t = x.double().reshape(2, R, 8, 8)
    mean, var = t.mean((1, 3)), t.var((1, 3), correction=0)
    rstd = (var + 1e-5).rsqrt()
    # joins of some 16 roundings relative to the differences from a value among the others; rstd as in
    # check_all, where a join's d^2 has 2 d times the means' errors
    e_from = 16 * ref.U32 * (t - t.median(1, keepdim=True)[0][..., :1]).abs().mean((1, 3))
    assert ((stats[..., 0].double() - mean).abs() <= e_from + ref.U32 * mean.abs()).all()
    assert ((stats[..., 1].double() - rstd).abs() <= 40 * ref.U32 * rstd + rstd ** 2 * e_from).all()
    want = ref.group_norm(x.double(), 8, w.double(), b.double(), "none")
    wide = lambda s: s.repeat_interleave(8, -1)[:, None]   # noqa: E731
    # x - mean rounded once, relative to x; rstd's error and some 8 roundings of the factors relative to y
    xhat = (x.double() - wide(mean)) * wide(rstd)
    tol = w.double().abs() * (wide(rstd * (e_from + ref.U32 * mean.abs())) + 2 * ref.U32 * x.double().abs() * wide(rstd)
                              + xhat.abs() * (48 * ref.U32 + wide(rstd * e_from))) + 8 * ref.U32 * (want.abs() + b.double().abs())
    ref.check(out, want, tol + 1e-30, "y")


@pytest.mark.parametrize("dtype,pdt", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", [(1000, 49, 64, 8), (2500, 1, 96, 12), (300, 600, 33, 3)], ids=lambda s: "x".join(map(str, s)))
def test_many_samples(shape, dtype, pdt):
    """Region features and rows: weight's and bias's gradients are sums over all samples."""
    N, R, C, groups = shape
    x, w, b, gy = make(N, R, C, dtype, pdt, seed=4)
    check_all(x, groups, w, b, gy, "relu" if R > 1 else "gelu")
