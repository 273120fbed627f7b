"""Attention on the GPU against float64, within bounds counted from its roundings."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2607_10071_amd as fb

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
LOWEST = torch.finfo(F32).min


def make(B, Lq, Lk, H, Hk, D, dtype, seed=0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * Lq + 11 * Lk + D)
    return [(torch.randn(s, generator=g, device="cuda") * std).to(dtype)
            for s in ((B, Lq, H, D), (B, Lk, Hk, D), (B, Lk, Hk, D), (B, Lq, H, D))], g


def run_forward(q, k, v, **kw):
    stats = torch.full((q.shape[0], q.shape[2], q.shape[1], 2), 7.0, device="cuda")
    rest = torch.empty_like(q, memory_format=torch.contiguous_format)
    out = fb.attention_forward(q, k, v, stats=stats, rest=rest, **kw)
    return out, rest, stats


def check_all(q, k, v, g, scale=None, mask=None, key_lengths=None):
    """The forward, its statistics, and all gradients."""
    kw = dict(scale=scale, mask=mask, key_lengths=key_lengths)
    want, tol = ref.attention(q, k, v, scale, mask, key_lengths, g)
    out, rest, stats = run_forward(q, k, v, **kw)
    ref.check(out, want["out"], tol["out"], "out")
    # the statistics name the softmax's denominator
    s, size, _ = ref.scores(q, k, q.shape[-1] ** -0.5 if scale is None else scale, mask, key_lengths)
    if s.shape[-1]:
        lse = torch.logsumexp(s, -1)
        empty = lse == -math.inf
        assert ((stats[..., 0] == -math.inf) == empty).all()
        near = (stats.double().sum(-1) - lse).abs()[~empty]
        lim = (size.amax(-1) * (q.shape[-1] + 8) * 2 * ref.U32 + lse.abs() * 2 ** -22 + ref.half(q.dtype) + 1e-5)[~empty]
        assert (near <= lim).all(), (near - lim).max()
    r = fb.attention_backward(g, q, k, v, out, stats, rest=rest if q.dtype != F32 else None, **kw)
    for n in "qkv":
        ref.check(r[n], want["grad_" + n], tol["grad_" + n], "grad_" + n)
    return out, r


SHAPES = [
    # B, Lq, Lk, H, Hk, D
    (1, 1, 1, 1, 1, 32), (2, 1, 129, 4, 4, 64), (2, 1, 1000, 8, 2, 128), (1, 5, 33, 3, 3, 1),
    (1, 33, 64, 2, 2, 32), (2, 70, 65, 4, 2, 64), (1, 128, 128, 2, 1, 96), (1, 200, 300, 3, 3, 128),
    (3, 77, 133, 6, 2, 72), (1, 129, 257, 2, 2, 33), (1, 31, 511, 5, 1, 17), (1, 300, 31, 2, 2, 8),
    (1, 17, 2100, 2, 2, 40), (1, 2100, 40, 1, 1, 32), (2, 64, 640, 4, 4, 100), (1, 3, 700, 9, 3, 127),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(shape, dtype):
    (q, k, v, g), _ = make(*shape, dtype)
    check_all(q, k, v, g)


def masks(kind, B, H, Lq, Lk, dtype, g):
    """(mask, key lengths)"""
    def rand(*s):
        return torch.rand(s, generator=g, device="cuda")

    if kind == "lengths":
        lens = (rand(B) * (Lk + 1)).int()
        lens[0] = 0
        return None, lens
    if kind == "keys":
        return rand(B, 1, 1, Lk) < 0.6, None
    if kind == "keys_of_heads":
        return rand(1, H, 1, Lk) < 0.6, None
    if kind == "pairs":
        return (rand(B, 1, Lq, Lk) < 0.5) & (rand(B, 1, Lq, 1) < 0.8), None
    if kind == "all":
        return (rand(B, H, Lq, Lk) < 0.5) & (rand(B, H, Lq, 1) < 0.8), (rand(B) * (Lk + 1)).int()
    if kind == "nothing":
        return torch.zeros((1, 1, 1, Lk), dtype=torch.bool, device="cuda"), None
    add = 2 * torch.randn((1, H, Lq, Lk), generator=g, device="cuda")
    if kind == "inf":
        add = add.masked_fill(rand(1, H, Lq, Lk) < 0.3, -math.inf).masked_fill(rand(1, 1, Lq, 1) < 0.2, -math.inf)
    if kind == "lowest":
        add = add.masked_fill(rand(1, H, Lq, Lk) < 0.3, LOWEST).masked_fill(rand(1, 1, Lq, 1) < 0.2, LOWEST)
    if kind == "of_type":
        low = torch.finfo(dtype).min
        add = add.to(dtype).masked_fill(rand(1, H, Lq, Lk) < 0.3, low).masked_fill(rand(1, 1, Lq, 1) < 0.2, low)
    return add, None


@pytest.mark.parametrize("kind", ["lengths", "keys", "keys_of_heads", "pairs", "all", "nothing", "add", "inf", "lowest",
                                  "of_type"])
@pytest.mark.parametrize("shape", [(2, 40, 150, 4, 2, 32), (3, 1, 777, 6, 3, 72), (2, 131, 97, 2, 2, 128),
                                   (1, 20, 1100, 2, 2, 37), (1, 70, 2500, 2, 1, 41)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_masks(shape, kind, dtype):
    (q, k, v, g), gen = make(*shape, dtype, seed=3)
    mask, lengths = masks(kind, shape[0], shape[3], shape[1], shape[2], dtype, gen)
    check_all(q, k, v, g, mask=mask, key_lengths=lengths)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_left_out_keys_may_hold_anything(dtype):
    (q, k, v, g), gen = make(2, 37, 200, 4, 2, 48, dtype)
    lengths = torch.tensor([130, 77], dtype=torch.int32, device="cuda")
    mask = torch.rand((2, 1, 1, 200), generator=gen, device="cuda") < 0.7
    clean = check_all(q, k, v, g, mask=mask, key_lengths=lengths)
    gone = ~mask[:, 0, 0] | (torch.arange(200, device="cuda") >= lengths[:, None])
    for bad in (math.nan, math.inf, -math.inf):
        kb, vb = k.clone(), v.clone()
        kb[gone], vb[gone] = bad, bad
        out, rest, stats = run_forward(q, kb, vb, mask=mask, key_lengths=lengths)
        assert torch.equal(out, clean[0])
        r = fb.attention_backward(g, q, kb, vb, out, stats, mask, lengths, rest=rest if dtype != F32 else None)
        for n in "qkv":
            assert torch.equal(r[n], clean[1][n]), n
        assert (r["k"][gone] == 0).all() and (r["v"][gone] == 0).all()


def test_lengths_outside_the_keys_are_taken_as_within():
    (q, k, v, g), _ = make(2, 9, 100, 2, 2, 32, BF16)
    got = fb.attention_forward(q, k, v, key_lengths=torch.tensor([-5, 1 << 30], dtype=torch.int32, device="cuda"))
    assert (got[0] == 0).all()
    assert torch.equal(got[1], fb.attention_forward(q, k, v)[1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("std,scale", [(6.0, None), (1.0, 4.0), (1e-3, None), (1.0, 1e-20)])
def test_large_and_small_scores(dtype, std, scale):
    (q, k, v, g), _ = make(1, 70, 333, 2, 2, 64, dtype, std=std)
    check_all(q, k, v, g, scale=scale)


@pytest.mark.parametrize("lq", [20, 150])
def test_growing_scores(lq):
    """Every tile's scores pass those before it: the references move all the way."""
    (q, k, v, g), _ = make(1, lq, 1500, 2, 2, 32, BF16)
    q = q.abs()
    k = (k.abs() * torch.linspace(0, 4, 1500, device="cuda")[None, :, None, None]).to(BF16)
    check_all(q, k, v, g)
    check_all(q, k.flip(1).contiguous(), v, g)


def test_small_float16_gradients_keep_their_digits():
    """Weights of one in 20000 and gradients of 1e-3: below float16's normal numbers unscaled."""
    (q, k, v, g), _ = make(1, 64, 20000, 1, 1, 32, F16, std=0.1)
    g = (g * 1e-2).to(F16)
    out, rest, stats = run_forward(q, k, v)
    r = fb.attention_backward(g, q, k, v, out, stats, rest=rest)
    d = [t.double().squeeze(0).squeeze(1).requires_grad_() for t in (q, k, v)]
    o = torch.softmax(d[0] @ d[1].t() * 32 ** -0.5, -1) @ d[2]
    want = torch.autograd.grad(o, d, g.double().squeeze(0).squeeze(1))
    for n, w in zip("qkv", want):
        got = r[n].double().squeeze(0).squeeze(1)
        # what float16 holds of the result itself: a step of 2^-24, and its relative half step;
        # the sums' terms are rounded to relative 2^-11 (weights, dS), a root-mean-square sum of them
        assert ((got - w).norm() <= 4 * 2 ** -11 * w.norm() + 2 ** -24 * w.numel() ** 0.5), n


def test_strides():
    """Heads of one projection, a cache longer than what is read, transposed heads, an expanded batch."""
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((2, 90, 3, 4, 32), generator=g, device="cuda").to(BF16)
    q, k, v = qkv.unbind(2)
    check_all(q, k, v, torch.randn(q.shape, generator=g, device="cuda").to(BF16))
    cache = torch.randn((2, 4, 500, 64), generator=g, device="cuda").to(F16)   # heads before positions
    k = cache.transpose(1, 2)[:, :333]
    v = cache.flip(2).transpose(1, 2)[:, :333]
    q = torch.randn((2, 4, 50, 64), generator=g, device="cuda").to(F16).transpose(1, 2)
    go = torch.randn((2, 4, 50, 64), generator=g, device="cuda").to(F16).transpose(1, 2)
    check_all(q, k, v, go)
    k1 = torch.randn((1, 70, 2, 24), generator=g, device="cuda").expand(3, -1, -1, -1)
    q3 = torch.randn((3, 40, 4, 24), generator=g, device="cuda")
    check_all(q3, k1, k1.flip(1), torch.randn(q3.shape, generator=g, device="cuda"))
    # odd addresses: 16-bit elements at any of them
    flat = torch.randn(4 * 60 * 2 * 20 + 3, generator=g, device="cuda").to(BF16)
    q, k, v, go = (flat[i:i + 60 * 2 * 20].view(1, 60, 2, 20) for i in (1, 2401, 3, 2402))
    check_all(q, k, v, go)


def test_out_in_place_of_a_larger_tensor():
    (q, k, v, _), _ = make(2, 33, 70, 4, 2, 40, BF16)
    big = torch.full((2, 33, 5, 4, 40), 3.0, dtype=BF16, device="cuda")
    fb.attention_forward(q, k, v, out=big[:, :, 2])
    assert torch.equal(big[:, :, 2], fb.attention_forward(q, k, v))
    big[:, :, 2] = 3.0
    assert (big == 3.0).all()


def test_masks_by_stride():
    (q, k, v, g), gen = make(2, 40, 130, 4, 2, 32, F32)
    wide = torch.randn((2, 1, 64, 200), generator=gen, device="cuda")
    view = wide[:, :, 3:43, 11:141]
    a, b = fb.attention_forward(q, k, v, mask=view), fb.attention_forward(q, k, v, mask=view.contiguous())
    assert torch.equal(a, b)
    check_all(q, k, v, g, mask=view.expand(2, 4, 40, 130))
    check_all(q, k, v, g, mask=(view > 0)[:1])


def test_empty():
    z = torch.zeros
    q, k = z((2, 3, 4, 32), device="cuda", dtype=BF16), z((2, 0, 2, 32), device="cuda", dtype=BF16)
    stats = z((2, 4, 3, 2), device="cuda")
    out = fb.attention_forward(q + 1, k, k, stats=stats)
    assert (out == 0).all() and (stats[..., 0] == -math.inf).all() and (stats[..., 1] == 0).all()
    r = fb.attention_backward(q + 1, q + 1, k, k, out, stats)
    assert (r["q"] == 0).all() and r["k"].shape == k.shape
    q0 = q[:, :0]
    k = z((2, 5, 2, 32), device="cuda", dtype=BF16) + 1
    out = fb.attention_forward(q0, k, k)
    r = fb.attention_backward(q0, q0, k, k, out.contiguous(), z((2, 4, 0, 2), device="cuda"))
    assert out.shape == q0.shape and (r["k"] == 0).all() and (r["v"] == 0).all()
    assert fb.attention_forward(q[:0], k[:0], k[:0]).shape == (0, 3, 4, 32)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_autograd(dtype):
    (q, k, v, g), gen = make(2, 60, 150, 4, 2, 40, dtype)
    lengths = torch.tensor([150, 61], dtype=torch.int32, device="cuda")
    mask = torch.randn((1, 4, 60, 150), generator=gen, device="cuda")
    want, tol = ref.attention(q, k, v, None, mask, lengths, g)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out = fb.attention_autograd(*leaves, mask=mask, key_lengths=lengths)
    got = torch.autograd.grad(out, leaves, g)
    for n, t in zip("qkv", got):
        ref.check(t, want["grad_" + n], tol["grad_" + n], n)
    # some of them, with another gradient's strides
    out = fb.attention_autograd(q, leaves[1], v, mask=mask, key_lengths=lengths)
    (gk,) = torch.autograd.grad(out, [leaves[1]], g.transpose(1, 3).contiguous().transpose(1, 3))
    assert torch.equal(gk, got[1])
    with torch.no_grad():
        assert torch.equal(fb.attention_autograd(*leaves, mask=mask, key_lengths=lengths), out.detach())


def test_one_state_has_no_gradient_through_its_weight():
    (q, k, v, g), _ = make(2, 40, 1, 2, 2, 32, BF16)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out = fb.attention_autograd(*leaves)
    gq, gk, gv = torch.autograd.grad(out, leaves, g)
    assert torch.equal(out, v.expand_as(q))
    # dP and delta are the same sum in two orders: 32 products of float32
    size = (g.double().abs() * v.double().abs()).sum(-1)
    assert (gq.double().abs() <= 40 * ref.U32 * (size * 32 ** -0.5)[..., None] * k.double().abs() * 1.01 + 1e-30).all()


def test_gradient_against_differences():
    (q, k, v, g), _ = make(1, 7, 50, 2, 1, 16, F32)
    leaves = [t.requires_grad_() for t in (q, k, v)]
    grads = torch.autograd.grad(fb.attention_autograd(*leaves), leaves, g)
    def loss(q, k, v):
        k, v = (t.repeat_interleave(2, 2) for t in (k, v))
        p = torch.softmax(torch.einsum("bihd,bjhd->bhij", q, k) * 16 ** -0.5, -1)
        return (torch.einsum("bhij,bjhd->bihd", p, v) * g.double()).sum()

    for i, gr in enumerate(grads):
        step = torch.randn(gr.shape, device="cuda", dtype=torch.float64)
        ends = []
        for e in (1e-4, -1e-4):
            moved = [x.detach().double() for x in leaves]
            moved[i] = moved[i] + e * step
            ends.append(loss(*moved))
        slope = (ends[0] - ends[1]) / 2e-4
        # differences are off by third derivatives times 1e-8, the gradient by float32's digits
        assert abs(slope - (gr.double() * step).sum()) < 1e-5 * (1 + (gr.double() * step).abs().sum()), i


def test_same_bits_again_and_on_another_stream():
    (q, k, v, g), _ = make(2, 300, 900, 4, 2, 64, BF16)
    first = [t.clone() for t in run_forward(q, k, v)]
    grads = fb.attention_backward(g, q, k, v, first[0], first[2], rest=first[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run_forward(q, k, v)
        more = fb.attention_backward(g, q, k, v, first[0], first[2], rest=first[1])
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert all(torch.equal(grads[n], more[n]) for n in "qkv")
    out = torch.empty_like(q)
    call = fb.prepare_attention_forward(q, k, v, out=out)
    call()
    call()
    assert torch.equal(out, first[0])


@pytest.mark.parametrize("lq", [1, 150])
def test_a_long_cache(lq):
    """Rows and batches further into a cache than 32 bits reach, in elements too."""
    B, Lk, row = 2, 2300, 1 << 20
    cache = torch.empty(B * Lk * row, dtype=F16, device="cuda")   # 9.6 GB, of which 64 channels a row
    k = cache.as_strided((B, Lk, 1, 64), (Lk * row, row, 64, 1))
    v = cache.as_strided((B, Lk, 1, 64), (Lk * row, row, 64, 1), 128)
    assert k.stride(0) + (Lk - 1) * row > 1 << 32
    (q, k0, v0, g), _ = make(B, lq, Lk, 1, 1, 64, F16)
    k.copy_(k0)
    v.copy_(v0)
    n = torch.tensor([Lk, Lk - 100], dtype=torch.int32, device="cuda")
    stats, stats0 = (torch.empty((B, 1, lq, 2), device="cuda") for _ in range(2))
    out = fb.attention_forward(q, k, v, key_lengths=n, stats=stats)
    out0 = fb.attention_forward(q, k0, v0, key_lengths=n, stats=stats0)
    assert torch.equal(out, out0) and torch.equal(stats, stats0)
    r = fb.attention_backward(g, q, k, v, out, stats, key_lengths=n)
    r0 = fb.attention_backward(g, q, k0, v0, out, stats, key_lengths=n)
    assert all(torch.equal(r[c], r0[c]) for c in "qkv")
    check_all(q, k0, v0, g, key_lengths=n)


@pytest.mark.parametrize("where", ["q", "k", "v"])
def test_nan_stays_in_its_row_or_column(where):
    """What is no number reaches the rows that read it, and no others."""
    (q, k, v, g), _ = make(2, 70, 300, 4, 2, 64, BF16)
    (q if where == "q" else k if where == "k" else v)[1, 5, 0 if where != "q" else 3, 7] = math.nan
    out, _, _ = run_forward(q, k, v)
    bad = torch.isnan(out)
    if where == "q":
        assert bad[1, 5, 3].all() and bad.sum() == 64
    elif where == "k":
        assert bad[1, :, :2].all() and bad.sum() == 70 * 2 * 64
    else:
        assert bad[1, :, :2, 7].all() and bad.sum() == 70 * 2


@pytest.mark.parametrize("what", ["rows", "heads", "share"])
def test_far_rows_and_heads(what):
    """Rows and query heads further apart than the library takes are read from a copy, also on another
    stream and as gradients; outputs and prepared calls are refused.  Single rows have no step."""
    # (the third: heads within the limit, 512 of which are not)
    H, Hk, far = (2, 2, (1 << 20) + 8) if what != "share" else (512, 1, (1 << 20) - 8)
    (q0, k0, v0, g0), _ = make(1, 40, 50, H, Hk, 32, BF16)

    def apart(t):
        n, h = t.shape[1], t.shape[2]
        step, head = (far, 32) if what == "rows" else (32, far)
        view = torch.empty((n - 1) * step + (h - 1) * head + 32, dtype=BF16, device="cuda").as_strided(
            t.shape, (0, step, head, 1))
        view.copy_(t)
        return view

    q, k, v, g = map(apart, (q0, k0, v0, g0))
    stats, stats0 = (torch.empty((1, H, 40, 2), device="cuda") for _ in range(2))
    out0 = fb.attention_forward(q0, k0, v0, stats=stats0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = fb.attention_forward(q, k, v, stats=stats, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, out0) and torch.equal(stats, stats0)
    r, r0 = (fb.attention_backward(*a, out, stats) for a in ((g, q, k, v), (g0, q0, k0, v0)))
    assert all(torch.equal(r[n], r0[n]) for n in "qkv")
    with pytest.raises(ValueError, match="prepared call"):
        fb.prepare_attention_forward(q, k, v, out=out)
    with pytest.raises(fb.FlashBevError):
        fb.attention_forward(q0, k0, v0, out=q)
    leaves = [t.requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(fb.attention_autograd(*leaves), leaves, g)
    want = torch.autograd.grad(fb.attention_autograd(*[t.requires_grad_() for t in (q0, k0, v0)]), [q0, k0, v0], g0)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # one row of a tensor whose rows are far apart is not far from anything
    one = q.detach()[:, :1]
    assert torch.equal(fb.attention_forward(one, k0, v0), fb.attention_forward(q0[:, :1].contiguous(), k0, v0))


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [32, 31, 128])
def test_gradients_without_queries(D, dtype):
    """Zeros for k and v, whatever the mask of no queries."""
    q = torch.ones((2, 0, 4, D), device="cuda", dtype=dtype)
    k = torch.ones((2, 150, 2, D), device="cuda", dtype=dtype)
    for mask in (None, torch.ones((2, 1, 0, 150), device="cuda", dtype=torch.bool),
                 torch.ones((1, 4, 0, 150), device="cuda", dtype=torch.bool),
                 torch.ones((2, 1, 1, 150), device="cuda", dtype=torch.bool),
                 torch.ones((2, 4, 0, 150), device="cuda")):
        leaves = [t.clone().requires_grad_() for t in (q, k, k)]
        out = fb.attention_autograd(*leaves, mask=mask)
        del_me = [torch.full_like(k, math.nan) for _ in range(4)]   # (what the gradients' memory may hold)
        del del_me
        got = torch.autograd.grad(out, leaves, torch.empty_like(q))
        assert out.shape == q.shape and got[0].shape == q.shape
        assert got[1].shape == got[2].shape == k.shape and (got[1] == 0).all() and (got[2] == 0).all()


def off_16_bytes(t, how):
    """t's values at addresses that are not multiples of 16 bytes: all of them, those of odd rows, of odd
    heads, or of odd batches."""
    B, L, H, D = t.shape
    head = D + (how == "heads")
    row = H * head + (how == "rows")
    batch = L * row + (how == "batches")
    flat = torch.zeros(B * batch + 1, dtype=t.dtype, device="cuda")
    view = flat.as_strided(t.shape, (batch, row, head, 1), 1 if how == "all" else 0)
    view.copy_(t)
    assert view.data_ptr() % 16 or any(s * t.element_size() % 16 for s in view.stride()[:3])
    return view


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(2, 70, 333, 4, 2, 32), (2, 130, 200, 2, 2, 64), (2, 60, 150, 4, 2, 128),
                                   (2, 5, 300, 2, 2, 64), (2, 45, 2100, 2, 1, 96)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("how", ["all", "rows", "heads", "batches"])
@pytest.mark.parametrize("which", ["q", "k", "v", "g", "qkvg"])
def test_rows_off_16_bytes(which, how, shape, dtype):
    """Elements of any alignment where loads to LDS take 16 bytes at multiples of them, with and without
    keys that a mask leaves out."""
    ts, gen = make(*shape, dtype, seed=8)
    moved = [off_16_bytes(t, how) if n in which else t for n, t in zip("qkvg", ts)]
    for mask in (None, torch.rand((2, 1, 1, shape[2]), generator=gen, device="cuda") < 0.7):
        check_all(*moved, mask=mask)
    (q, k, v, g), lengths = moved, torch.tensor([shape[2], shape[2] // 3], dtype=torch.int32, device="cuda")
    check_all(q, k, v, g, key_lengths=lengths)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(fb.attention_autograd(*leaves), leaves, g)
    want, tol = ref.attention(*ts[:3], None, None, None, g)
    for n, t in zip("qkv", got):
        ref.check(t, want["grad_" + n], tol["grad_" + n], "grad_" + n)


def backward_checked(q, k, v, g, mask=None, key_lengths=None, more=None):
    """All gradients within their bounds (``more``: what to add to them)."""
    kw = dict(mask=mask, key_lengths=key_lengths)
    want, tol = ref.attention(q, k, v, None, mask, key_lengths, g)
    out, rest, stats = run_forward(q, k, v, **kw)
    ref.check(out, want["out"], tol["out"], "out")
    r = fb.attention_backward(g, q, k, v, out, stats, rest=rest if q.dtype != F32 else None, **kw)
    for n in "qkv":
        ref.check(r[n], want["grad_" + n], tol["grad_" + n] + (more or {}).get(n, 0.0), "grad_" + n)
    return r


def some_masks(B, H, Lq, Lk, gen):
    def rand(*s):
        return torch.rand(s, generator=gen, device="cuda")

    return {"none": None, "keys": rand(B, 1, 1, Lk) < 0.7, "pairs": rand(B, 1, Lq, Lk) < 0.6,
            "add": 2 * torch.randn((1, H, Lq, Lk), generator=gen, device="cuda")}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [1e20, 3e30, 1e-25])
@pytest.mark.parametrize("kind", ["none", "keys", "pairs", "add"])
@pytest.mark.parametrize("D", [32, 64, 63, 128])
def test_gradients_whose_squares_leave_float32(D, kind, size, dtype):
    """Rows of grad_out with norms that float32 cannot square, next to ordinary ones."""
    (q, k, v, g), gen = make(2, 70, 150, 4, 2, D, dtype, seed=9)
    g[:, ::2] = (g[:, ::2].float() * size).to(dtype)
    backward_checked(q, k, v, g, some_masks(2, 4, 70, 150, gen)[kind])


def test_gradients_of_many_problems():
    """More tiles of 16 rows than one row of the grid takes, the last ones too."""
    B, Lq, Lk, D = (1 << 21) + 3, 1, 2, 8
    (q, k, v, g), _ = make(B, Lq, Lk, 1, 1, D, BF16)
    out, rest, stats = run_forward(q, k, v)
    r = fb.attention_backward(g, q, k, v, out, stats, rest=rest)
    for b in (0, 1 << 18, 1 << 20, (1 << 21) - 1, B - 2):
        s = slice(b, b + 2)
        want, tol = ref.attention(q[s], k[s], v[s], grad_out=g[s])
        ref.check(out[s], want["out"], tol["out"], "out")
        for n in "qkv":
            ref.check(r[n][s], want["grad_" + n], tol["grad_" + n], "grad_" + n)
    del out, rest, stats, r
    torch.cuda.empty_cache()


def spread_of(v):
    """The power of two that float16's dS loses for the largest row of v: 1 up to 2048 (the most of weights
    of 2^6 and twice |v| over 8 is then 2^15), and as much more as that row passes it."""
    most = v.detach().double().square().sum(-1).sqrt().amax().item()
    return 2.0 ** max(0, math.ceil(math.log2(most)) - 11)


def more_of(q, k, v, g):
    """What float16's steps below its normal numbers add where dS is made smaller by ``spread_of``, per unit
    of the bounds' own terms (with weights of one): n steps of 2^-25 of 8 |g|, rows of 16."""
    d, share = q.shape[-1] ** -0.5 * 2.0 ** -25 * spread_of(v), q.shape[2] // k.shape[2]
    norm = g.double().square().sum(-1).sqrt()
    return {"q": d * k.shape[1] * 8 * norm[..., None] * k.double().abs().amax(),
            "k": d * q.shape[1] * share * 16 * norm.amax() * q.double().abs().amax()}


@pytest.mark.parametrize("size", [300.0, 2000.0, 60000.0])
@pytest.mark.parametrize("kind", ["none", "lengths", "keys", "pairs", "add"])
@pytest.mark.parametrize("shape", [(2, 70, 333, 4, 2, 32), (1, 150, 333, 2, 2, 64), (2, 5, 700, 4, 2, 63), (1, 130, 400, 2, 1, 128),
                                   (1, 40, 2500, 2, 2, 96)], ids=lambda s: "x".join(map(str, s)))
def test_large_values_in_float16(shape, kind, size):
    """Values up to float16's largest: dS, of which the forward's reference may leave weights of 2^6, stays
    within float16."""
    B, Lq, Lk, H, Hk, D = shape
    (q, k, v, g), gen = make(*shape, F16, seed=10)
    # (values and gradients along one direction of each head: their products are as large as they get)
    u = torch.where(torch.rand((Hk, D), generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    v = (v.float() * 0.01 + torch.rand((B, Lk, Hk, 1), generator=gen, device="cuda") * 2 - 1).mul(u).mul(size / 1.1).to(F16)
    g = ((g.float() * 0.1 + 1) * u.repeat_interleave(H // Hk, 0) * 3 / size).to(F16)
    # scores that grow by a few units behind the first keys, which the references follow late
    q, k = (q.float().abs() * 0.5).to(F16), (k.float() * 0.3 + torch.linspace(0, 1.0, Lk, device="cuda")[None, :, None, None]).to(F16)
    mask = some_masks(B, H, Lq, Lk, gen).get(kind)
    lengths = torch.tensor([Lk, Lk // 2][:B], dtype=torch.int32, device="cuda") if kind == "lengths" else None
    r = backward_checked(q, k, v, g, mask, lengths, more_of(q, k, v, g))
    if kind in ("lengths", "keys"):   # keys that are left out have no say in it
        gone = ~mask[:, 0, 0] if mask is not None else torch.arange(Lk, device="cuda") >= lengths[:, None]
        for bad in (math.nan, math.inf, -65504.0):
            kb, vb = k.clone(), v.clone()
            kb[gone], vb[gone] = bad, bad
            out, rest, stats = run_forward(q, kb, vb, mask=mask, key_lengths=lengths)
            again = fb.attention_backward(g, q, kb, vb, out, stats, mask, lengths, rest=rest)
            assert all(torch.equal(r[n], again[n]) for n in "qkv")


def test_one_score_above_the_first_keys():
    """float16, v of 30000: a weight of 2^5.5 above its reference, whose dS was infinite."""
    q, k = torch.zeros((1, 64, 1, 32), device="cuda", dtype=F16), torch.zeros((1, 333, 1, 32), device="cuda", dtype=F16)
    v, g = torch.zeros_like(k), torch.zeros_like(q)
    q[..., 0], k[:, 200, :, 0] = 4.0, 3.8 * 32 ** 0.5 / 4.0
    v[..., 1], v[:, 200, :, 1] = -30000.0, 30000.0
    g[..., 1] = 0.01
    backward_checked(q, k, v, g, more=more_of(q, k, v, g))


@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("kind", ["inf", "pairs"])
def test_large_values_behind_masks_of_rows_in_float16(kind, D):
    """Keys that an added mask, or one for each row, leaves out for all rows: their values take nothing from the
    other keys' gradients."""
    (q, k, v, g), gen = make(2, 90, 300, 4, 2, D, F16, seed=11)
    gone = torch.rand((2, 1, 1, 300), generator=gen, device="cuda") < 0.3
    mask = torch.zeros((2, 1, 90, 300), device="cuda").masked_fill(gone, -math.inf)
    if kind == "pairs":
        mask = mask == 0
    far = v.clone()
    far[gone[:, 0, 0]] = 60000.0
    clean = backward_checked(q, k, v, g, mask)
    r = backward_checked(q, k, far, g, mask, more=more_of(q, k, far, g))
    assert torch.equal(r["k"], clean["k"]) and torch.equal(r["v"], clean["v"])
