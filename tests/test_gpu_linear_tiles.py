"""The linear operator's kernels of large tiles against float64, at sizes that no tile
divides (``linear_plan`` says which kernel each takes).

Two kinds of comparison.  Products of small whole numbers are exact in float32 in any order
(sums below 2^24), so the result is the exact one rounded once, to the bit, and any element
that is lost, doubled or misplaced shows.  Activations of random products are held to the
bounds of ``block_ref``."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

import block_ref as ref  # noqa: E402
from linear_plan import BACKWARD, FORWARD  # noqa: E402

TYPES = [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32")]


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


def whole(gen, *shape, dtype, most=2):
    """Whole numbers of -most to most."""
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").to(dtype)


def close(got, want, err):
    """``ref.close`` on the device."""
    lim = err + ref.u(got.dtype) * (want.abs() + err) + ref.tiny(got.dtype)
    off = (got.double() - want).abs()
    assert (off <= lim).all(), f"worst {float((off / lim).max()):.3g} times the bound"


def inside(t, gen):
    """t's values in rows of a wider tensor at an odd place, numbers around them."""
    big = whole(gen, t.shape[0] + 2, t.shape[1] + 24, dtype=t.dtype)
    view = big[1:-1, 8:8 + t.shape[1]]
    view.copy_(t)
    return big, view


def untouched(big, before, N):
    keep = torch.ones_like(big, dtype=torch.bool)
    keep[1:-1, 8:8 + N] = False
    return torch.equal(big[keep], before[keep])


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("size", [f[0] for f in FORWARD], ids=str)
def test_forward_exact(fb, device, size, types):
    """out, pre and the residual in place, at most 2 * 2 * 2056 + 2 in magnitude."""
    M, K, N = size
    dt, odt = (ref.DTYPES[t] for t in types)
    gen = torch.Generator(device=device).manual_seed(M + N)
    x, w, b = (whole(gen, *s, dtype=dt) for s in ((M, K), (N, K), (N,)))
    pre = x.double() @ w.double().t() + b.double()
    r = whole(gen, M, N, dtype=odt, most=8)
    assert torch.equal(fb.linear_forward(x, w, b, residual=r, scale=0.5, out_dtype=odt),
                       (r.double() + 0.5 * pre).to(odt))
    assert torch.equal(fb.linear_forward(x, w, out_dtype=odt), (pre - b.double()).to(odt))
    # in place, between rows of a wider tensor that stay as they are
    big, into = inside(r, gen)
    pbig, p = inside(r.to(dt), gen)
    before, pbefore = big.clone(), pbig.clone()
    got = fb.linear_forward(x, w, b, "relu", into, -1.0, out=into, pre=p)
    assert got is into and torch.equal(into, (r.double() - pre.clamp(min=0)).to(odt))
    assert torch.equal(p, pre.to(dt))
    assert untouched(big, before, N) and untouched(pbig, pbefore, N)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("size", [f[0] for f in FORWARD if f[0][1] <= 200], ids=str)
def test_forward_activations(fb, device, size, act, types):
    M, K, N = size
    dt, odt = (ref.DTYPES[t] for t in types)
    gen = torch.Generator(device=device).manual_seed(M + N)
    rand = lambda *s: torch.randn(s, generator=gen, device=device)
    x, w, b = rand(M, K).to(dt), (rand(N, K) * (2 * K ** -0.5)).to(dt), rand(N).to(dt)
    r = rand(M, N).to(odt)
    for bias, residual, scale in ((b, r, 0.75), (None, None, 1.0)):
        want, pre, e, e_pre = ref.linear(x, w, bias, act, residual, scale)
        p = torch.empty(M, N, dtype=dt, device=device)
        close(fb.linear_forward(x, w, bias, act, residual, scale, out_dtype=odt, pre=p), want, e)
        close(p, pre, e_pre)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("size", [b[0] for b in BACKWARD], ids=str)
def test_backward_exact(fb, device, size, types):
    """Sums of at most 40001 products of at most 4 in magnitude; the float16 ones stay
    below 65504 (40001 random terms add up to some hundreds).  With relu d is 0 or grad_out."""
    M, K, N = size
    dt, odt = (ref.DTYPES[t] for t in types)
    gen = torch.Generator(device=device).manual_seed(M + N)
    x, w = whole(gen, M, K, dtype=dt), whole(gen, N, K, dtype=dt)
    g, pre = whole(gen, M, N, dtype=odt), whole(gen, M, N, dtype=dt)
    for act in ("none", "relu"):
        d = g.double() * (pre > 0) if act == "relu" else g.double()
        want = {"x": d @ w.double(), "weight": d.t() @ x.double(), "bias": d.sum(0)}
        got = fb.linear_backward(g, x, w, pre, act, 0.5)
        for k in want:
            assert torch.equal(got[k], (0.5 * want[k]).to(dt)), (act, k)
    # gradients into rows of wider tensors, which stay as they are around them
    big, gx = inside(torch.zeros_like(x), gen)
    wbig, gw = inside(torch.zeros_like(w), gen)
    before, wbefore = big.clone(), wbig.clone()
    fb.linear_backward(g, x, w, pre, "relu", 0.5, want=(), grad_x=gx, grad_weight=gw)
    assert torch.equal(gx, got["x"]) and torch.equal(gw, got["weight"])
    assert untouched(big, before, K) and untouched(wbig, wbefore, K)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(40001, 520, 72), (40001, 2056, 200), (9001, 1032, 72), (200, 2056, 4099)],
                         ids=str)
def test_places_that_are_no_multiple_of_16_bytes(fb, device, size, dtype):
    """Plans of 128 and 256 tiles at addresses and strides that the streamed kernels do not
    take: all three products, to the bit."""
    M, K, N = size
    dt = ref.DTYPES[dtype]
    gen = torch.Generator(device=device).manual_seed(M + K)

    def odd(rows, cols, most=2):
        return whole(gen, rows, cols + 3, dtype=dt, most=most)[:, 1:cols + 1]

    x, w, g = odd(M, K), odd(N, K), odd(M, N)
    xd, wd, gd = x.double(), w.double(), g.double()
    assert torch.equal(fb.linear_forward(x, w), (xd @ wd.t()).to(dt))
    got = fb.linear_backward(g, x, w)
    assert torch.equal(got["x"], (gd @ wd).to(dt)) and torch.equal(got["weight"], (gd.t() @ xd).to(dt))
    assert torch.equal(got["bias"], gd.sum(0).to(dt))


def test_input_gradients_past_32_bits(fb, device):
    """grad_out and grad_x past 2^32 bytes."""
    M, K, N = (1 << 23) + 5, 320, 264
    gen = torch.Generator(device=device).manual_seed(2)
    g = torch.zeros(M, N, dtype=torch.bfloat16, device=device)
    g[-5:] = whole(gen, 5, N, dtype=torch.bfloat16)
    w = whole(gen, N, K, dtype=torch.bfloat16)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=device)
    got = fb.linear_backward(g, x, w, want=("x",))["x"]
    assert torch.equal(got[-5:], (g[-5:].double() @ w.double()).to(torch.bfloat16))
    assert (got[:-5] == 0).all()


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("K,N", [(64, 64), (1032, 200), (4096, 64), (8192, 1000), (8200, 33), (4099, 70), (2048, 4099)])
@pytest.mark.parametrize("M", [1, 2, 16, 17, 32, 33])
def test_few_rows_exact(fb, device, M, K, N, types):
    """On both sides of the rule that sends up to 32 rows to one pass over the weight or to
    tiles; sums of at most 8200 products of at most 4 in magnitude."""
    dt, odt = (ref.DTYPES[t] for t in types)
    gen = torch.Generator(device=device).manual_seed(M + N)
    x, w, b = (whole(gen, *s, dtype=dt) for s in ((M, K), (N, K), (N,)))
    pre = x.double() @ w.double().t() + b.double()
    r = whole(gen, M, N, dtype=odt, most=8)
    big, into = inside(r, gen)
    before = big.clone()
    p = torch.empty(M, N, dtype=dt, device=device)
    assert fb.linear_forward(x, w, b, "relu", into, 0.5, out=into, pre=p) is into
    assert torch.equal(into, (r.double() + 0.5 * pre.clamp(min=0)).to(odt))
    assert torch.equal(p, pre.to(dt)) and untouched(big, before, N)
