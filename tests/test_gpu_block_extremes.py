"""The encoder block's operators at the ends of what they take: the widest rows, the largest
row stride, thousands of samples, inputs below the normal numbers."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

import block_ref as ref  # noqa: E402
import test_gpu_norm as tn  # noqa: E402

WIDE = 1 << 18   # FLASHBLOCK_WIDTH_MAX
FAR = 1 << 20    # FLASHBLOCK_LD_MAX


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


def whole(gen, *shape, dtype, most=2):
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(3, WIDE, 5), (20, WIDE - 1, 24), (40, WIDE, 9), (40, WIDE - 3, 8),
                                   (3, 8, WIDE), (70, 16, WIDE), (70, 9, WIDE - 1)])
def test_widest_rows(fb, device, M, K, N, dtype):
    """Whole numbers: sums of at most 2^18 products of at most 4 are exact."""
    dt = ref.DTYPES[dtype]
    gen = torch.Generator(device=device).manual_seed(M)
    x, w, g = (whole(gen, *s, dtype=dt) for s in ((M, K), (N, K), (M, N)))
    xd, wd, gd = x.double(), w.double(), g.double()
    assert torch.equal(fb.linear_forward(x, w), (xd @ wd.t()).to(dt))
    got = fb.linear_backward(g, x, w)
    assert torch.equal(got["x"], (gd @ wd).to(dt)) and torch.equal(got["weight"], (gd.t() @ xd).to(dt))
    assert torch.equal(got["bias"], gd.sum(0).to(dt))
    with pytest.raises(fb.FlashBevError):
        fb.linear_forward(torch.zeros(1, WIDE + 8, device=device), torch.zeros(1, WIDE + 8, device=device))


def apart(t, ld):
    """t's rows at the stride `ld`."""
    big = torch.empty(t.shape[0] * ld, dtype=t.dtype, device=t.device)
    view = big.as_strided(t.shape, (ld, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("M", [5, 300])
@pytest.mark.parametrize("ld", [FAR, FAR - 1])
def test_largest_row_stride(fb, device, M, ld):
    """float32 rows 4 MiB apart (and at places off 16 bytes) in every operand: a tile's last row
    lies past 2^30 bytes from its first."""
    K, N = 72, 40
    gen = torch.Generator(device=device).manual_seed(M)
    x, w, g = (whole(gen, *s, dtype=torch.float32) for s in ((M, K), (N, K), (M, N)))
    xs, ws, gs = apart(x, ld), apart(w, ld), apart(g, ld)
    out, gx, gw = apart(g, ld), apart(x, ld), apart(w, ld)
    fb.linear_forward(xs, ws, residual=gs, out=out)
    assert torch.equal(out, g + (x.double() @ w.double().t()).float())
    fb.linear_backward(gs, xs, ws, want=(), grad_x=gx, grad_weight=gw)
    assert torch.equal(gx, (g.double() @ w.double()).float())
    assert torch.equal(gw, (g.double().t() @ x.double()).float())
    y, s = fb.norm_forward(x, residual=x, scale=0.5)
    ys, ss = fb.norm_forward(xs, residual=xs, scale=0.5, out=gx, out_s=apart(x, ld))
    assert torch.equal(ys, y) and torch.equal(ss, s)


@pytest.mark.parametrize("M,K,N", [(5, 72, 40), (70, 72, 40), (70, 73, 41), (6000, 200, 2056)])
def test_inputs_below_the_normal_numbers(fb, device, M, K, N):
    """float16 from 2^-24 to 2^-15: multiples of 2^-24 whose products with whole numbers add up
    exactly in float32, and are its normal numbers."""
    gen = torch.Generator(device=device).manual_seed(M)
    x = (whole(gen, M, K, dtype=torch.float32, most=511) * 2.0 ** -24).half()
    w, g = whole(gen, N, K, dtype=torch.float16), whole(gen, M, N, dtype=torch.float16)
    assert (x != 0).any() and x.abs().max() < torch.finfo(torch.float16).smallest_normal
    want = x.double() @ w.double().t()
    assert torch.equal(fb.linear_forward(x, w, out_dtype=torch.float32).double(), want)
    assert torch.equal(fb.linear_forward(x, w), want.half())
    got = fb.linear_backward(g, x, w, want=("weight",))["weight"]
    assert torch.equal(got, (g.double().t() @ x.double()).half())


@pytest.mark.parametrize("types", tn.TYPES, ids="-".join)
@pytest.mark.parametrize("G,R,C", [(3001, 1, 40), (1500, 2, 72), (700, 3, 771), (2000, 5, 33), (40, 1, 5001)])
def test_a_gate_for_each_of_many_samples(fb, device, G, R, C, types):
    t, gy, gs = tn.make(G + C, G * R, C, types, "layer", "rms", True, "sample", True, G)
    tn.check_forward(fb, t, "layer", "rms", 0.75, 1e-5, G)
    tn.check_backward(fb, t, gy, gs, "layer", "rms", 0.75, 1e-5, G)
