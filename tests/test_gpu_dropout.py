"""Dropout on the GPU: the generator's words in Python's integers, values to the rounding."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2607_10071_amd as fb

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)]
IDS = ["f32", "f16", "bf16", "f16_f32", "bf16_f32"]


def test_the_generator_is_the_published_one():
    """Words of the paper's own test vectors (its library's kat_vectors, Philox 4x32-10)."""
    assert ref.philox_block([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    f = 0xffffffff
    assert ref.philox_block([f] * 4, [f] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert ref.philox_block([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0]) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def expected(x, p, seed, offset, residual, scale, dtype):
    """(result, bound)"""
    keep = ref.kept(x.numel(), p, seed, offset).reshape(x.shape).to(x.device)
    factor = scale / (1 - p) if p < 1 else 0.0
    want = torch.where(keep, x.double() * factor, 0.0)
    tol = want.abs() * 2.1 * ref.U32   # the factor and the product
    if residual is not None:
        want = want + residual.double()
        tol = tol + want.abs() * ref.U32
    return want, tol + ref.half(dtype) * want.abs() + ref._floor(dtype), keep


@pytest.mark.parametrize("dtype,sdt", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 5), (2, 4, 8), (17, 33), (5, 1000), (2, 3, 77), (64, 64)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0, 2.0 ** -33, 1e-9])
def test_values(shape, dtype, sdt, p):
    g = torch.Generator(device="cuda").manual_seed(len(shape))
    x = torch.randn(shape, generator=g, device="cuda").to(dtype)
    r = torch.randn(shape, generator=g, device="cuda").to(sdt)
    for seed, offset in ((0, 0), (-5, 3), (0xFEDCBA9876543210, (1 << 64) - 1)):
        for res in (None, r):
            want, tol, keep = expected(x, p, seed, offset, res, 0.75, sdt if res is not None else dtype)
            got = fb.dropout_forward(x, p, seed, offset, residual=res, scale=0.75)
            assert got.dtype == (sdt if res is not None else dtype)
            ref.check(got, want, tol, "out")
        gx = fb.dropout_backward(r, p, seed, offset, 0.75, dtype=dtype)
        want, tol, _ = expected(r, p, seed, offset, None, 0.75, dtype)
        ref.check(gx, want, tol, "grad_x")
        # the state in device memory gives the same
        words = torch.tensor([seed - (1 << 64) if seed >= 1 << 63 else seed,
                              offset - (1 << 64) if offset >= 1 << 63 else offset], device="cuda")
        assert torch.equal(got, fb.dropout_forward(x, p, words, residual=r, scale=0.75))
        assert torch.equal(gx, fb.dropout_backward(r, p, words, scale=0.75, dtype=dtype))


@pytest.mark.parametrize("dtype,sdt", TYPES, ids=IDS)
@pytest.mark.parametrize("C", [3, 8, 40, 77])
def test_strides_do_not_change_the_mask(dtype, sdt, C):
    g = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn((50, C + 9), generator=g, device="cuda").to(dtype)[:, 2:C + 2]
    r = torch.randn((50, C + 21), generator=g, device="cuda").to(sdt)[:, 5:C + 5]
    want = fb.dropout_forward(x.contiguous(), 0.3, 11, 5, residual=r.contiguous(), scale=0.5)
    exact, tol, _ = expected(x, 0.3, 11, 5, r, 0.5, sdt)
    ref.check(want, exact, tol)
    room = torch.full((50, C + 4), 9.0, device="cuda", dtype=sdt)
    assert torch.equal(fb.dropout_forward(x, 0.3, 11, 5, residual=r, scale=0.5, out=room[:, 1:C + 1]), want)
    assert (room[:, 0] == 9).all() and (room[:, C + 1:] == 9).all()
    assert torch.equal(fb.dropout_forward(x, 0.3, 11, 5, residual=r.contiguous(), scale=0.5), want)
    gx = fb.dropout_backward(r, 0.3, 11, 5, dtype=dtype)
    assert torch.equal(gx, fb.dropout_backward(r.contiguous(), 0.3, 11, 5, dtype=dtype))
    # onto the residual itself
    s = r.contiguous()
    fb.dropout_forward(x, 0.3, 11, 5, residual=s, scale=0.5, out=s)
    assert torch.equal(s, want)


def test_what_is_dropped_may_hold_anything():
    keep = ref.kept(400, 0.5, 3, 0).reshape(20, 20).cuda()
    x = torch.ones((20, 20), device="cuda")
    for bad in (math.nan, math.inf, -math.inf):
        y = torch.where(keep, x, bad)
        assert torch.equal(fb.dropout_forward(y, 0.5, 3), torch.where(keep, 2.0, 0.0))
        assert torch.equal(fb.dropout_forward(y, 0.5, 3, residual=x), torch.where(keep, 3.0, 1.0))
        assert torch.equal(fb.dropout_backward(y, 0.5, 3), torch.where(keep, 2.0, 0.0))


def test_places_past_32_bits():
    """The words of elements past 2^32 (blocks past 2^30) and past 2^34 (blocks past 2^32)."""
    for M, C, p in (((1 << 17) + 1, 1 << 15, 0.25), ((1 << 17) + 3, (1 << 17) + 8, 0.25)):
        big = torch.empty((M, C), device="cuda", dtype=BF16)
        big.fill_(1.0)
        out = fb.dropout_forward(big, p, 77, 1)
        for row in (0, M // 2 + 1, M - 1):
            n = 64
            for first in (0, C - n):
                keep = ref.kept(n, p, 77, 1, row * C + first)
                assert torch.equal(out[row, first:first + n].cpu() != 0, keep), (M, C, row, first)
        del big, out


def test_share_and_independence():
    x = torch.ones((4000, 1000), device="cuda")
    a = fb.dropout_forward(x, 0.1, 1, 0) != 0
    n = a.numel()
    # five standard deviations of a binomial count
    assert abs(a.sum().item() - 0.9 * n) < 5 * math.sqrt(0.09 * n)
    for other in (fb.dropout_forward(x, 0.1, 1, 1), fb.dropout_forward(x, 0.1, 2, 0)):
        both = (a & (other != 0)).sum().item()
        assert abs(both - 0.81 * n) < 5 * math.sqrt(0.81 * 0.19 * n)


@pytest.mark.parametrize("dtype,sdt", TYPES, ids=IDS)
def test_autograd(dtype, sdt):
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((30, 50), generator=g, device="cuda").to(dtype).requires_grad_()
    r = torch.randn((30, 50), generator=g, device="cuda").to(sdt).requires_grad_()
    go = torch.randn((30, 50), generator=g, device="cuda").to(sdt)
    for seed in (9, torch.tensor([9, 0], device="cuda")):
        out = fb.dropout_autograd(x, 0.4, seed, residual=r, scale=0.5)
        gx, gr = torch.autograd.grad(out, [x, r], go)
        assert gx.dtype == dtype and torch.equal(gr, go)
        want, tol, _ = expected(go, 0.4, 9, 0, None, 0.5, dtype)
        ref.check(gx, want, tol)
        (gx2,) = torch.autograd.grad(fb.dropout_autograd(x, 0.4, seed, residual=r.detach(), scale=0.5), [x],
                                     go.t().contiguous().t())
        assert torch.equal(gx, gx2)
    out = fb.dropout_autograd(x, 0.4, seed)
    seed.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.float().sum().backward()


def test_captured_graph_drops_anew():
    x = torch.randn((64, 128), device="cuda")
    state = torch.tensor([5, 0], device="cuda")
    out = torch.empty_like(x)
    fb.dropout_forward(x, 0.5, state, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.dropout_forward(x, 0.5, state, out=out)
    for step in range(4):
        state.copy_(torch.tensor([5, step]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fb.dropout_forward(x, 0.5, 5, step)), step


@pytest.mark.parametrize("residual", [False, True])
def test_prepared(residual):
    """The same call again, of what its tensors then hold; with a device tensor as the seed too."""
    x, r = torch.randn(33, 70, device="cuda"), torch.randn(33, 70, device="cuda") if residual else None
    state = torch.tensor([5, 6], device="cuda")
    out = torch.empty_like(x)
    calls = [(fb.prepare_dropout_forward(x, 0.4, 5, 6, residual=r, scale=0.5, out=out), (5, 6)),
             (fb.prepare_dropout_forward(x, 0.4, state, residual=r, scale=0.5, out=out), None)]
    for step in range(3):
        x.copy_(torch.randn_like(x))
        state.copy_(torch.tensor([step, 9]))
        for call, seed in calls:
            out.fill_(7)
            call()
            assert torch.equal(out, fb.dropout_forward(x, 0.4, *(seed or (step, 9)), residual=r, scale=0.5))
