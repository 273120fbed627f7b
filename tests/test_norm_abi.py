"""The norm operator's argument checks (CPU only): every refusal comes before any HIP
call, so device addresses here are numbers that nothing reads."""
import ctypes

import pytest
import torch

import paper_2607_10071_amd as fb
from paper_2607_10071_amd import block
from test_linear_abi import BASE, MB, S, _Cuda

FIELDS = dict(M=16, ldx=32, ldr=32, lds=32, ldy=32, groups=1, C=32, dtype=2, stream_dtype=2,
              param_dtype=2, norm=1, post_norm=0, eps=1e-5, scale=1.0)


def pack(**kw):
    return block._PACK_NORM.pack(*{**FIELDS, **kw}.values())


def vectors(gate=0, weight=0, bias=0, post_weight=0, post_bias=0):
    return block._PACK_VECTORS.pack(gate, weight, bias, post_weight, post_bias)


def forward(args, v=vectors(), x=BASE, r=0, s=BASE + MB, y=BASE + 2 * MB):
    return fb._packed_call("flashblock_norm_forward", "PPPPPPP")(args, v, x, r, s, y, 0)


def backward(args, v=vectors(), gy=BASE, gs=BASE + MB, x=BASE + 2 * MB, s=BASE + 3 * MB,
             gx=BASE + 4 * MB, ldgx=32, gr=BASE + 5 * MB, ldgr=32, grads=vectors(), ws=BASE + 8 * MB,
             wsb=1 << 20):
    return fb._packed_call("flashblock_norm_backward", "PPPPPPPQPQPPQP")(
        args, v, gy, gs, x, s, gx, ldgx, gr, ldgr, grads, ws, wsb, 0)


def test_packed_structure_is_the_c_one():
    a = block.Norm(*FIELDS.values())
    assert bytes(memoryview(a).cast("B")) == pack()
    src = open(__import__("test_linear_abi").HEADER).read()
    for k, v in block.NORMS.items():
        assert f"FLASHBLOCK_NORM_{k.upper()} = {v}" in src


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), "ERR_SHAPE"), (dict(C=-1), "ERR_SHAPE"), (dict(groups=0), "ERR_SHAPE"),
    (dict(groups=3), "ERR_SHAPE"), (dict(ldx=31), "ERR_SHAPE"), (dict(lds=31), "ERR_SHAPE"),
    (dict(ldy=31), "ERR_SHAPE"), (dict(dtype=3), "ERR_DTYPE"), (dict(stream_dtype=1), "ERR_DTYPE"),
    (dict(param_dtype=1), "ERR_DTYPE"), (dict(norm=3), "ERR_VALUE"), (dict(norm=0), "ERR_VALUE"),
    (dict(post_norm=-1), "ERR_VALUE"), (dict(eps=0.0), "ERR_VALUE"), (dict(eps=-1.0), "ERR_VALUE"),
    (dict(eps=float("nan")), "ERR_VALUE"), (dict(scale=float("inf")), "ERR_VALUE"),
    (dict(M=1 << 31), "ERR_UNSUPPORTED"), (dict(C=16385, ldx=1 << 15), "ERR_UNSUPPORTED"),
    (dict(ldx=(1 << 20) + 1), "ERR_UNSUPPORTED"),
])
def test_sizes_and_types(kw, status):
    assert forward(pack(**kw)) == S[status]
    n = ctypes.c_uint64()
    size = fb._packed_call("flashblock_norm_backward_workspace_size", "PPP")(
        pack(**kw), vectors(weight=1), ctypes.byref(n))
    assert size == (S["OK"] if next(iter(kw)).startswith("ld") else S[status])


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), "ERR_NULLPTR"), (dict(y=0), "ERR_NULLPTR"), (dict(x=BASE + 1), "ERR_ALIGN"),
    (dict(r=BASE + 3 * MB + 1), "ERR_ALIGN"), (dict(s=BASE + MB + 1), "ERR_ALIGN"),
    (dict(y=BASE + 2 * MB + 1), "ERR_ALIGN"), (dict(s=BASE), "ERR_ALIAS"), (dict(y=BASE), "ERR_ALIAS"),
    (dict(y=BASE + MB), "ERR_ALIAS"), (dict(r=BASE + 2 * MB), "ERR_ALIAS"),
    (dict(r=BASE + MB + 2), "ERR_ALIAS"), (dict(v=None), "ERR_NULLPTR"),
    (dict(v=vectors(weight=BASE + 3 * MB + 1)), "ERR_ALIGN"),
    (dict(v=vectors(gate=BASE + MB)), "ERR_ALIAS"), (dict(v=vectors(bias=BASE + 2 * MB)), "ERR_ALIAS"),
    (dict(v=vectors(post_weight=BASE + 3 * MB)), "ERR_VALUE"),
    (dict(v=vectors(post_bias=BASE + 3 * MB)), "ERR_VALUE"),
])
def test_pointers(kw, status):
    assert forward(pack(), **kw) == S[status]


def test_forms():
    none = pack(norm=0, post_norm=1)
    assert forward(none) == S["ERR_VALUE"]                      # y without a norm
    assert forward(none, y=0, s=0) == S["ERR_NULLPTR"]          # nothing to write
    assert forward(none, v=vectors(weight=BASE + 3 * MB), y=0) == S["ERR_VALUE"]
    assert forward(pack(ldr=33), r=BASE + MB) == S["ERR_ALIAS"]   # in place needs one stride
    assert forward(None) == S["ERR_NULLPTR"]
    assert forward(pack(M=0), x=0, s=0, y=0) == S["OK"]
    assert forward(pack(C=0), x=0, s=0, y=0) == S["OK"]


W = dict(grads=vectors(weight=BASE + 6 * MB))


@pytest.mark.parametrize("kw,args,status", [
    (dict(gx=0, gr=0), {}, "ERR_NULLPTR"), (dict(gy=0, gs=0), {}, "ERR_NULLPTR"),
    (dict(s=0), {}, "ERR_NULLPTR"), (dict(x=0), dict(post_norm=2), "ERR_NULLPTR"),
    (dict(x=0, grads=vectors(gate=BASE + 6 * MB)), {}, "ERR_NULLPTR"),
    (dict(ldgx=31), {}, "ERR_SHAPE"), (dict(ldgr=31), {}, "ERR_SHAPE"), (dict(), dict(ldy=31), "ERR_SHAPE"),
    (dict(), dict(ldr=31), "ERR_SHAPE"), (dict(gy=BASE + 1), {}, "ERR_ALIGN"),
    (dict(gx=BASE + 4 * MB + 1), {}, "ERR_ALIGN"), (dict(grads=vectors(weight=BASE + 6 * MB + 1)), {},
                                                   "ERR_ALIGN"),
    (dict(gx=BASE), {}, "ERR_ALIAS"), (dict(gr=BASE + 3 * MB), {}, "ERR_ALIAS"),
    (dict(gx=BASE + 5 * MB), {}, "ERR_ALIAS"), (dict(grads=vectors(weight=BASE + MB)), {}, "ERR_ALIAS"),
    (dict(**W, ws=0), {}, "ERR_NULLPTR"), (dict(**W, ws=BASE + 8 * MB + 8), {}, "ERR_ALIGN"),
    (dict(**W, wsb=0), {}, "ERR_SCRATCH"), (dict(**W, ws=BASE + 5 * MB), {}, "ERR_ALIAS"),
    (dict(grads=vectors(post_weight=BASE + 6 * MB)), {}, "ERR_VALUE"),
    (dict(**W), dict(norm=0, post_norm=1), "ERR_VALUE"), (dict(), dict(norm=0, post_norm=1), "ERR_VALUE"),
])
def test_backward_refusals(kw, args, status):
    assert backward(pack(**args), **kw) == S[status]


def test_backward_reads_only_what_its_gradients_need():
    # refused for the workspace, so past the checks of the pointers that are not needed
    assert backward(pack(), x=0, gx=0, gr=0, **{**W, "wsb": 0}) == S["ERR_SCRATCH"]
    assert backward(pack(norm=0, post_norm=1), gy=0, s=0, grads=vectors(post_weight=BASE + 6 * MB),
                    wsb=0) == S["ERR_SCRATCH"]
    assert backward(pack(M=0), gy=0, gs=0, x=0, s=0, gx=0, gr=0) == S["OK"]


def test_workspace_of_many_samples():
    n = ctypes.c_uint64()
    call = fb._packed_call("flashblock_norm_backward_workspace_size", "PPP")
    assert call(pack(), vectors(), ctypes.byref(n)) == 0 and n.value == 0
    assert call(pack(), None, ctypes.byref(n)) == 0 and n.value == 0
    assert call(pack(M=1 << 20, groups=1 << 20), vectors(gate=1), ctypes.byref(n)) == 0
    assert n.value >= (1 << 20) * 32 * 4
    assert call(pack(M=40000, C=256), vectors(weight=1, bias=1), ctypes.byref(n)) == 0
    assert 0 < n.value <= 2 * 2048 * 256 * 4 and n.value % 256 == 0


def test_the_bindings_own_checks():
    x = torch.zeros(4, 6, 8)
    v = torch.zeros(8)
    with pytest.raises(ValueError):
        fb.norm_forward(x)   # a host tensor
    for bad in (dict(gate=torch.zeros(6, 8)), dict(gate=torch.zeros(4, 7)), dict(gate=torch.zeros(7)),
                dict(weight=torch.zeros(9)), dict(bias=torch.zeros(8, dtype=torch.float64)),
                dict(weight=v.half()), dict(weight=v, bias=v.half()), dict(weight=torch.zeros(8, 1))):
        bad = {k: _Cuda(t) for k, t in bad.items()}
        args = {**dict.fromkeys(("gate", "weight", "bias", "post_weight", "post_bias")), **bad}
        with pytest.raises(ValueError):
            block._norm_vectors(_Cuda(x), *args.values())
    with pytest.raises(ValueError):
        block._norm_code("batch", "norm")
    assert block._norm_code(None, "norm") == 0
