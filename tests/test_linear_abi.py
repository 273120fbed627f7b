"""The linear operator's argument checks (CPU only): every refusal comes before any
HIP call, so device addresses here are numbers that nothing reads."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2607_10071_amd as fb
from paper_2607_10071_amd import block

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "block", "flashblock.h")
S = fb.STATUS
BASE = 0x7F0000000000
MB = 1 << 20


def pack(M=16, ldx=32, ldw=32, ldr=64, ldo=64, ldp=64, K=32, N=64, dtype=2, out_dtype=2, act=0,
         scale=1.0):
    return block._PACK_LINEAR.pack(M, ldx, ldw, ldr, ldo, ldp, K, N, dtype, out_dtype, act, scale)


def forward(args, x=BASE, w=BASE + MB, b=0, r=0, out=BASE + 2 * MB, pre=0, ws=0, wsb=0):
    return fb._packed_call("flashblock_linear_forward", "PPPPPPPPQP")(args, x, w, b, r, out, pre, ws,
                                                                    wsb, 0)


def backward(args, g=BASE, x=BASE + MB, w=BASE + 2 * MB, pre=0, gx=BASE + 3 * MB, ldgx=32,
             gw=BASE + 4 * MB, ldgw=32, gb=BASE + 5 * MB, ws=BASE + 6 * MB, wsb=1 << 30):
    return fb._packed_call("flashblock_linear_backward", "PPPPPPQPQPPQP")(
        args, g, x, w, pre, gx, ldgx, gw, ldgw, gb, ws, wsb, 0)


def test_the_library_exports_what_the_header_declares():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(flashblock_\w+)\s*\(", src))
    out = subprocess.run(["nm", "-D", "--defined-only", fb.library_path()], capture_output=True,
                         text=True, check=True).stdout
    assert names and set(re.findall(r" T (flashblock_\w+)", out)) == names


def test_header_is_plain_c(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not found")
    c = tmp_path / "t.c"
    c.write_text('#include "block/flashblock.h"\nint main(void) { return sizeof(flashblock_linear) != 72; }\n')
    exe = str(tmp_path / "t")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic",
                    "-I" + os.path.join(ROOT, "include"), str(c), "-o", exe], check=True)
    subprocess.run([exe], check=True)


def test_header_constants():
    src = open(HEADER).read()
    for k, v in block.ACTIVATIONS.items():
        assert re.search(rf"FLASHBLOCK_ACT_{k.upper()} = {v}\b", src), k


def test_packed_structure_is_the_c_one():
    a = block.Linear(5, 6, 7, 8, 9, 10, 11, 12, 1, 0, 3, 0.5)
    assert bytes(memoryview(a).cast("B")) == block._PACK_LINEAR.pack(5, 6, 7, 8, 9, 10, 11, 12, 1, 0,
                                                                     3, 0.5)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), "ERR_SHAPE"), (dict(K=-1), "ERR_SHAPE"), (dict(N=-1), "ERR_SHAPE"),
    (dict(ldx=31), "ERR_SHAPE"), (dict(ldw=31), "ERR_SHAPE"), (dict(ldo=63), "ERR_SHAPE"),
    (dict(dtype=3), "ERR_DTYPE"), (dict(dtype=-1), "ERR_DTYPE"), (dict(out_dtype=1), "ERR_DTYPE"),
    (dict(act=5), "ERR_VALUE"), (dict(act=-1), "ERR_VALUE"), (dict(scale=float("nan")), "ERR_VALUE"),
    (dict(scale=float("inf")), "ERR_VALUE"), (dict(M=1 << 31), "ERR_UNSUPPORTED"),
    (dict(M=(1 << 31) - 255), "ERR_UNSUPPORTED"),
    (dict(K=(1 << 18) + 1, ldx=1 << 19, ldw=1 << 19), "ERR_UNSUPPORTED"),
    (dict(N=(1 << 18) + 1), "ERR_UNSUPPORTED"), (dict(ldx=(1 << 20) + 1), "ERR_UNSUPPORTED"),
])
def test_sizes_and_types(kw, status):
    assert forward(pack(**kw)) == S[status]
    n = ctypes.c_uint64()
    size = fb._packed_call("flashblock_linear_workspace_size", "PP")(pack(**kw), ctypes.byref(n))
    assert size == (S["OK"] if "ld" in next(iter(kw)) else S[status])


def test_null_structures():
    assert forward(None) == S["ERR_NULLPTR"]
    assert backward(None) == S["ERR_NULLPTR"]
    n = ctypes.c_uint64()
    assert fb._packed_call("flashblock_linear_workspace_size", "PP")(None, ctypes.byref(n)) == \
        S["ERR_NULLPTR"]
    assert fb._packed_call("flashblock_linear_workspace_size", "PP")(pack(), None) == S["ERR_NULLPTR"]


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), "ERR_NULLPTR"), (dict(w=0), "ERR_NULLPTR"), (dict(out=0), "ERR_NULLPTR"),
    (dict(x=BASE + 1), "ERR_ALIGN"), (dict(w=BASE + MB + 1), "ERR_ALIGN"),
    (dict(b=BASE + 3 * MB + 1), "ERR_ALIGN"), (dict(r=BASE + 3 * MB + 1), "ERR_ALIGN"),
    (dict(out=BASE + 2 * MB + 1), "ERR_ALIGN"), (dict(pre=BASE + 3 * MB + 1), "ERR_ALIGN"),
    (dict(out=BASE), "ERR_ALIAS"), (dict(out=BASE + MB), "ERR_ALIAS"),
    (dict(b=BASE + 2 * MB), "ERR_ALIAS"), (dict(r=BASE + 2 * MB + 2), "ERR_ALIAS"),
    (dict(pre=BASE + 2 * MB), "ERR_ALIAS"), (dict(pre=BASE), "ERR_ALIAS"),
])
def test_pointers(kw, status):
    assert forward(pack(), **kw) == S[status]


def test_a_residual_in_place_needs_the_same_stride():
    assert forward(pack(ldr=65), r=BASE + 2 * MB) == S["ERR_ALIAS"]


def test_workspace():
    args = pack(M=4096, K=8192, N=64, ldx=8192, ldw=8192)
    n = ctypes.c_uint64()
    assert fb._packed_call("flashblock_linear_workspace_size", "PP")(args, ctypes.byref(n)) == 0
    assert n.value > 0 and n.value % 256 == 0
    far = dict(x=BASE, w=BASE + (256 << 20), out=BASE + (512 << 20))
    ws = BASE + (1 << 30)
    assert forward(args, **far) == S["ERR_NULLPTR"]
    assert forward(args, ws=ws + 128, wsb=n.value, **far) == S["ERR_ALIGN"]
    assert forward(args, ws=ws, wsb=n.value - 1, **far) == S["ERR_SCRATCH"]
    assert forward(args, ws=BASE + (512 << 20), wsb=n.value, **far) == S["ERR_ALIAS"]


def test_empty_calls_enqueue_nothing():
    assert forward(pack(M=0), x=0, out=0) == S["OK"]
    assert forward(pack(N=0, ldr=0, ldo=0, ldp=0), w=0, out=0) == S["OK"]
    assert backward(pack(M=0, N=0), g=0, x=0, w=0, gx=0, gw=0, gb=0) == S["OK"]


@pytest.mark.parametrize("kw,args,status", [
    (dict(gx=0, gw=0, gb=0), {}, "ERR_NULLPTR"), (dict(g=0), {}, "ERR_NULLPTR"),
    (dict(x=0), {}, "ERR_NULLPTR"), (dict(w=0), {}, "ERR_NULLPTR"),
    (dict(), dict(act=1), "ERR_NULLPTR"),                      # an activation without pre
    (dict(ldgx=31), {}, "ERR_SHAPE"), (dict(ldgw=31), {}, "ERR_SHAPE"),
    (dict(), dict(ldo=63), "ERR_SHAPE"), (dict(g=BASE + 1), {}, "ERR_ALIGN"),
    (dict(gb=BASE + 5 * MB + 1), {}, "ERR_ALIGN"), (dict(gx=BASE), {}, "ERR_ALIAS"),
    (dict(gw=BASE + MB), {}, "ERR_ALIAS"), (dict(gx=BASE + 4 * MB), {}, "ERR_ALIAS"),
    (dict(gb=BASE + 3 * MB), {}, "ERR_ALIAS"), (dict(ws=BASE + 6 * MB + 8), {}, "ERR_ALIGN"),
    (dict(wsb=0), {}, "ERR_SCRATCH"), (dict(ws=BASE + 5 * MB), {}, "ERR_ALIAS"),
    (dict(), dict(M=-1), "ERR_SHAPE"), (dict(), dict(dtype=7, out_dtype=7), "ERR_DTYPE"),
])
def test_backward_refusals(kw, args, status):
    assert backward(pack(**args), **kw) == S[status]


def test_backward_reads_only_what_its_gradients_need():
    # refused for the workspace, so past the checks of the pointers that are not needed
    assert backward(pack(), x=0, gw=0, wsb=0) == S["ERR_SCRATCH"]
    assert backward(pack(), w=0, gx=0, wsb=0) == S["ERR_SCRATCH"]
    assert backward(pack(), x=0, w=0, gx=0, gw=0, wsb=0) == S["ERR_SCRATCH"]


def test_sizes_do_not_wrap():
    n = ctypes.c_uint64()
    big = pack(M=(1 << 31) - 256, K=1 << 18, N=1 << 18, ldx=1 << 18, ldw=1 << 18, act=2, ldp=1 << 18,
               ldo=1 << 18)
    call = fb._packed_call("flashblock_linear_backward_workspace_size", "PiiiP")
    assert call(big, 1, 1, 1, ctypes.byref(n)) == 0
    assert n.value >= ((1 << 31) - 256) * (1 << 18) * 2


class _Cuda:
    """A tensor that says it is on the device, for the binding's own checks."""

    def __init__(self, t):
        self._t = t
        self.is_cuda = True

    def __getattr__(self, k):
        return getattr(self._t, k)


def test_rows_of_strided_tensors():
    def rows(t):
        return block._rows(_Cuda(t), "t")

    t = torch.zeros(4, 6, 10)
    assert rows(t) == (24, 10)
    assert rows(t[..., :7]) == (24, 10)
    assert rows(t[:, :, 3:]) == (24, 10)
    assert rows(t[0]) == (6, 10) and rows(t[:, 0]) == (4, 60) and rows(t[0, 0]) == (1, 10)
    assert rows(t[0, 0, :4]) == (1, 4)
    assert rows(t[:1, 2:3, :5]) == (1, 5)
    assert rows(torch.zeros(3, 0)) == (3, 0) and rows(torch.zeros(0, 5)) == (0, 5)
    for bad in (t[:, :4], t.transpose(0, 1), t[..., ::2], t.transpose(1, 2),
                torch.zeros(1, 4).expand(3, 4)):
        with pytest.raises(ValueError):
            rows(bad)
    with pytest.raises(ValueError):
        rows(torch.zeros(()))


def test_host_tensors_and_bad_types_are_refused():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError):
        fb.linear_forward(x, w)
    with pytest.raises(ValueError):
        fb.linear_backward(torch.zeros(4, 6), x, w)
    with pytest.raises(ValueError):
        block._act_code("tanh")
    assert block._act_code(None) == 0
    with pytest.raises(ValueError):
        block._out_type(torch.float16, _Cuda(x.bfloat16()))
    with pytest.raises(TypeError):
        fb._dtype_code(torch.zeros(1, dtype=torch.float64))
    with pytest.raises(ValueError):
        block._weight(_Cuda(w.half()), _Cuda(x))
    with pytest.raises(ValueError):
        block._weight(_Cuda(torch.zeros(6, 7)), _Cuda(x))
