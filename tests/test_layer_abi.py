"""Argument checks of attention, group norm and dropout (CPU only): every refusal comes before
any HIP call, so device addresses here are numbers that nothing reads."""
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2607_10071_amd as fb
from paper_2607_10071_amd import layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "block", "flashlayer.h")
S = fb.STATUS
BASE = 0x7F0000000000
MB = 1 << 20


def attention_args(B=2, Lq=8, Lk=16, H=4, Hk=2, D=32, dtype=2, mask=0, scale=1.0, **strides):
    d = dict(q_batch=Lq * H * D, q_row=H * D, q_head=D, k_batch=Lk * Hk * D, k_row=Hk * D, k_head=D,
             v_batch=Lk * Hk * D, v_row=Hk * D, v_head=D, o_batch=Lq * H * D, o_row=H * D, o_head=D,
             mask_batch=0, mask_head=0, mask_row=0)
    d.update(strides)
    return layer._PACK_ATTENTION.pack(*d.values(), B, Lq, Lk, H, Hk, D, dtype, mask, scale)


def attention(args, q=BASE, k=BASE + MB, v=BASE + 2 * MB, mask=0, lengths=0, out=BASE + 3 * MB, rest=0, stats=0,
              ws=0, wsb=0):
    return fb._packed_call("flashlayer_attention_forward", "PPPPPPPPPPQP")(args, q, k, v, mask, lengths, out, rest,
                                                                        stats, ws, wsb, 0)


def attention_backward(args, g=BASE, q=BASE + MB, k=BASE + 2 * MB, v=BASE + 3 * MB, mask=0, lengths=0,
                       out=BASE + 4 * MB, rest=0, stats=BASE + 5 * MB, gq=BASE + 6 * MB, gk=BASE + 7 * MB,
                       gv=BASE + 8 * MB, ws=BASE + 9 * MB, wsb=1 << 30):
    return fb._packed_call("flashlayer_attention_backward", "PPPPPPPPPPPPPPQP")(
        args, g, q, k, v, mask, lengths, out, rest, stats, gq, gk, gv, ws, wsb, 0)


def group_args(N=2, R=100, ldx=64, ldy=64, C=64, groups=8, dtype=2, param_dtype=0, act=0, eps=1e-5):
    return layer._PACK_GROUP_NORM.pack(N, R, ldx, ldy, C, groups, dtype, param_dtype, act, eps)


def group_norm(args, x=BASE, w=0, b=0, y=BASE + MB, stats=0, ws=BASE + 2 * MB, wsb=1 << 30):
    return fb._packed_call("flashlayer_group_norm_forward", "PPPPPPPQP")(args, x, w, b, y, stats, ws, wsb, 0)


def group_norm_backward(args, g=BASE, x=BASE + MB, stats=BASE + 2 * MB, w=0, b=0, gx=BASE + 3 * MB, gw=BASE + 4 * MB,
                        gb=BASE + 5 * MB, ws=BASE + 6 * MB, wsb=1 << 30):
    return fb._packed_call("flashlayer_group_norm_backward", "PPPPPPPPPPQP")(args, g, x, stats, w, b, gx, gw, gb, ws,
                                                                          wsb, 0)


def drop_args(M=16, ldx=32, ldr=32, ldo=32, seed=1, offset=2, p=0.1, C=32, dtype=2, stream_dtype=2, scale=1.0):
    return layer._PACK_DROPOUT.pack(M, ldx, ldr, ldo, seed, offset, p, C, dtype, stream_dtype, scale)


def dropout(args, x=BASE, r=0, state=0, out=BASE + MB):
    return fb._packed_call("flashlayer_dropout_forward", "PPPPPP")(args, x, r, state, out, 0)


def dropout_backward(args, g=BASE, state=0, gx=BASE + MB):
    return fb._packed_call("flashlayer_dropout_backward", "PPPPP")(args, g, state, gx, 0)


def test_the_library_exports_what_the_header_declares():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(flashlayer_\w+)\s*\(", src))
    out = subprocess.run(["nm", "-D", "--defined-only", fb.library_path()], capture_output=True, text=True,
                         check=True).stdout
    assert len(names) == 10 and set(re.findall(r" T (flashlayer_\w+)", out)) == names


def test_header_is_plain_c(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not found")
    c = tmp_path / "t.c"
    c.write_text('#include "block/flashlayer.h"\nint main(void) { return sizeof(flashlayer_attention) != 160 || '
                 'sizeof(flashlayer_group_norm) != 56 || sizeof(flashlayer_dropout) != 72; }\n')
    exe = str(tmp_path / "t")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I" + os.path.join(ROOT, "include"),
                    str(c), "-o", exe], check=True)
    subprocess.run([exe], check=True)


def test_header_constants():
    src = open(HEADER).read()
    assert re.search(rf"FLASHLAYER_HEAD_MAX {layer.HEAD_MAX}\b", src)
    for k, v in layer.MASKS.items():
        assert re.search(rf"FLASHLAYER_MASK_{k.upper()} = {v}\b", src), k


def test_packed_structures_are_the_c_ones():
    a = layer.Attention(*range(1, 16), 21, 22, 23, 24, 25, 26, 1, 2, 0.5)
    assert bytes(memoryview(a).cast("B")) == layer._PACK_ATTENTION.pack(*range(1, 16), 21, 22, 23, 24, 25, 26, 1, 2, 0.5)
    a = layer.GroupNorm(1, 2, 3, 4, 5, 6, 1, 0, 3, 0.25)
    assert bytes(memoryview(a).cast("B")) == layer._PACK_GROUP_NORM.pack(1, 2, 3, 4, 5, 6, 1, 0, 3, 0.25)
    a = layer.Dropout(1, 2, 3, 4, 5, 6, 0.5, 7, 1, 0, 0.25)
    assert bytes(memoryview(a).cast("B")) == layer._PACK_DROPOUT.pack(1, 2, 3, 4, 5, 6, 0.5, 7, 1, 0, 0.25)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), "ERR_SHAPE"), (dict(Lq=-1), "ERR_SHAPE"), (dict(Lk=-1), "ERR_SHAPE"), (dict(H=3), "ERR_SHAPE"),
    (dict(Hk=0), "ERR_SHAPE"), (dict(D=-1), "ERR_SHAPE"), (dict(D=129), "ERR_UNSUPPORTED"), (dict(dtype=3), "ERR_DTYPE"),
    (dict(dtype=-1), "ERR_DTYPE"), (dict(mask=4), "ERR_VALUE"), (dict(mask=-1), "ERR_VALUE"),
    (dict(scale=0.0), "ERR_VALUE"), (dict(scale=-1.0), "ERR_VALUE"), (dict(scale=float("nan")), "ERR_VALUE"),
    (dict(scale=float("inf")), "ERR_VALUE"), (dict(k_row=-1), "ERR_SHAPE"), (dict(mask_row=-1), "ERR_SHAPE"),
    (dict(k_row=(1 << 20) + 1), "ERR_UNSUPPORTED"), (dict(v_row=(1 << 20) + 1), "ERR_UNSUPPORTED"),
    (dict(Lk=0x7FFFFE01), "ERR_UNSUPPORTED"), (dict(Lq=1 << 30, H=4, Hk=1), "ERR_UNSUPPORTED"),
    (dict(Lq=1 << 27, H=64, Hk=1), "ERR_UNSUPPORTED"),
])
def test_attention_sizes_and_types(kw, status):
    assert attention(attention_args(**kw)) == S[status]
    assert attention_backward(attention_args(**kw)) == S[status]
    n = fb.layer.ctypes.c_uint64()
    size = fb._packed_call("flashlayer_attention_workspace_size", "PP")
    assert size(attention_args(**kw), fb.layer.ctypes.byref(n)) == S[status]


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), "ERR_NULLPTR"), (dict(k=0), "ERR_NULLPTR"), (dict(v=0), "ERR_NULLPTR"), (dict(out=0), "ERR_NULLPTR"),
    (dict(q=BASE + 1), "ERR_ALIGN"), (dict(k=BASE + MB + 1), "ERR_ALIGN"), (dict(out=BASE + 3 * MB + 1), "ERR_ALIGN"),
    (dict(stats=BASE + 5 * MB + 2), "ERR_ALIGN"), (dict(lengths=BASE + 5 * MB + 2), "ERR_ALIGN"),
    (dict(rest=BASE + 5 * MB + 1), "ERR_ALIGN"), (dict(out=BASE + 64), "ERR_ALIAS"), (dict(out=BASE + MB), "ERR_ALIAS"),
    (dict(out=BASE + 2 * MB - 64), "ERR_ALIAS"), (dict(rest=BASE + 3 * MB), "ERR_ALIAS"),
    (dict(stats=BASE + 3 * MB), "ERR_ALIAS"), (dict(lengths=BASE + 3 * MB + 8), "ERR_ALIAS"),
])
def test_attention_pointers(kw, status):
    assert attention(attention_args(), **kw) == S[status]


def test_attention_more_refusals():
    assert attention(attention_args(mask=1)) == S["ERR_NULLPTR"]
    assert attention(attention_args(mask=3), mask=BASE + 6 * MB + 2) == S["ERR_ALIGN"]
    assert attention(attention_args(mask=1, mask_row=16), mask=BASE + 3 * MB + 1) == S["ERR_ALIAS"]
    # outputs whose elements share places
    assert attention(attention_args(o_head=0)) == S["ERR_SHAPE"]
    assert attention(attention_args(o_row=32)) == S["ERR_SHAPE"]
    assert attention(attention_args(o_batch=0)) == S["ERR_SHAPE"]
    assert attention(None) == S["ERR_NULLPTR"]
    # spans that leave 64 bits
    assert attention(attention_args(q_batch=1 << 62)) == S["ERR_UNSUPPORTED"]
    # few queries to many keys need a workspace
    long = attention_args(Lq=1, Lk=50000)
    assert attention(long) == S["ERR_NULLPTR"]
    far = dict(k=BASE + 64 * MB, v=BASE + 128 * MB)
    assert attention(long, ws=BASE + 512 * MB + 4, wsb=1 << 30, **far) == S["ERR_ALIGN"]
    assert attention(long, ws=BASE + 512 * MB, wsb=64, **far) == S["ERR_SCRATCH"]
    assert attention(long, ws=BASE, wsb=1 << 30, **far) == S["ERR_ALIAS"]


@pytest.mark.parametrize("kw,status", [
    (dict(g=0), "ERR_NULLPTR"), (dict(q=0), "ERR_NULLPTR"), (dict(k=0), "ERR_NULLPTR"), (dict(v=0), "ERR_NULLPTR"),
    (dict(out=0), "ERR_NULLPTR"), (dict(stats=0), "ERR_NULLPTR"), (dict(gk=0), "ERR_NULLPTR"),
    (dict(gv=0), "ERR_NULLPTR"), (dict(gq=0, gk=0, gv=0), "ERR_NULLPTR"), (dict(ws=0), "ERR_NULLPTR"),
    (dict(ws=BASE + 9 * MB + 8), "ERR_ALIGN"), (dict(wsb=100), "ERR_SCRATCH"), (dict(gq=BASE), "ERR_ALIAS"),
    (dict(gk=BASE + 6 * MB), "ERR_ALIAS"), (dict(gv=BASE + 7 * MB + 64), "ERR_ALIAS"),
    (dict(gq=BASE + 4 * MB), "ERR_ALIAS"), (dict(gq=BASE + 5 * MB), "ERR_ALIAS"), (dict(gq=BASE + 6 * MB + 1), "ERR_ALIGN"),
    (dict(stats=BASE + 5 * MB + 1), "ERR_ALIGN"),
])
def test_attention_backward_pointers(kw, status):
    assert attention_backward(attention_args(), **kw) == S[status]


def test_attention_without_elements():
    assert attention(attention_args(B=0), q=0, k=0, v=0, out=0) == 0
    assert attention(attention_args(Lq=0), q=0, out=0) == 0
    assert attention_backward(attention_args(B=0), *[0] * 4) == 0
    n = fb.layer.ctypes.c_uint64()
    size = fb._packed_call("flashlayer_attention_backward_workspace_size", "PiiP")
    assert size(attention_args(B=0), 1, 1, fb.layer.ctypes.byref(n)) == 0 and n.value == 0
    assert size(attention_args(), 1, 1, None) == S["ERR_NULLPTR"]


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), "ERR_SHAPE"), (dict(R=-1), "ERR_SHAPE"), (dict(C=-8), "ERR_SHAPE"), (dict(groups=0), "ERR_SHAPE"),
    (dict(groups=7), "ERR_SHAPE"), (dict(ldx=63), "ERR_SHAPE"), (dict(ldy=63), "ERR_SHAPE"), (dict(dtype=3), "ERR_DTYPE"),
    (dict(param_dtype=1), "ERR_DTYPE"), (dict(act=5), "ERR_VALUE"), (dict(act=-1), "ERR_VALUE"), (dict(eps=0.0), "ERR_VALUE"),
    (dict(eps=float("nan")), "ERR_VALUE"), (dict(eps=float("inf")), "ERR_VALUE"),
    (dict(C=16392, ldx=16392, ldy=16392, groups=8), "ERR_UNSUPPORTED"), (dict(ldx=(1 << 20) + 1), "ERR_UNSUPPORTED"),
    (dict(N=1 << 20, R=1 << 20), "ERR_UNSUPPORTED"), (dict(N=1 << 40, R=1 << 40), "ERR_UNSUPPORTED"),
])
def test_group_norm_sizes_and_types(kw, status):
    assert group_norm(group_args(**kw)) == S[status]
    assert group_norm_backward(group_args(**kw)) == S[status]


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), "ERR_NULLPTR"), (dict(y=0), "ERR_NULLPTR"), (dict(x=BASE + 1), "ERR_ALIGN"), (dict(w=BASE + 3 * MB + 2), "ERR_ALIGN"),
    (dict(stats=BASE + 3 * MB + 2), "ERR_ALIGN"), (dict(y=BASE), "ERR_ALIAS"), (dict(w=BASE + MB), "ERR_ALIAS"),
    (dict(stats=BASE + MB), "ERR_ALIAS"),
])
def test_group_norm_pointers(kw, status):
    assert group_norm(group_args(), **kw) == S[status]


def test_group_norm_workspaces():
    big = group_args(R=5000)
    n = fb.layer.ctypes.c_uint64()
    assert fb._packed_call("flashlayer_group_norm_workspace_size", "PP")(big, fb.layer.ctypes.byref(n)) == 0 and n.value
    far = dict(y=BASE + 64 * MB)
    assert group_norm(big, ws=0, **far) == S["ERR_NULLPTR"]
    assert group_norm(big, ws=BASE + 128 * MB + 8, **far) == S["ERR_ALIGN"]
    assert group_norm(big, ws=BASE + 128 * MB, wsb=n.value - 1, **far) == S["ERR_SCRATCH"]
    assert group_norm(big, ws=BASE, **far) == S["ERR_ALIAS"]
    assert group_norm_backward(group_args(), wsb=64) == S["ERR_SCRATCH"]
    assert group_norm_backward(group_args(), gx=0, gw=0, gb=0) == S["ERR_NULLPTR"]
    assert group_norm_backward(group_args(), gx=BASE) == S["ERR_ALIAS"]
    assert group_norm_backward(group_args(), gb=BASE + 4 * MB) == S["ERR_ALIAS"]
    assert group_norm_backward(group_args(), stats=0) == S["ERR_NULLPTR"]


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), "ERR_SHAPE"), (dict(C=-1), "ERR_SHAPE"), (dict(ldx=31), "ERR_SHAPE"), (dict(ldo=31), "ERR_SHAPE"),
    (dict(dtype=3), "ERR_DTYPE"), (dict(stream_dtype=1), "ERR_DTYPE"), (dict(p=-0.1), "ERR_VALUE"), (dict(p=1.1), "ERR_VALUE"),
    (dict(p=float("nan")), "ERR_VALUE"), (dict(scale=float("inf")), "ERR_VALUE"), (dict(M=1 << 31), "ERR_UNSUPPORTED"),
    (dict(C=(1 << 18) + 1, ldx=1 << 19, ldo=1 << 19), "ERR_UNSUPPORTED"), (dict(ldx=(1 << 20) + 1), "ERR_UNSUPPORTED"),
    (dict(ldo=(1 << 20) + 1), "ERR_UNSUPPORTED"),
])
def test_dropout_sizes_and_types(kw, status):
    assert dropout(drop_args(**kw)) == S[status]
    assert dropout_backward(drop_args(**kw)) == S[status]


def test_dropout_pointers():
    a = drop_args()
    assert dropout(a, x=0) == dropout(a, out=0) == dropout_backward(a, gx=0) == dropout(None) == S["ERR_NULLPTR"]
    assert dropout(a, x=BASE + 1) == dropout(a, out=BASE + MB + 1) == dropout(a, state=BASE + 4 * MB + 4) == S["ERR_ALIGN"]
    assert dropout(a, r=BASE + 4 * MB + 1) == S["ERR_ALIGN"]
    assert dropout(a, out=BASE) == dropout(a, out=BASE + 64) == dropout_backward(a, gx=BASE + 64) == S["ERR_ALIAS"]
    assert dropout(a, r=BASE + MB + 64) == dropout(a, state=BASE + MB) == S["ERR_ALIAS"]
    assert dropout(drop_args(ldr=40), r=BASE + MB) == S["ERR_ALIAS"]
    assert dropout(drop_args(ldr=31), r=BASE + 4 * MB) == S["ERR_SHAPE"]
    assert dropout(drop_args(M=0), x=0, out=0) == dropout_backward(drop_args(C=0), g=0, gx=0) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros((1, 2, 4, 8))
    for call in (lambda: fb.attention_forward(x, x, x), lambda: fb.attention_forward(x[0], x, x),
                 lambda: fb.attention_forward(x, x[..., :4], x), lambda: fb.attention_forward(x, x[:, :, :3], x),
                 lambda: fb.attention_forward(x, x, x.half()), lambda: fb.attention_backward(x, x, x, x, x, x, want=("p",)),
                 lambda: fb.attention_forward(torch.zeros((1, 2, 4, 130)), torch.zeros((1, 2, 4, 130)), x),
                 lambda: fb.group_norm_forward(x, 2), lambda: fb.group_norm_forward(x, 3), lambda: fb.group_norm_forward(x[0, 0, 0], 1),
                 lambda: fb.group_norm_forward(x, 2, activation="tanh"),
                 lambda: fb.group_norm_backward(x, x, x, 2, want=("gate",)),
                 lambda: fb.dropout_forward(x, 0.1, 0), lambda: fb.dropout_forward(x, 0.1, 1 << 64),
                 lambda: fb.dropout_forward(x, 0.1, torch.zeros(2, dtype=torch.int64)),
                 lambda: fb.prepare_attention_forward(x, x, x), lambda: fb.prepare_group_norm_forward(x, 2),
                 lambda: fb.prepare_dropout_forward(x, 0.1, 1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        layer._generator(1.5, 0)


@pytest.mark.parametrize("kw", [dict(q_row=(1 << 20) + 1), dict(q_head=(1 << 20) + 1), dict(o_row=(1 << 20) + 1),
                                dict(o_head=(1 << 20) + 1), dict(H=1024, Hk=1, q_head=1 << 19),
                                dict(H=1024, Hk=1, o_head=1 << 19)])
def test_attention_rows_that_lie_too_far_apart(kw):
    """A tile's rows lie within 32 bits of its first one."""
    assert attention(attention_args(**kw)) == S["ERR_UNSUPPORTED"]
    assert attention_backward(attention_args(**kw)) == S["ERR_UNSUPPORTED"]


def workspace_of(**kw):
    n = fb.layer.ctypes.c_uint64()
    assert fb._packed_call("flashlayer_attention_workspace_size", "PP")(attention_args(**kw), fb.layer.ctypes.byref(n)) == 0
    return n.value


def test_attention_workspace_by_mask():
    """Copies of the keys where a boolean mask is the same for all rows, or rows end inside a granule;
    what a mask says for each row needs none."""
    big = dict(B=1, Lq=4096, Lk=4096, H=32, Hk=32)
    assert workspace_of(**big) == workspace_of(**big, mask=2, mask_row=4096) == workspace_of(**big, mask=1, mask_row=4096) == 0
    keys = workspace_of(**big, mask=1)
    assert keys >= 2 * 32 * 4096 * 32 * 2
    assert workspace_of(**big, mask=1, mask_head=4096) >= keys          # (a head's own rows are its own keys)
    assert workspace_of(**{**big, "Hk": 16}, mask=1, mask_head=4096) == 0   # (heads that share keys differ)
    assert workspace_of(**big, D=31) >= 2 * 32 * 4096 * 32 * 2
    # a workspace that is too small, and none
    args = attention_args(B=1, Lq=40, Lk=4096, H=1, Hk=1)
    need = workspace_of(B=1, Lq=40, Lk=4096, H=1, Hk=1)
    assert need > 0
    far = [BASE + i * (MB << 4) for i in range(5)]
    call = lambda ws, wsb: attention(args, far[0], far[1], far[2], out=far[3], ws=ws, wsb=wsb)
    assert call(far[4], need - 1) == S["ERR_SCRATCH"] and call(0, need) == S["ERR_NULLPTR"]
    assert call(far[3], need) != 0   # (on the output)


def test_a_thread_sees_all_autograd_classes_or_none(monkeypatch):
    """The classes are made on first use, and several threads may be the first."""
    seen = []

    class Watched(dict):
        def update(self, other):
            super().update(other)
            seen.append(set(self))

        def __setitem__(self, k, v):
            super().__setitem__(k, v)
            seen.append(set(self))

    monkeypatch.setattr(layer, "_AUTOGRAD", Watched())
    names = {"attention", "group_norm", "dropout"}
    assert set(layer._autograd_functions()) == names and seen == [names]


def backward_workspace_of(want_q=1, want_kv=1, **kw):
    n = fb.layer.ctypes.c_uint64()
    size = fb._packed_call("flashlayer_attention_backward_workspace_size", "PiiP")
    assert size(attention_args(**kw), want_q, want_kv, fb.layer.ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("kw", [dict(), dict(mask=1), dict(mask=1, mask_row=16), dict(mask=3), dict(D=31), dict(D=31, mask=1),
                                dict(D=128, dtype=0, mask=1)])
def test_a_backward_without_queries_reads_nothing(kw):
    """There is no mask to read then (that of no queries has no address), and nothing to copy: grad_k and
    grad_v are zeros."""
    assert backward_workspace_of(Lq=0, **kw) == 0
    assert backward_workspace_of(Lq=1, **kw) > 0


@pytest.mark.parametrize("kw", [dict(C=0, groups=1), dict(C=0, groups=3), dict(N=0), dict(R=0), dict(C=0, groups=1, R=5000)])
def test_group_norm_without_elements(kw):
    n = fb.layer.ctypes.c_uint64()
    for size in ("flashlayer_group_norm_workspace_size", "flashlayer_group_norm_backward_workspace_size"):
        n.value = 7
        assert fb._packed_call(size, "PP")(group_args(**kw), fb.layer.ctypes.byref(n)) == 0 and n.value == 0
    assert group_norm(group_args(**kw), x=0, y=0, ws=0) == 0
    assert group_norm_backward(group_args(**kw), g=0, x=0, stats=0, gx=0, gw=0, gb=0, ws=0) == 0
