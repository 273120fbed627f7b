"""The operators around FlashSCA in an encoder block (``include/block/flashblock.h``):
the matrix product with bias, activation and residual in its epilogue, and the
norms before and after a block with its gate and residual scale.

As in the package's other calls, this only marshals arguments: every product, norm
and gradient runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import functools
import struct

from . import (FlashBevError, _dtype_code, _on_device, _on_stream, _one_device, _Prepared,
               _packed_call, _stream_handle, _workspace)

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
NORMS = {"none": 0, "layer": 1, "rms": 2}
LD_MAX = 1 << 20   # FLASHBLOCK_LD_MAX

# The C structures as packed bytes (see the package's other calls).
_PACK_LINEAR = struct.Struct("@6q5if")
_PACK_NORM = struct.Struct("@6q6i2f")
_PACK_VECTORS = struct.Struct("@5P")


class Linear(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("ldr", ctypes.c_int64), ("ldo", ctypes.c_int64), ("ldp", ctypes.c_int64),
                ("K", ctypes.c_int32), ("N", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("scale", ctypes.c_float)]


class Norm(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldr", ctypes.c_int64),
                ("lds", ctypes.c_int64), ("ldy", ctypes.c_int64), ("groups", ctypes.c_int64),
                ("C", ctypes.c_int32), ("dtype", ctypes.c_int32), ("stream_dtype", ctypes.c_int32),
                ("param_dtype", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("post_norm", ctypes.c_int32), ("eps", ctypes.c_float), ("scale", ctypes.c_float)]


assert _PACK_LINEAR.size == ctypes.sizeof(Linear) and _PACK_NORM.size == ctypes.sizeof(Norm)


def _rows(t, name: str):
    """(rows, row stride) of a device tensor [..., width] whose leading dimensions
    are one sequence of rows at one stride, its last one contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    shape = t.shape
    if not shape:
        raise ValueError(f"{name} must have at least one dimension")
    width = shape[-1]
    if t.is_contiguous():
        if len(shape) == 2:
            return shape[0], width
        return (t.numel() // width if width else _product(shape[:-1])), width
    return _strided_rows(t, name)


def _strided_rows(t, name: str):
    shape, strides = t.shape, t.stride()
    width = shape[-1]
    rows, ld = _product(shape[:-1]), width
    if not rows or not width:
        return rows, ld
    if width > 1 and strides[-1] != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    step = None   # elements from one row to the next, then over all rows so far
    for n, st in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n == 1:
            continue
        if step is None:
            ld, step = st, st * n
        elif st != step:
            raise ValueError(f"{name}'s leading dimensions must be rows at one stride")
        else:
            step *= n
    if ld < width:
        raise ValueError(f"{name}'s rows must not overlap")
    return rows, ld


def _near(t, ld: int, device, s: int):
    """(t, its row stride), or a copy, made on the stream ``s`` of the call that reads
    it, where the library does not take rows so far apart."""
    if ld <= LD_MAX:
        return t, ld
    with _on_stream(device, s):
        return t.contiguous(), t.shape[-1]


def _no_copies(*lds) -> None:
    if max(lds) > LD_MAX:
        raise ValueError(f"a prepared call takes rows at most {LD_MAX} elements apart")


def _product(shape) -> int:
    n = 1
    for v in shape:
        n *= v
    return n


def _same(t, name: str, dtype, shape) -> None:
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} [{', '.join(str(int(v)) for v in shape)}]")


def _vector(t, name: str, dtype, n: int) -> int:
    """The address of a contiguous device vector, 0 for None."""
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} vector [{n}]")
    return t.data_ptr()


def _addr(t) -> int:
    return 0 if t is None else t.data_ptr()


_LINEAR_GRADS = ("x", "weight", "bias")
_VECTORS = ("gate", "weight", "bias", "post_weight", "post_bias")
_NORM_INPUTS = ("x", "residual", *_VECTORS)


def _wanted(want, names) -> None:
    for k in want:
        if k not in names:
            raise ValueError(f"want takes {names}")


def _act_code(activation) -> int:
    try:
        return ACTIVATIONS[activation or "none"]
    except KeyError:
        raise ValueError(f"activation must be one of {tuple(ACTIVATIONS)}") from None


def _out_type(out_dtype, x):
    """out's dtype: the input's, or float32."""
    import torch

    if out_dtype is None:
        return x.dtype
    if out_dtype != x.dtype and out_dtype != torch.float32:
        raise ValueError(f"out_dtype must be {x.dtype} or torch.float32")
    return out_dtype


def _weight(weight, x):
    """(N, row stride) of a weight [N, K] in x's dtype."""
    if weight.dim() != 2 or not x.dim() or weight.shape[1] != x.shape[-1]:
        raise ValueError("weight must be [N, K] with x [..., K]")
    if weight.dtype != x.dtype:
        raise ValueError(f"weight must be {x.dtype}")
    return weight.shape[0], _rows(weight, "weight")[1]


def linear_forward(x, weight, bias=None, activation="none", residual=None, scale: float = 1.0,
                   out=None, out_dtype=None, pre=None, stream=None):
    """residual + scale * act(x weight^T + bias) on the GPU.

    x           CUDA tensor [..., K] (float32, float16 or bfloat16): rows of
                contiguous elements, at any one row stride.  (Of inputs whose rows
                lie more than LD_MAX = 2^20 elements apart a copy is read; outputs
                must lie closer.)
    weight      [N, K] in x's dtype, rows likewise.
    bias        optional [N] in x's dtype.
    activation  "none", "relu", "gelu" (erf), "gelu_tanh" or "silu".
    residual    optional [..., N] in the output's dtype; may be ``out`` itself.
    scale       factor of the activated product.
    out         optional [..., N] to write into.
    out_dtype   x's dtype (default), or torch.float32: FlashSCA's offsets and
                logits, say, which it reads as float32.
    pre         optional [..., N] in x's dtype to write the sums before the
                activation into (the backward of an activation reads them).
    stream      as in the package's other calls.

    Sums are float32, each output is rounded once.  Returns ``out``; the call is
    asynchronous.
    """
    return _linear_forward(x, weight, bias, activation, residual, scale, out, out_dtype, pre, stream)[0]


def _linear_forward(x, weight, bias, activation, residual, scale, out, out_dtype, pre, stream):
    """linear_forward's (out, sizes for _linear_gradients)."""
    call, args, keep, out, sizes = _linear_call(x, weight, bias, activation, residual, scale, out,
                                                out_dtype, pre, stream, False)
    with _on_device(sizes[-1]):
        rc = call(*args)
    if rc != 0:
        raise FlashBevError(rc, "flashblock_linear_forward")
    return out, sizes


def prepare_linear_forward(x, weight, bias=None, activation="none", residual=None, scale: float = 1.0,
                           out=None, pre=None, stream=None) -> _Prepared:
    """``linear_forward`` with every argument fixed (``out`` given): a callable that
    enqueues the same call again (same tensors, same stream).  A workspace, where the
    sizes need one, is allocated once, here."""
    if out is None:
        raise ValueError("a prepared call needs out")
    call, args, keep, _, sizes = _linear_call(x, weight, bias, activation, residual, scale, out, None, pre,
                                              stream, True)
    return _Prepared(call, args, keep, "flashblock_linear_forward", sizes[-1])


def _linear_call(x, weight, bias, activation, residual, scale, out, out_dtype, pre, stream, again):
    """(C call, its arguments, the tensors they point into, out, sizes for
    _linear_gradients).  ``again``: the call may be made more than once."""
    import torch

    M, ldx = _rows(x, "x")
    code = _dtype_code(x)
    N, ldw = _weight(weight, x)
    K = x.shape[-1]
    shape = (*x.shape[:-1], N)
    odt = _out_type(out.dtype if out is not None and out_dtype is None else out_dtype, x)
    if out is None:
        out = torch.empty(shape, dtype=odt, device=x.device)
        ldo = N
    else:
        _same(out, "out", odt, shape)
        ldo = _rows(out, "out")[1]
    ldr = ldp = N
    if residual is not None:
        _same(residual, "residual", odt, shape)
        ldr = _rows(residual, "residual")[1]
    if pre is not None:
        _same(pre, "pre", x.dtype, shape)
        ldp = _rows(pre, "pre")[1]
    b = _vector(bias, "bias", x.dtype, N)
    act, out_code = _act_code(activation), code if odt == x.dtype else 0
    dev = _one_device(x, weight, bias, residual, out, pre)
    s = _stream_handle(stream, dev)
    if ldx > LD_MAX or ldw > LD_MAX or (ldr > LD_MAX and residual is not out):
        if again:
            _no_copies(ldx, ldw, ldr)
        x, ldx = _near(x, ldx, dev, s)
        weight, ldw = _near(weight, ldw, dev, s)
        if residual is not None:
            residual, ldr = _near(residual, ldr, dev, s)
    args = _PACK_LINEAR.pack(M, ldx, ldw, ldr, ldo, ldp, K, N, code, out_code, act, scale)
    need = _linear_need(M, K, N, code)
    ws = _workspace(need, dev, s) if need else None
    return (_packed_call("flashblock_linear_forward", "PPPPPPPPQP"),
            (args, x.data_ptr(), weight.data_ptr(), b, _addr(residual), out.data_ptr(), _addr(pre),
             _addr(ws), need, s), (x, weight, bias, residual, out, pre, ws), out,
            (M, ldx, ldw, K, N, code, out_code, act, scale, dev))


def _size(name: str, kinds: str, *args) -> int:
    """A workspace size from the C call ``name``."""
    n = ctypes.c_uint64()
    rc = _packed_call(name, kinds)(*args, ctypes.byref(n))
    if rc != 0:
        raise FlashBevError(rc, name)
    return n.value


# Workspace sizes depend on the sizes and types alone, which calls repeat.


@functools.lru_cache(maxsize=4096)
def _linear_need(M: int, K: int, N: int, code: int) -> int:
    return _size("flashblock_linear_workspace_size", "PP",
                 _PACK_LINEAR.pack(M, K, K, N, N, N, K, N, code, code, 0, 1.0))


@functools.lru_cache(maxsize=4096)
def _linear_backward_need(M: int, K: int, N: int, code: int, out_code: int, act: int, x: bool,
                          weight: bool, bias: bool) -> int:
    return _size("flashblock_linear_backward_workspace_size", "PiiiP",
                 _PACK_LINEAR.pack(M, K, K, N, N, N, K, N, code, out_code, act, 1.0), x, weight, bias)


@functools.lru_cache(maxsize=4096)
def _norm_need(M: int, groups: int, C: int, flags) -> int:
    return _size("flashblock_norm_backward_workspace_size", "PPP",
                 _PACK_NORM.pack(M, C, C, C, C, groups, C, 0, 0, 0, 1, 1, 1.0, 1.0),
                 _PACK_VECTORS.pack(*flags))


def linear_backward(grad_out, x, weight, pre=None, activation="none", scale: float = 1.0,
                    want=_LINEAR_GRADS, grad_x=None, grad_weight=None, grad_bias=None,
                    stream=None):
    """The gradients of ``linear_forward`` for ``grad_out`` [..., N] (in the
    output's dtype): a dict with "x", "weight" and "bias", in x's dtype, None for
    those not in ``want`` and not passed in.  The residual's gradient is
    ``grad_out`` itself.  ``pre`` is the forward's, needed with an activation.

    d = scale act'(pre) grad_out is formed in float32 and, where it is not
    grad_out itself, rounded to x's dtype for the products (a float16 d must
    stay within float16's range); the bias gradient sums it unrounded.
    """
    import torch

    _wanted(want, _LINEAR_GRADS)
    M, ldx = _rows(x, "x")
    code = _dtype_code(x)
    N, ldw = _weight(weight, x)
    K = x.shape[-1]
    shape = (*x.shape[:-1], N)
    odt = _out_type(grad_out.dtype, x)
    _same(grad_out, "grad_out", odt, shape)
    ldo = _rows(grad_out, "grad_out")[1]
    act, ldp = _act_code(activation), N
    if act:
        if pre is None:
            raise ValueError("the backward of an activation needs pre")
        _same(pre, "pre", x.dtype, shape)
        ldp = _rows(pre, "pre")[1]
    outs, ld = {}, {}
    for name, given, like in (("x", grad_x, x.shape), ("weight", grad_weight, weight.shape),
                              ("bias", grad_bias, (N,))):
        if given is not None:
            _same(given, "grad_" + name, x.dtype, like)
            ld[name] = _rows(given, "grad_" + name)[1]
            if name == "bias" and not given.is_contiguous():
                raise ValueError("grad_bias must be contiguous")
        elif name in want:
            given = (torch.empty(like, dtype=x.dtype, device=x.device) if name == "bias"
                     else torch.empty_like(x if name == "x" else weight,
                                           memory_format=torch.contiguous_format))
            ld[name] = K
        outs[name] = given
    if all(t is None for t in outs.values()):
        return outs
    dev = _one_device(grad_out, x, weight, pre if act else None, *outs.values())
    if max(ldo, ldx, ldw, ldp) > LD_MAX:
        s = _stream_handle(stream, dev)
        grad_out, ldo = _near(grad_out, ldo, dev, s)
        x, ldx = _near(x, ldx, dev, s)
        weight, ldw = _near(weight, ldw, dev, s)
        if act:
            pre, ldp = _near(pre, ldp, dev, s)
    sizes = (M, ldx, ldw, K, N, code, code if odt == x.dtype else 0, act, scale, dev)
    _linear_gradients(sizes, grad_out, ldo, x, weight, pre if act else None, ldp, outs["x"],
                      ld.get("x", K), outs["weight"], ld.get("weight", K), outs["bias"], stream)
    return outs


def _linear_gradients(sizes, grad_out, ldo, x, weight, pre, ldp, grad_x, ldgx, grad_weight, ldgw,
                      grad_bias, stream):
    """The backward call on checked tensors."""
    M, ldx, ldw, K, N, code, out_code, act, scale, dev = sizes
    args = _PACK_LINEAR.pack(M, ldx, ldw, N, ldo, ldp, K, N, code, out_code, act, scale)
    s = _stream_handle(stream, dev)
    need = _linear_backward_need(M, K, N, code, out_code, act, grad_x is not None,
                                 grad_weight is not None, grad_bias is not None)
    ws = _workspace(need, dev, s) if need else None
    call = _packed_call("flashblock_linear_backward", "PPPPPPQPQPPQP")
    with _on_device(dev):
        rc = call(args, grad_out.data_ptr(), x.data_ptr(), weight.data_ptr(), _addr(pre),
                  _addr(grad_x), ldgx, _addr(grad_weight), ldgw, _addr(grad_bias), _addr(ws), need, s)
    if rc != 0:
        raise FlashBevError(rc, "flashblock_linear_backward")


def _norm_code(kind, name: str) -> int:
    try:
        return NORMS[kind or "none"]
    except KeyError:
        raise ValueError(f"{name} must be one of {tuple(NORMS)}") from None


def _norm_vectors(x, gate, weight, bias, post_weight, post_bias):
    """(samples, dtype code, packed addresses) of a norm call's vectors."""
    import torch

    C = x.shape[-1]
    groups, dtype = 1, None
    for t in (gate, weight, bias, post_weight, post_bias):
        if t is None:
            continue
        if dtype is None:
            dtype = t.dtype
            if dtype != x.dtype and dtype != torch.float32:
                raise ValueError(f"gate, weights and biases must be {x.dtype} or torch.float32")
        elif t.dtype != dtype:
            raise ValueError("gate, weights and biases must have one dtype")
    if gate is not None and gate.dim() == 2:
        if x.dim() < 2 or tuple(gate.shape) != (x.shape[0], C):
            raise ValueError(f"gate must be [{C}] or, one row for each of x's first dimension, "
                             f"[{x.shape[0]}, {C}]")
        if not gate.is_cuda or not gate.is_contiguous():
            raise ValueError("gate must be a contiguous device tensor")
        groups = gate.shape[0]
        g = gate.data_ptr()
    else:
        g = _vector(gate, "gate", dtype, C)
    ptrs = (g, _vector(weight, "weight", dtype, C), _vector(bias, "bias", dtype, C),
            _vector(post_weight, "post_weight", dtype, C), _vector(post_bias, "post_bias", dtype, C))
    return groups or 1, dtype, _PACK_VECTORS.pack(*ptrs)


def _adds_nothing(x, residual, gate, scale, post_norm, out_s) -> bool:
    """Whether s is x itself."""
    return residual is None and gate is None and scale == 1.0 and not _norm_code(
        post_norm, "post_norm") and (out_s is None)


def norm_forward(x, weight=None, bias=None, residual=None, gate=None, scale: float = 1.0,
                 norm="layer", post_norm=None, post_weight=None, post_bias=None, eps: float = 1e-5,
                 out=None, out_s=None, stream=None):
    """The norms around a block, on the GPU:

        u = N_post(x) post_weight + post_bias        (x without ``post_norm``)
        s = residual + (scale * gate) * u
        y = N(s) weight + bias                       (None without ``norm``)

    x            CUDA tensor [..., C] (float32, float16 or bfloat16): a block's
                 output, rows at any one row stride (far ones as in
                 ``linear_forward``).
    weight, bias, post_weight, post_bias
                 optional [C], in x's dtype or float32 (one for all vectors).
    residual     optional [..., C] in x's dtype or float32: the stream that the
                 block is added to.  s has its dtype (x's without it).
    gate         optional [C], or [G, C] with x [G, ..., C]: a row for each
                 sample.
    scale        residual scale.
    norm, post_norm
                 "layer", "rms" or None; one of them at least.
    eps          of both norms.
    out, out_s   optional tensors to write y and s into; ``out_s`` may be
                 ``residual``.
    stream       as in the package's other calls.

    N(s) reads s as it is stored.  Returns (y, s); s is x itself where nothing
    changes it.  Asynchronous.
    """
    return _norm_forward(x, weight, bias, residual, gate, scale, norm, post_norm, post_weight, post_bias,
                         eps, out, out_s, stream)[:2]


def _norm_forward(x, weight, bias, residual, gate, scale, norm, post_norm, post_weight, post_bias, eps,
                  out, out_s, stream):
    """norm_forward's (y, s, sizes for _norm_gradients)."""
    call, args, y, s, sizes, keep = _norm_call(x, weight, bias, residual, gate, scale, norm, post_norm,
                                               post_weight, post_bias, eps, out, out_s, stream, False)
    with _on_device(sizes[-1]):
        rc = call(*args)
    if rc != 0:
        raise FlashBevError(rc, "flashblock_norm_forward")
    return y, s, sizes


def prepare_norm_forward(x, weight=None, bias=None, residual=None, gate=None, scale: float = 1.0,
                         norm="layer", post_norm=None, post_weight=None, post_bias=None,
                         eps: float = 1e-5, out=None, out_s=None, stream=None) -> _Prepared:
    """``norm_forward`` with every argument fixed (``out`` given with a norm, ``out_s``
    where anything is added or there is no norm): a callable that enqueues the same call
    again (same tensors, same stream)."""
    if (out is None and _norm_code(norm, "norm")) or (out_s is None and not _adds_nothing(
            x, residual, gate, scale, post_norm, out_s)):
        raise ValueError("a prepared call needs out and out_s")
    call, args, _, _, sizes, keep = _norm_call(x, weight, bias, residual, gate, scale, norm, post_norm,
                                               post_weight, post_bias, eps, out, out_s, stream, True)
    return _Prepared(call, args, keep, "flashblock_norm_forward", sizes[-1])


def _norm_call(x, weight, bias, residual, gate, scale, norm, post_norm, post_weight, post_bias, eps, out,
               out_s, stream, again):
    """(C call, its arguments, y, s, sizes for _norm_gradients, the tensors that the
    arguments point into).  ``again``: the call may be made more than once."""
    import torch

    M, ldx = _rows(x, "x")
    code = _dtype_code(x)
    kind, post = _norm_code(norm, "norm"), _norm_code(post_norm, "post_norm")
    C = x.shape[-1]
    groups, pdt, vectors = _norm_vectors(x, gate, weight, bias, post_weight, post_bias)
    sdt = residual.dtype if residual is not None else x.dtype
    if sdt != x.dtype and sdt != torch.float32:
        raise ValueError(f"residual must be {x.dtype} or torch.float32")
    ldr = lds = ldy = C
    if residual is not None:
        _same(residual, "residual", sdt, x.shape)
        ldr = _rows(residual, "residual")[1]
    same = kind and _adds_nothing(x, residual, gate, scale, post_norm, out_s)
    if out_s is not None:
        _same(out_s, "out_s", sdt, x.shape)
        lds = _rows(out_s, "out_s")[1]
    elif not same:
        out_s = torch.empty_like(x, dtype=sdt, memory_format=torch.contiguous_format)
    if not kind:
        if out is not None:
            raise ValueError("out needs a norm")
    elif out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        _same(out, "out", x.dtype, x.shape)
        ldy = _rows(out, "out")[1]
    types = (code, code if sdt == x.dtype else 0, code if pdt is None or pdt == x.dtype else 0, kind, post,
             eps, scale)
    dev = _one_device(x, weight, bias, residual, gate, post_weight, post_bias, out, out_s)
    s = _stream_handle(stream, dev)
    stays = x if same else out_s
    if ldx > LD_MAX or (ldr > LD_MAX and residual is not out_s):
        if again:
            _no_copies(ldx, ldr)
        x, ldx = _near(x, ldx, dev, s)
        if residual is not None:
            residual, ldr = _near(residual, ldr, dev, s)
    args = _PACK_NORM.pack(M, ldx, ldr, lds, ldy, groups, C, *types)
    return (_packed_call("flashblock_norm_forward", "PPPPPPP"),
            (args, vectors, x.data_ptr(), _addr(residual), _addr(out_s), _addr(out), s), out, stays,
            (M, ldx, ldx if same else lds, groups, C, types, dev),
            (x, weight, bias, residual, gate, post_weight, post_bias, out, out_s))


def norm_backward(grad_y, grad_s, x, s, weight=None, gate=None, scale: float = 1.0, norm="layer",
                  post_norm=None, post_weight=None, post_bias=None, eps: float = 1e-5, want=("x",),
                  stream=None):
    """The gradients of ``norm_forward`` for ``grad_y`` (in x's dtype) and
    ``grad_s`` (in the stream's), either of which may be None.

    x, s     the forward's input and its second result.
    want     which of "x", "residual", "gate", "weight", "bias", "post_weight" and
             "post_bias"; the vectors' gradients come in the vectors' dtype
             (x's, where no vector is given).  Each vector asked for takes at least
             one float32 row of workspace for every sample of a gate [G, C].

    Returns a dict of those gradients.  Asynchronous.
    """
    import torch

    M, ldx = _rows(x, "x")
    code = _dtype_code(x)
    kind, post = _norm_code(norm, "norm"), _norm_code(post_norm, "post_norm")
    C = x.shape[-1]
    groups, pdt, vectors = _norm_vectors(x, gate, weight, None, post_weight, post_bias)
    pdt = pdt or x.dtype
    sdt = s.dtype
    if sdt != x.dtype and sdt != torch.float32:
        raise ValueError(f"s must be {x.dtype} or torch.float32")
    _same(s, "s", sdt, x.shape)
    lds = _rows(s, "s")[1]
    ldgy = ldgs = C
    if grad_y is not None:
        _same(grad_y, "grad_y", x.dtype, x.shape)
        ldgy = _rows(grad_y, "grad_y")[1]
    if grad_s is not None:
        _same(grad_s, "grad_s", sdt, x.shape)
        ldgs = _rows(grad_s, "grad_s")[1]
    _wanted(want, _NORM_INPUTS)
    if not want:
        return {}
    dev = _one_device(grad_y, grad_s, x, s, weight, gate, post_weight, post_bias)
    if max(ldx, lds, ldgy, ldgs) > LD_MAX:
        st = _stream_handle(stream, dev)
        x, ldx = _near(x, ldx, dev, st)
        s, lds = _near(s, lds, dev, st)
        if grad_y is not None:
            grad_y, ldgy = _near(grad_y, ldgy, dev, st)
        if grad_s is not None:
            grad_s, ldgs = _near(grad_s, ldgs, dev, st)
    types = (code, code if sdt == x.dtype else 0, code if pdt == x.dtype else 0, kind, post, eps, scale)
    return _norm_gradients((M, ldx, lds, groups, C, types, dev), grad_y, ldgy, grad_s, ldgs, x, s, gate,
                           vectors, pdt, want, stream)


def _norm_gradients(sizes, grad_y, ldgy, grad_s, ldgs, x, s, gate, vectors, pdt, want, stream):
    """The backward call on checked tensors: a dict of the gradients in ``want``."""
    import torch

    M, ldx, lds, groups, C, types, dev = sizes
    outs = {}
    for k in want:
        if k == "x":
            outs[k] = torch.empty_like(x, memory_format=torch.contiguous_format)
        elif k == "residual":
            outs[k] = torch.empty_like(s, memory_format=torch.contiguous_format)
        else:
            outs[k] = torch.empty((C,) if k != "gate" or gate is None else gate.shape, dtype=pdt,
                                  device=dev)
    args = _PACK_NORM.pack(M, ldx, ldgs, lds, ldgy, groups, C, *types)
    grads = _PACK_VECTORS.pack(*[_addr(outs.get(k)) for k in _VECTORS])
    st = _stream_handle(stream, dev)
    need = _norm_need(M, groups, C, tuple([k in outs for k in _VECTORS]))
    ws = _workspace(need, dev, st) if need else None
    call = _packed_call("flashblock_norm_backward", "PPPPPPPQPQPPQP")
    with _on_device(dev):
        rc = call(args, vectors, _addr(grad_y), _addr(grad_s), x.data_ptr(), s.data_ptr(),
                  _addr(outs.get("x")), C, _addr(outs.get("residual")), C, grads, _addr(ws), need, st)
    if rc != 0:
        raise FlashBevError(rc, "flashblock_norm_backward")
    return outs


# ---------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------
_AUTOGRAD = {}


def _as_rows(t, width: int):
    """(a gradient as it came, its row stride) where its rows are at one stride that
    the library takes, else of a copy."""
    if not t.is_contiguous():
        try:
            ld = _strided_rows(t, "gradient")[1]
            if ld <= LD_MAX:
                return t, ld
        except ValueError:
            pass
        t = t.contiguous()
    return t, width


def _restored(t, name: str, dtype, shape, device):
    """A saved tensor as it came back.  Hooks on saved tensors hand over anything:
    the kernels read it as what was saved, so another type, size or place is refused.
    Its strides are its own."""
    if t.dtype != dtype or t.shape != shape or t.device != device:
        raise ValueError(f"{name} was saved as {dtype} {tuple(shape)} on {device} and came back as "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _autograd_functions():
    """The torch.autograd.Function classes, made on first use."""
    if _AUTOGRAD:
        return _AUTOGRAD
    import torch
    from torch.autograd.function import once_differentiable

    # The gradients that autograd hands over fit the forward's outputs, so only
    # their strides are looked at.

    def linear_grads(ctx, grad_out):
        x, weight, pre = ctx.saved_tensors
        needs = ctx.needs_input_grad
        residual = grad_out if needs[3] else None
        if not (needs[0] or needs[1] or needs[2]):
            return None, None, None, residual, None, None, None
        (M, K, N, *rest), shape, dtype = ctx.sizes
        dev = rest[-1]
        g, ldo = _as_rows(grad_out, N)
        x, ldx = _as_rows(_restored(x, "x", dtype, shape, dev), K)
        weight, ldw = _as_rows(_restored(weight, "weight", dtype, (N, K), dev), K)
        ldp = N
        if pre is not None:
            pre, ldp = _as_rows(_restored(pre, "pre", dtype, (*shape[:-1], N), dev), N)
        gx = torch.empty_like(x, memory_format=torch.contiguous_format) if needs[0] else None
        gw = torch.empty_like(weight, memory_format=torch.contiguous_format) if needs[1] else None
        gb = torch.empty(N, dtype=x.dtype, device=x.device) if needs[2] else None
        _linear_gradients((M, ldx, ldw, K, N, *rest), g, ldo, x, weight, pre, ldp, gx, K, gw, K, gb, None)
        return gx, gw, gb, residual, None, None, None

    def norm_grads(ctx, grad_y, grad_s):
        x, s, weight, gate, post_weight, post_bias = ctx.saved_tensors
        if grad_y is None and grad_s is None:
            return (None,) * 11
        (M, groups, C, types, dev), want, shape, gate_shape, (dt, sdt, pdt) = ctx.sizes
        ldgy = ldgs = C
        x, ldx = _as_rows(_restored(x, "x", dt, shape, dev), C)
        s, lds = (x, ldx) if s is None else _as_rows(_restored(s, "s", sdt, shape, dev), C)
        if grad_y is not None:
            grad_y, ldgy = _as_rows(grad_y, C)
        if grad_s is not None:
            grad_s, ldgs = _as_rows(grad_s, C)
        # (contiguous for the call, and alive until it is enqueued)
        gate, weight, post_weight, post_bias = [
            None if t is None else _restored(t, name, pdt, like, dev).contiguous()
            for t, name, like in ((gate, "gate", gate_shape), (weight, "weight", (C,)),
                                  (post_weight, "post_weight", (C,)), (post_bias, "post_bias", (C,)))]
        vectors = _PACK_VECTORS.pack(_addr(gate), _addr(weight), 0, _addr(post_weight), _addr(post_bias))
        r = _norm_gradients((M, ldx, lds, groups, C, types, dev), grad_y, ldgy, grad_s, ldgs, x, s, gate,
                            vectors, pdt, want, None)
        return (*map(r.get, _NORM_INPUTS), None, None, None, None)

    # the wrapper, which refuses a second derivative, only where a graph of the
    # gradients is made (it takes some 10 us)
    linear_once, norm_once = once_differentiable(linear_grads), once_differentiable(norm_grads)

    class _Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, residual, activation, scale, out_dtype):
            # in x's type: float32 would be twice the bytes to write and read again, for
            # gradients 0.00235 off in place of 0.00241 (bfloat16, gelu)
            pre = None
            if _act_code(activation) and any(ctx.needs_input_grad[:3]):
                pre = torch.empty((*x.shape[:-1], weight.shape[0]), dtype=x.dtype, device=x.device)
            out, sizes = _linear_forward(x, weight, bias, activation, residual, scale, None, out_dtype,
                                         pre, None)
            ctx.sizes = sizes[:1] + sizes[3:], x.shape, x.dtype   # without the strides
            ctx.save_for_backward(x, weight, pre)
            return out

        @staticmethod
        def backward(ctx, grad_out):
            return (linear_once if torch.is_grad_enabled() else linear_grads)(ctx, grad_out)

    class _Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, gate, weight, bias, post_weight, post_bias, scale, norm,
                    post_norm, eps):
            ctx.set_materialize_grads(False)
            y, s, sizes = _norm_forward(x, weight, bias, residual, gate, scale, norm, post_norm,
                                        post_weight, post_bias, eps, None, None, None)
            sdt = s.dtype
            if s is x:
                s = None
            ctx.save_for_backward(x, s, weight, gate, post_weight, post_bias)
            pdt = x.dtype
            for t in (gate, weight, bias, post_weight, post_bias):
                if t is not None:
                    pdt = t.dtype
                    break
            want = [k for k, n in zip(_NORM_INPUTS, ctx.needs_input_grad) if n]
            ctx.sizes = (sizes[:1] + sizes[3:], want, x.shape, None if gate is None else gate.shape,
                         (x.dtype, sdt, pdt))   # without the strides
            return y, s

        @staticmethod
        def backward(ctx, grad_y, grad_s):
            return (norm_once if torch.is_grad_enabled() else norm_grads)(ctx, grad_y, grad_s)

    # both at once: another thread takes what it finds here as the whole
    _AUTOGRAD.update({"linear": _Linear, "norm": _Norm})
    return _AUTOGRAD


def linear_autograd(x, weight, bias=None, activation="none", residual=None, scale: float = 1.0,
                    out_dtype=None):
    """``linear_forward`` as a differentiable function of x, weight, bias and
    residual; the gradients are ``linear_backward``'s, computed only for the inputs
    that need them.  (In a HIP graph capture forward and gradients together, by
    torch.autograd.grad, with no eager graph of the same leaves alive.)"""
    return _autograd_functions()["linear"].apply(x, weight, bias, residual, activation, scale,
                                                 out_dtype)


def norm_autograd(x, weight=None, bias=None, residual=None, gate=None, scale: float = 1.0,
                  norm="layer", post_norm=None, post_weight=None, post_bias=None, eps: float = 1e-5):
    """``norm_forward`` as a differentiable function of x, residual, gate, weights
    and biases; the gradients are ``norm_backward``'s, computed only for the inputs
    that need them.  (In a HIP graph as for ``linear_autograd``.)"""
    y, s = _autograd_functions()["norm"].apply(x, residual, gate, weight, bias, post_weight, post_bias,
                                               scale, norm, post_norm, eps)
    return y, x if s is None else s
