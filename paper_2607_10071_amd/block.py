"""The operators around FlashSCA in an encoder block (``include/block/flashblock.h``):
the matrix product with bias, activation and residual in its epilogue.

As in the package's other calls, this only marshals arguments: every product and
gradient runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import struct

from . import (FlashBevError, _dtype_code, _on_device, _one_device,
               _packed_call, _stream_handle, _workspace)

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}

# The C structures as packed bytes (see the package's other calls).
_PACK_LINEAR = struct.Struct("@6q5if")


class Linear(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("ldr", ctypes.c_int64), ("ldo", ctypes.c_int64), ("ldp", ctypes.c_int64),
                ("K", ctypes.c_int32), ("N", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("scale", ctypes.c_float)]


assert _PACK_LINEAR.size == ctypes.sizeof(Linear)


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
        return (t.numel() // width if width else _product(shape[:-1])), width
    rows, ld = _product(shape[:-1]), width
    if rows and width:
        strides = t.stride()
        if width > 1 and strides[-1] != 1:
            raise ValueError(f"{name}'s last dimension must be contiguous")
        step = None   # elements from one row to the next, and rows below it
        for n, st in zip(reversed(shape[:-1]), reversed(strides[:-1])):
            if n == 1:
                continue
            if step is None:
                ld, step = st, st * n
            elif st != step:
                raise ValueError(f"{name}'s leading dimensions must be rows at one stride")
            else:
                step *= n
        if step is not None and ld < width:
            raise ValueError(f"{name}'s rows must not overlap")
    return rows, ld


def _product(shape) -> int:
    n = 1
    for v in shape:
        n *= v
    return n


def _same(t, name: str, dtype, shape) -> None:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {dtype} [{', '.join(str(int(v)) for v in shape)}]")


def _vector(t, name: str, dtype, n: int) -> int:
    """The address of a contiguous device vector, 0 for None."""
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    _same(t, name, dtype, (n,))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _addr(t) -> int:
    return 0 if t is None else t.data_ptr()


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
                contiguous elements, at any one row stride.
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
    args = _PACK_LINEAR.pack(M, ldx, ldw, ldr, ldo, ldp, K, N, code,
                             code if odt == x.dtype else 0, _act_code(activation), scale)
    dev = _one_device(x, weight, bias, residual, out, pre)
    s = _stream_handle(stream, dev)
    need = _size("flashblock_linear_workspace_size", "PP", args)
    ws = _workspace(need, dev, s) if need else None
    call = _packed_call("flashblock_linear_forward", "PPPPPPPPQP")
    with _on_device(dev):
        rc = call(args, x.data_ptr(), weight.data_ptr(), b, _addr(residual), out.data_ptr(),
                  _addr(pre), _addr(ws), need, s)
    if rc != 0:
        raise FlashBevError(rc, "flashblock_linear_forward")
    return out


def _size(name: str, kinds: str, *args) -> int:
    """A workspace size from the C call ``name``."""
    n = ctypes.c_uint64()
    rc = _packed_call(name, kinds)(*args, ctypes.byref(n))
    if rc != 0:
        raise FlashBevError(rc, name)
    return n.value


def linear_backward(grad_out, x, weight, pre=None, activation="none", scale: float = 1.0,
                    want=("x", "weight", "bias"), grad_x=None, grad_weight=None, grad_bias=None,
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
            given = torch.empty(like, dtype=x.dtype, device=x.device)
            ld[name] = K
        outs[name] = given
    if all(t is None for t in outs.values()):
        return outs
    args = _PACK_LINEAR.pack(M, ldx, ldw, N, ldo, ldp, K, N, code, code if odt == x.dtype else 0, act,
                             scale)
    dev = _one_device(grad_out, x, weight, pre if act else None, *outs.values())
    s = _stream_handle(stream, dev)
    need = _size("flashblock_linear_backward_workspace_size", "PiiiP", args,
                 *(int(outs[k] is not None) for k in ("x", "weight", "bias")))
    ws = _workspace(need, dev, s) if need else None
    call = _packed_call("flashblock_linear_backward", "PPPPPPQPQPPQP")
    with _on_device(dev):
        rc = call(args, grad_out.data_ptr(), x.data_ptr(), weight.data_ptr(),
                  pre.data_ptr() if act else 0, _addr(outs["x"]), ld.get("x", K),
                  _addr(outs["weight"]), ld.get("weight", K), _addr(outs["bias"]), _addr(ws), need, s)
    if rc != 0:
        raise FlashBevError(rc, "flashblock_linear_backward")
    return outs


# ---------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------
_AUTOGRAD = {}


def _as_rows(t):
    """A gradient as it came where its rows are at one stride, else a copy."""
    try:
        _rows(t, "gradient")
        return t
    except ValueError:
        return t.contiguous()


def _autograd_functions():
    """The torch.autograd.Function classes, made on first use."""
    if _AUTOGRAD:
        return _AUTOGRAD
    import torch
    from torch.autograd.function import once_differentiable

    class _Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, residual, activation, scale, out_dtype):
            pre = None
            if _act_code(activation) and any(ctx.needs_input_grad[:3]):
                pre = torch.empty((*x.shape[:-1], weight.shape[0]), dtype=x.dtype, device=x.device)
            out = linear_forward(x, weight, bias, activation, residual, scale, out_dtype=out_dtype,
                                 pre=pre)
            ctx.save_for_backward(x, weight, pre)
            ctx.meta = (activation, scale)
            return out

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_out):
            x, weight, pre = ctx.saved_tensors
            activation, scale = ctx.meta
            needs = ctx.needs_input_grad
            want = tuple(k for k, n in zip(("x", "weight", "bias"), needs) if n)
            r = dict.fromkeys(("x", "weight", "bias"))
            if want:
                r = linear_backward(_as_rows(grad_out), x, weight, pre, activation, scale, want)
            return (r["x"], r["weight"], r["bias"], grad_out if needs[3] else None, None, None, None)

    _AUTOGRAD["linear"] = _Linear
    return _AUTOGRAD


def linear_autograd(x, weight, bias=None, activation="none", residual=None, scale: float = 1.0,
                    out_dtype=None):
    """``linear_forward`` as a differentiable function of x, weight, bias and
    residual; the gradients are ``linear_backward``'s, computed only for the inputs
    that need them."""
    return _autograd_functions()["linear"].apply(x, weight, bias, residual, activation, scale,
                                                 out_dtype)
