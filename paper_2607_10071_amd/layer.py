"""The operators that complete a layer of an encoder or a decoder around FlashSCA and the
linear and norm operators (``include/block/flashlayer.h``): attention of queries to the states
of an encoder of another length, group norm with an activation on channels-last maps, and
dropout from a counter-based generator onto a residual.

As in the package's other calls, this only marshals arguments: every score, norm, random word
and gradient is computed in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import functools
import struct

from . import (FlashBevError, _dtype_code, _on_device, _on_stream, _one_device, _Prepared, _packed_call,
               _stream_handle, _workspace)
from .block import (_act_code, _addr, _as_rows, _near, _no_copies, _restored, _rows, _same, _size, _vector,
                    _wanted, LD_MAX)

HEAD_MAX = 128   # FLASHLAYER_HEAD_MAX

# The C structures as packed bytes (see the package's other calls).
_PACK_ATTENTION = struct.Struct("@15q8if4x")
_PACK_GROUP_NORM = struct.Struct("@4q5if")
_PACK_DROPOUT = struct.Struct("@4q2Qd3if")


class Attention(ctypes.Structure):
    _fields_ = [(f"{t}_{d}", ctypes.c_int64) for t, ds in
                (("q", "batch row head"), ("k", "batch row head"), ("v", "batch row head"),
                 ("o", "batch row head"), ("mask", "batch head row")) for d in ds.split()] \
        + [(n, ctypes.c_int32) for n in ("B", "Lq", "Lk", "H", "Hk", "D", "dtype", "mask")] \
        + [("scale", ctypes.c_float)]


class GroupNorm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("N", "R", "ldx", "ldy")] \
        + [(n, ctypes.c_int32) for n in ("C", "groups", "dtype", "param_dtype", "act")] \
        + [("eps", ctypes.c_float)]


class Dropout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("M", "ldx", "ldr", "ldo")] \
        + [("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("p", ctypes.c_double)] \
        + [(n, ctypes.c_int32) for n in ("C", "dtype", "stream_dtype")] + [("scale", ctypes.c_float)]


assert _PACK_ATTENTION.size == ctypes.sizeof(Attention)
assert _PACK_GROUP_NORM.size == ctypes.sizeof(GroupNorm)
assert _PACK_DROPOUT.size == ctypes.sizeof(Dropout)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
MASKS = {"none": 0, "bool": 1, "add": 2, "add_f32": 3}
_ATTENTION_GRADS = ("q", "k", "v")


def _heads(t, name: str, shape):
    """(batch, row, head) strides of a device tensor [B, L, heads, D] of ``shape`` whose
    channels are contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must be [{', '.join(str(int(v)) for v in shape)}]")
    s = t.stride()
    if s[3] != 1 and shape[3] > 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return s[0], s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0   # (no step along one element)


def _near_heads(t, strides, share: int, dev, s: int, again: bool = False):
    """(t, its strides), or a copy, made on the stream ``s`` of the call that reads it, where
    the library does not take rows so far apart.  share: of the query heads that one head of
    the states serves (queries and their gradients), or 0 (states, whose heads may be anywhere)."""
    _, row, head = strides
    if row <= LD_MAX and (share == 0 or (head <= LD_MAX and share * head <= 1 << 28)):
        return t, strides
    if again:
        raise ValueError(f"a prepared call takes rows and heads at most {LD_MAX} elements apart")
    with _on_stream(dev, s):
        t = t.contiguous()
    return t, _heads(t, "the copy", t.shape)


def _sizes(q, k, v):
    """(B, Lq, Lk, H, Hk, D) of an attention's inputs."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q must be [B, Lq, H, D], k and v [B, Lk, Hk, D]")
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    if k.shape[0] != B or k.shape[3] != D:
        raise ValueError("q and k must have the same batches and channels")
    if (H % Hk if Hk else H):
        raise ValueError("q's heads must be a multiple of k's")
    if D > HEAD_MAX:
        raise ValueError(f"heads must have at most {HEAD_MAX} channels")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError(f"k and v must be {q.dtype}")
    return B, Lq, Lk, H, Hk, D


def _mask(mask, q, B, H, Lq, Lk):
    """(type, batch, head and row strides) of a mask that broadcasts to [B, H, Lq, Lk]."""
    import torch

    if mask is None:
        return 0, 0, 0, 0
    if not mask.is_cuda:
        raise ValueError("mask must be a device tensor")
    if mask.dtype is torch.bool:
        kind = 1
    elif mask.dtype is q.dtype:
        kind = 2
    elif mask.dtype is torch.float32:
        kind = 3
    else:
        raise ValueError(f"mask must be torch.bool, {q.dtype} or torch.float32")
    if mask.requires_grad and torch.is_grad_enabled():
        raise ValueError("the mask gets no gradient")
    shape = mask.shape
    if len(shape) != 4 or shape[3] != Lk or any(n != 1 and n != m for n, m in zip(shape, (B, H, Lq))):
        raise ValueError(f"mask must be [{B} or 1, {H} or 1, {Lq} or 1, {Lk}]")
    s = mask.stride()
    if s[3] != 1 and Lk > 1:
        raise ValueError("mask's keys must be contiguous")
    return kind, s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0


def _lengths(key_lengths, B: int) -> int:
    import torch

    if key_lengths is not None and key_lengths.dtype is not torch.int32:
        raise ValueError("key_lengths must be torch.int32")
    return _vector(key_lengths, "key_lengths", torch.int32, B)


def _scale(scale, D: int) -> float:
    return (D or 1) ** -0.5 if scale is None else scale


# (whether a mask has heads and rows of its own decides how it is read)
@functools.lru_cache(maxsize=4096)
def _attention_need(B, Lq, Lk, H, Hk, D, code, kind, heads: bool, rows: bool) -> int:
    return _size("flashlayer_attention_workspace_size", "PP",
                 _PACK_ATTENTION.pack(*[0] * 13, heads, rows, B, Lq, Lk, H, Hk, D, code, kind, 1.0))


@functools.lru_cache(maxsize=4096)
def _attention_backward_need(B, Lq, Lk, H, Hk, D, code, kind, heads: bool, rows: bool, q: bool, kv: bool) -> int:
    return _size("flashlayer_attention_backward_workspace_size", "PiiP",
                 _PACK_ATTENTION.pack(*[0] * 13, heads, rows, B, Lq, Lk, H, Hk, D, code, kind, 1.0), q, kv)


def attention_forward(q, k, v, mask=None, key_lengths=None, scale=None, out=None, rest=None, stats=None,
                      stream=None):
    """softmax(scale q k^T + mask) v for each head, on the GPU.

    q            CUDA tensor [B, Lq, H, D] (float32, float16 or bfloat16), D at most 128,
                 its channels contiguous, any other strides: a product's [B, Lq, H D] rows
                 seen as heads, say (long calls are up to twice as fast where all rows begin at
                 multiples of 16 bytes).  Where rows, or the heads of q, lie more than 2^20 elements
                 apart a copy is read (prepared calls and outputs are refused).
    k, v         [B, Lk, Hk, D] in q's dtype, strides likewise (the halves of one projection,
                 a cache longer than what it holds); query head h reads head h // (H / Hk).
    mask         optional [B or 1, H or 1, Lq or 1, Lk], its keys contiguous: torch.bool (False
                 leaves the place out), or q's dtype or float32, added to the scaled score.  It
                 gets no gradient.  A boolean mask that is the same for all queries and heads leaves
                 its keys out altogether: their k and v may hold anything.
    key_lengths  optional int32 device vector [B]: keys from key_lengths[b] on are left out and
                 not read.
    scale        of the scores, D ** -0.5 by default; positive.
    out          optional [B, Lq, H, D] to write into, strides as q's.
    rest         optional contiguous [B, Lq, H, D] in q's dtype: what rounding took from out.
    stats        optional contiguous float32 [B, H, Lq, 2]: each row's reference score and the
                 logarithm of its sum of exponentials.
    stream       as in the package's other calls.

    Scores, softmax and sums are float32; p is rounded to q's dtype for its product with v.  A
    query that sees no key gets zeros.  Returns ``out``; asynchronous.
    """
    call, args, keep, out, dev = _attention_call(q, k, v, mask, key_lengths, scale, out, rest, stats, stream, False)
    with _on_device(dev):
        rc = call(*args)
    if rc != 0:
        raise FlashBevError(rc, "flashlayer_attention_forward")
    return out


def prepare_attention_forward(q, k, v, mask=None, key_lengths=None, scale=None, out=None, stats=None,
                              stream=None) -> _Prepared:
    """``attention_forward`` with every argument fixed (``out`` given): a callable that enqueues the
    same call again (same tensors, same stream).  A workspace, where the sizes need one, is
    allocated once, here."""
    if out is None:
        raise ValueError("a prepared call needs out")
    call, args, keep, _, dev = _attention_call(q, k, v, mask, key_lengths, scale, out, None, stats, stream, True)
    return _Prepared(call, args, keep, "flashlayer_attention_forward", dev)


def _attention_call(q, k, v, mask, key_lengths, scale, out, rest, stats, stream, again):
    """(C call, its arguments, the tensors they point into, out, device)."""
    import torch

    sizes = B, Lq, Lk, H, Hk, D = _sizes(q, k, v)
    code = _dtype_code(q)
    qs, ks, vs = _heads(q, "q", q.shape), _heads(k, "k", k.shape), _heads(v, "v", k.shape)
    kind, mb, mh, mr = _mask(mask, q, B, H, Lq, Lk)
    lengths = _lengths(key_lengths, B)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif out.dtype != q.dtype:
        raise ValueError(f"out must be {q.dtype}")
    os = _heads(out, "out", q.shape)
    if rest is not None:
        _same(rest, "rest", q.dtype, q.shape)
    if stats is not None:
        _same(stats, "stats", torch.float32, (B, H, Lq, 2))
    for t, name in ((rest, "rest"), (stats, "stats")):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    dev = _one_device(q, k, v, mask, key_lengths, out, rest, stats)
    s = _stream_handle(stream, dev)
    (q, qs), (k, ks), (v, vs) = (_near_heads(t, st, share, dev, s, again) for t, st, share in
                                 ((q, qs, H // Hk if Hk else 1), (k, ks, 0), (v, vs, 0)))
    args = _PACK_ATTENTION.pack(*qs, *ks, *vs, *os, mb, mh, mr, *sizes, code, kind, _scale(scale, D))
    need = _attention_need(*sizes, code, kind, mh != 0, mr != 0)
    ws = _workspace(need, dev, s) if need else None
    return (_packed_call("flashlayer_attention_forward", "PPPPPPPPPPQP"),
            (args, q.data_ptr(), k.data_ptr(), v.data_ptr(), _addr(mask), lengths, out.data_ptr(),
             _addr(rest), _addr(stats), _addr(ws), need, s),
            (q, k, v, mask, key_lengths, out, rest, stats, ws), out, dev)


def attention_backward(grad_out, q, k, v, out, stats, mask=None, key_lengths=None, scale=None,
                       want=_ATTENTION_GRADS, rest=None, stream=None):
    """The gradients of ``attention_forward`` for ``grad_out`` [B, Lq, H, D] in q's dtype: a dict
    with "q", "k" and "v" in q's dtype, None for those not in ``want``.

    out, stats   the forward's, contiguous.
    rest         the forward's, optional: with it grad_out . out, which a row's gradients are
                 differences from, is formed of all of out's digits.

    p and its gradient are rounded to q's dtype for their products (float16 ones after scaling by
    powers of two, so that small ones keep their digits).
    """
    import torch

    _wanted(want, _ATTENTION_GRADS)
    B, Lq, Lk, H, Hk, D = _sizes(q, k, v)
    _same(out, "out", q.dtype, q.shape)
    _same(grad_out, "grad_out", q.dtype, q.shape)
    _same(stats, "stats", torch.float32, (B, H, Lq, 2))
    if rest is not None:
        _same(rest, "rest", q.dtype, q.shape)
    for t, name in ((out, "out"), (stats, "stats"), (rest, "rest")):
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous device tensor")
    got = _attention_gradients(grad_out, q, k, v, out, rest, stats, mask, key_lengths, scale, "q" in want,
                               "k" in want or "v" in want, stream)
    return {n: t if n in want else None for n, t in zip(_ATTENTION_GRADS, got)}


def _attention_gradients(grad_out, q, k, v, out, rest, stats, mask, key_lengths, scale, want_q, want_kv,
                         stream):
    """(grad_q, grad_k, grad_v), None where they are not wanted."""
    import torch

    if not want_q and not want_kv:
        return None, None, None
    sizes = B, Lq, Lk, H, Hk, D = _sizes(q, k, v)
    code = _dtype_code(q)
    qs, ks, vs = _heads(q, "q", q.shape), _heads(k, "k", k.shape), _heads(v, "v", k.shape)
    gs = _heads(grad_out, "grad_out", q.shape)
    kind, mb, mh, mr = _mask(mask, q, B, H, Lq, Lk)
    lengths = _lengths(key_lengths, B)
    dev = _one_device(grad_out, q, k, v, out, rest, stats, mask, key_lengths)
    s = _stream_handle(stream, dev)
    share = H // Hk if Hk else 1
    (q, qs), (grad_out, gs), (k, ks), (v, vs) = (_near_heads(t, st, n, dev, s) for t, st, n in
                                                 ((q, qs, share), (grad_out, gs, share), (k, ks, 0), (v, vs, 0)))
    gq = torch.empty(q.shape, dtype=q.dtype, device=dev) if want_q else None
    gk, gv = ((torch.empty(k.shape, dtype=q.dtype, device=dev) for _ in "kv") if want_kv else (None, None))
    args = _PACK_ATTENTION.pack(*qs, *ks, *vs, *gs, mb, mh, mr, *sizes, code, kind, _scale(scale, D))
    need = _attention_backward_need(*sizes, code, kind, mh != 0, mr != 0, want_q, want_kv)
    ws = _workspace(need, dev, s) if need else None
    call = _packed_call("flashlayer_attention_backward", "PPPPPPPPPPPPPPQP")
    with _on_device(dev):
        rc = call(args, grad_out.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), _addr(mask), lengths,
                  out.data_ptr(), _addr(rest), stats.data_ptr(), _addr(gq), _addr(gk), _addr(gv), _addr(ws),
                  need, s)
    if rc != 0:
        raise FlashBevError(rc, "flashlayer_attention_backward")
    return gq, gk, gv


# ---------------------------------------------------------------------------
# group norm
# ---------------------------------------------------------------------------
_GROUP_NORM_INPUTS = ("x", "weight", "bias")


@functools.lru_cache(maxsize=4096)
def _group_norm_need(N, R, C, groups, code, backward: bool) -> int:
    return _size("flashlayer_group_norm_backward_workspace_size" if backward
                 else "flashlayer_group_norm_workspace_size", "PP",
                 _PACK_GROUP_NORM.pack(N, R, C, C, C, groups, code, code, 0, 1.0))


def _group_sizes(x, groups):
    """(samples, positions, channels, row stride) of x [N, ..., C]."""
    if x.dim() < 2:
        raise ValueError("x must be [N, ..., C]")
    C = x.shape[-1]
    if groups < 1 or C % groups:
        raise ValueError(f"groups must divide the {C} channels")
    M, ld = _rows(x, "x")
    N = x.shape[0]
    return N, M // N if N else 0, C, ld


def _group_vectors(x, weight, bias):
    """(dtype, weight's address, bias's)."""
    import torch

    C, dtype = x.shape[-1], None
    for t in (weight, bias):
        if t is not None:
            if t.dtype != x.dtype and t.dtype != torch.float32:
                raise ValueError(f"weight and bias must be {x.dtype} or torch.float32")
            if dtype is not None and t.dtype != dtype:
                raise ValueError("weight and bias must have one dtype")
            dtype = t.dtype
    dtype = dtype or x.dtype
    return dtype, _vector(weight, "weight", dtype, C), _vector(bias, "bias", dtype, C)


def group_norm_forward(x, groups: int, weight=None, bias=None, activation="none", eps: float = 1e-5, out=None,
                       stats=None, stream=None):
    """act(N(x) weight + bias) on the GPU, N over each sample's positions and each of ``groups``
    groups of consecutive channels.

    x             CUDA tensor [N, ..., C] (float32, float16 or bfloat16), channels last: a
                  feature map [N, H, W, C], say; rows at any one stride (far ones as in
                  ``linear_forward``).
    weight, bias  optional [C], in x's dtype or float32 (one for both).
    activation    "none", "relu", "gelu" (erf), "gelu_tanh" or "silu".
    out           optional tensor like x to write into.
    stats         optional contiguous float32 [N, groups, 2] for the means and
                  1 / sqrt(variance + eps), which the backward reads.
    stream        as in the package's other calls.

    Statistics are float32, formed of differences from means; each output is rounded once.
    Returns ``out``; asynchronous.
    """
    return _group_norm_forward(x, groups, weight, bias, activation, eps, out, stats, stream)


def _group_norm_forward(x, groups, weight, bias, activation, eps, out, stats, stream):
    call, args, keep, out, dev = _group_norm_call(x, groups, weight, bias, activation, eps, out, stats, stream,
                                                  False)
    with _on_device(dev):
        rc = call(*args)
    if rc != 0:
        raise FlashBevError(rc, "flashlayer_group_norm_forward")
    return out


def prepare_group_norm_forward(x, groups: int, weight=None, bias=None, activation="none", eps: float = 1e-5,
                               out=None, stats=None, stream=None) -> _Prepared:
    """``group_norm_forward`` with every argument fixed (``out`` given): a callable that enqueues
    the same call again (same tensors, same stream, one workspace)."""
    if out is None:
        raise ValueError("a prepared call needs out")
    call, args, keep, _, dev = _group_norm_call(x, groups, weight, bias, activation, eps, out, stats, stream,
                                                True)
    return _Prepared(call, args, keep, "flashlayer_group_norm_forward", dev)


def _group_norm_call(x, groups, weight, bias, activation, eps, out, stats, stream, again):
    """(C call, its arguments, the tensors they point into, out, device)."""
    import torch

    N, R, C, ldx = _group_sizes(x, groups)
    code, act = _dtype_code(x), _act_code(activation)
    pdt, w, b = _group_vectors(x, weight, bias)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        ldy = C
    else:
        _same(out, "out", x.dtype, x.shape)
        ldy = _rows(out, "out")[1]
    if stats is not None:
        _same(stats, "stats", torch.float32, (N, groups, 2))
        if not stats.is_contiguous():
            raise ValueError("stats must be contiguous")
    dev = _one_device(x, weight, bias, out, stats)
    s = _stream_handle(stream, dev)
    if ldx > LD_MAX:
        if again:
            _no_copies(ldx)
        x, ldx = _near(x, ldx, dev, s)
    args = _PACK_GROUP_NORM.pack(N, R, ldx, ldy, C, groups, code, code if pdt == x.dtype else 0, act, eps)
    need = _group_norm_need(N, R, C, groups, code, False)
    ws = _workspace(need, dev, s) if need else None
    return (_packed_call("flashlayer_group_norm_forward", "PPPPPPPQP"),
            (args, x.data_ptr(), w, b, out.data_ptr(), _addr(stats), _addr(ws), need, s),
            (x, weight, bias, out, stats, ws), out, dev)


def group_norm_backward(grad_y, x, stats, groups: int, weight=None, bias=None, activation="none", want=("x",),
                        stream=None):
    """The gradients of ``group_norm_forward`` for ``grad_y`` (like x), of its input and ``stats``:
    a dict of those in ``want``, of "x", "weight" and "bias" (weight's and bias's in their dtype,
    x's where there is neither).  With an activation bias is read too."""
    import torch

    _wanted(want, _GROUP_NORM_INPUTS)
    N, R, C, ldx = _group_sizes(x, groups)
    _same(grad_y, "grad_y", x.dtype, x.shape)
    _same(stats, "stats", torch.float32, (N, groups, 2))
    if not stats.is_cuda or not stats.is_contiguous():
        raise ValueError("stats must be a contiguous device tensor")
    pdt, w, b = _group_vectors(x, weight, bias)
    act = _act_code(activation)
    ldg = _rows(grad_y, "grad_y")[1]
    dev = _one_device(grad_y, x, stats, weight, bias)
    if max(ldx, ldg) > LD_MAX:
        s = _stream_handle(stream, dev)
        x, ldx = _near(x, ldx, dev, s)
        grad_y, ldg = _near(grad_y, ldg, dev, s)
    return _group_norm_gradients((N, R, C, groups, act, dev), grad_y, ldg, x, ldx, stats, w, b, pdt, want, stream)


def _group_norm_gradients(sizes, grad_y, ldg, x, ldx, stats, w, b, pdt, want, stream):
    """The backward call on checked tensors."""
    import torch

    if not want:
        return {}
    N, R, C, groups, act, dev = sizes
    code = _dtype_code(x)
    outs = {n: torch.empty(x.shape, dtype=x.dtype, device=dev) if n == "x"
            else torch.empty(C, dtype=pdt, device=dev) for n in want}
    args = _PACK_GROUP_NORM.pack(N, R, ldx, ldg, C, groups, code, code if pdt == x.dtype else 0, act, 1.0)
    s = _stream_handle(stream, dev)
    need = _group_norm_need(N, R, C, groups, code, True)
    ws = _workspace(need, dev, s) if need else None
    call = _packed_call("flashlayer_group_norm_backward", "PPPPPPPPPPQP")
    with _on_device(dev):
        rc = call(args, grad_y.data_ptr(), x.data_ptr(), stats.data_ptr(), w, b, _addr(outs.get("x")),
                  _addr(outs.get("weight")), _addr(outs.get("bias")), _addr(ws), need, s)
    if rc != 0:
        raise FlashBevError(rc, "flashlayer_group_norm_backward")
    return outs


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
def _generator(seed, offset):
    """(seed, offset, device words) of a call: whole numbers of 64 bits, or a device tensor that
    holds both."""
    import torch

    if isinstance(seed, torch.Tensor):
        if offset != 0:
            raise ValueError("the tensor of the generator holds its offset too")
        if not seed.is_cuda or seed.dtype != torch.int64 or seed.shape != (2,) or not seed.is_contiguous():
            raise ValueError("seed must be a whole number or a contiguous torch.int64 device tensor [2]")
        return 0, 0, seed
    for v, name in ((seed, "seed"), (offset, "offset")):
        if not isinstance(v, int):
            raise TypeError(f"{name} must be a whole number")
        if not -(1 << 63) <= v < 1 << 64:
            raise ValueError(f"{name} must fit 64 bits")
    return seed & 0xFFFFFFFFFFFFFFFF, offset & 0xFFFFFFFFFFFFFFFF, None


def dropout_forward(x, p: float, seed, offset: int = 0, residual=None, scale: float = 1.0, out=None,
                    stream=None):
    """residual + scale * x / (1 - p) where an element is kept, residual elsewhere, on the GPU.

    x         CUDA tensor [..., C] (float32, float16 or bfloat16): rows at any one stride (far
              ones as in ``linear_forward``).
    p         the share that is dropped, 0 to 1.
    seed      whole number of 64 bits: the generator's key.  Or an int64 device tensor [2] that
              holds the key and the offset, which the kernel reads: a captured graph, whose
              arguments are fixed, drops anew after an update of it.
    offset    whole number of 64 bits, another for each step and place of a program.
    residual  optional [..., C] in x's dtype or float32: the stream that x is added to.  The
              result has its dtype (x's without it).  It may be ``out`` itself.
    scale     residual scale.
    out       optional tensor to write into.
    stream    as in the package's other calls.

    Element e of x in row-major order is dropped where word e % 4 of block e / 4 of Philox 4x32-10
    is below round(p 2^32): the same elements whatever x's type and strides and however often;
    nothing of the mask is stored.  Returns ``out``; asynchronous.
    """
    call, args, keep, out, dev = _dropout_call(x, p, seed, offset, residual, scale, out, stream, False)
    with _on_device(dev):
        rc = call(*args)
    if rc != 0:
        raise FlashBevError(rc, "flashlayer_dropout_forward")
    return out


def prepare_dropout_forward(x, p: float, seed, offset: int = 0, residual=None, scale: float = 1.0, out=None,
                            stream=None) -> _Prepared:
    """``dropout_forward`` with every argument fixed (``out`` given): a callable that enqueues the same
    call again (same tensors, same stream; with a device tensor as the seed, of what it then holds)."""
    if out is None:
        raise ValueError("a prepared call needs out")
    call, args, keep, _, dev = _dropout_call(x, p, seed, offset, residual, scale, out, stream, True)
    return _Prepared(call, args, keep, "flashlayer_dropout_forward", dev)


def _dropout_call(x, p, seed, offset, residual, scale, out, stream, again):
    """(C call, its arguments, the tensors they point into, out, device)."""
    import torch

    M, ldx = _rows(x, "x")
    code = _dtype_code(x)
    C = x.shape[-1]
    seed, offset, state = _generator(seed, offset)
    sdt = x.dtype if residual is None else residual.dtype
    if residual is None and out is not None:
        sdt = out.dtype
    if sdt != x.dtype and sdt != torch.float32:
        raise ValueError(f"residual and out must be {x.dtype} or torch.float32")
    ldr = ldo = C
    if residual is not None:
        _same(residual, "residual", sdt, x.shape)
        ldr = _rows(residual, "residual")[1]
    if out is None:
        out = torch.empty(x.shape, dtype=sdt, device=x.device)
    else:
        _same(out, "out", sdt, x.shape)
        ldo = _rows(out, "out")[1]
    dev = _one_device(x, residual, out, state)
    s = _stream_handle(stream, dev)
    if ldx > LD_MAX or (ldr > LD_MAX and residual is not out):
        if again:
            _no_copies(ldx, ldr)
        x, ldx = _near(x, ldx, dev, s)
        if residual is not None:
            residual, ldr = _near(residual, ldr, dev, s)
    args = _PACK_DROPOUT.pack(M, ldx, ldr, ldo, seed, offset, p, C, code, code if sdt == x.dtype else 0, scale)
    return (_packed_call("flashlayer_dropout_forward", "PPPPPP"),
            (args, x.data_ptr(), _addr(residual), _addr(state), out.data_ptr(), s), (x, residual, state, out), out,
            dev)


def dropout_backward(grad_out, p: float, seed, offset: int = 0, scale: float = 1.0, dtype=None, stream=None):
    """The gradient of ``dropout_forward`` with respect to x for ``grad_out`` [..., C] (in the
    result's dtype): scale / (1 - p) grad_out where the element was kept, in ``dtype`` (x's;
    grad_out's by default).  The residual's gradient is ``grad_out`` itself."""
    seed, offset, state = _generator(seed, offset)
    return _dropout_gradient(grad_out, p, seed, offset, state, scale, dtype or grad_out.dtype, stream)


def _dropout_gradient(grad_out, p, seed, offset, state, scale, dtype, stream):
    import torch

    M, ldg = _rows(grad_out, "grad_out")
    C = grad_out.shape[-1]
    if grad_out.dtype != dtype and grad_out.dtype != torch.float32:
        raise ValueError(f"grad_out must be {dtype} or torch.float32")
    dev = _one_device(grad_out, state)
    s = _stream_handle(stream, dev)
    grad_out, ldg = _near(grad_out, ldg, dev, s)
    gx = torch.empty(grad_out.shape, dtype=dtype, device=dev)
    code = _dtype_code(gx)
    args = _PACK_DROPOUT.pack(M, C, C, ldg, seed, offset, p, C, code, code if grad_out.dtype == dtype else 0, scale)
    call = _packed_call("flashlayer_dropout_backward", "PPPPP")
    with _on_device(dev):
        rc = call(args, grad_out.data_ptr(), _addr(state), gx.data_ptr(), s)
    if rc != 0:
        raise FlashBevError(rc, "flashlayer_dropout_backward")
    return gx


# ---------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------
_AUTOGRAD = {}


def _unit_channels(t):
    """A gradient or saved tensor as it came, or a copy where its channels are not contiguous."""
    return t if t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def _autograd_functions():
    """The torch.autograd.Function classes, made on first use."""
    if _AUTOGRAD:
        return _AUTOGRAD
    import torch
    from torch.autograd.function import once_differentiable

    def attention_grads(ctx, grad_out):
        q, k, v, out, rest, stats, mask, key_lengths = ctx.saved_tensors
        needs = ctx.needs_input_grad
        (qs, ks, mask_like, lengths_like), dt, dev, scale = ctx.sizes
        q, k, v = (_unit_channels(_restored(t, name, dt, like, dev))
                   for t, name, like in ((q, "q", qs), (k, "k", ks), (v, "v", ks)))
        out = _restored(out, "out", dt, qs, dev).contiguous()
        if rest is not None:
            rest = _restored(rest, "rest", dt, qs, dev).contiguous()
        stats = _restored(stats, "stats", torch.float32, (qs[0], qs[2], qs[1], 2), dev).contiguous()
        if mask is not None:
            mask = _unit_channels(_restored(mask, "mask", *mask_like, dev))
        if key_lengths is not None:
            key_lengths = _restored(key_lengths, "key_lengths", torch.int32, lengths_like, dev).contiguous()
        gq, gk, gv = _attention_gradients(_unit_channels(grad_out), q, k, v, out, rest, stats, mask, key_lengths,
                                          scale, needs[0], needs[1] or needs[2], None)
        return gq, gk if needs[1] else None, gv if needs[2] else None, None, None, None

    def group_norm_grads(ctx, grad_y):
        x, stats, weight, bias = ctx.saved_tensors
        (N, R, C, groups, act, dev), dt, pdt, shape, want = ctx.sizes
        g, ldg = _as_rows(grad_y, C)
        x, ldx = _as_rows(_restored(x, "x", dt, shape, dev), C)
        stats = _restored(stats, "stats", torch.float32, (N, groups, 2), dev).contiguous()
        # (contiguous for the call, and alive until it is enqueued)
        weight, bias = [None if t is None else _restored(t, n, pdt, (C,), dev).contiguous()
                        for t, n in ((weight, "weight"), (bias, "bias"))]
        r = _group_norm_gradients((N, R, C, groups, act, dev), g, ldg, x, ldx, stats, _addr(weight), _addr(bias),
                                  pdt, want, None)
        return r.get("x"), None, r.get("weight"), r.get("bias"), None, None

    def dropout_grads(ctx, grad_out):
        p, seed, offset, scale, dt, dev = ctx.sizes
        state = None
        if ctx.saved_tensors:
            state = _restored(ctx.saved_tensors[0], "seed", torch.int64, (2,), dev).contiguous()
        g = _as_rows(grad_out, grad_out.shape[-1])[0] if ctx.needs_input_grad[0] else None
        gx = None if g is None else _dropout_gradient(g, p, seed, offset, state, scale, dt, None)
        return gx, None, None, None, grad_out if ctx.needs_input_grad[4] else None, None

    # the wrapper, which refuses a second derivative, only where a graph of the gradients is
    # made (see the linear and norm operators')
    attention_once, group_norm_once, dropout_once = map(once_differentiable,
                                                        (attention_grads, group_norm_grads, dropout_grads))

    class _Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, mask, key_lengths, scale):
            rest = stats = None
            if any(ctx.needs_input_grad[:3]):
                # 16-bit outputs keep what rounding took: a row's gradients are differences
                # from grad_out . out, which a softmax over few states makes nearly all of
                if q.dtype != torch.float32:
                    rest = torch.empty(q.shape, dtype=q.dtype, device=q.device)
                stats = torch.empty((q.shape[0], q.shape[2], q.shape[1], 2), dtype=torch.float32, device=q.device)
            out = attention_forward(q, k, v, mask, key_lengths, scale, None, rest, stats)
            ctx.save_for_backward(q, k, v, out, rest, stats, mask, key_lengths)
            ctx.sizes = ((q.shape, k.shape, None if mask is None else (mask.dtype, mask.shape),
                          None if key_lengths is None else key_lengths.shape), q.dtype, q.device, scale)
            return out

        @staticmethod
        def backward(ctx, grad_out):
            return (attention_once if torch.is_grad_enabled() else attention_grads)(ctx, grad_out)

    class _GroupNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, groups, weight, bias, activation, eps):
            stats = torch.empty((x.shape[0], groups, 2), dtype=torch.float32, device=x.device) \
                if x.dim() > 1 and groups > 0 else None
            out = _group_norm_forward(x, groups, weight, bias, activation, eps, None, stats, None)
            needs = ctx.needs_input_grad
            C, N = x.shape[-1], x.shape[0]
            pdt = weight.dtype if weight is not None else bias.dtype if bias is not None else x.dtype
            want = [n for n, i in zip(_GROUP_NORM_INPUTS, (0, 2, 3)) if needs[i]]
            ctx.save_for_backward(x, stats, weight, bias)
            ctx.sizes = ((N, x.numel() // (N * C) if N * C else 0, C, groups, _act_code(activation), x.device),
                         x.dtype, pdt, x.shape, want)
            return out

        @staticmethod
        def backward(ctx, grad_y):
            return (group_norm_once if torch.is_grad_enabled() else group_norm_grads)(ctx, grad_y)

    class _Dropout(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, p, seed, offset, residual, scale):
            out = dropout_forward(x, p, seed, offset, residual, scale)
            seed, offset, state = _generator(seed, offset)
            if state is not None:
                ctx.save_for_backward(state)
            ctx.sizes = p, seed, offset, scale, x.dtype, x.device
            return out

        @staticmethod
        def backward(ctx, grad_out):
            return (dropout_once if torch.is_grad_enabled() else dropout_grads)(ctx, grad_out)

    # all at once: another thread takes what it finds here as the whole
    _AUTOGRAD.update({"attention": _Attention, "group_norm": _GroupNorm, "dropout": _Dropout})
    return _AUTOGRAD


def attention_autograd(q, k, v, mask=None, key_lengths=None, scale=None):
    """``attention_forward`` as a differentiable function of q, k and v; the gradients are
    ``attention_backward``'s, computed only for the inputs that need them.  (In a HIP graph as
    for ``linear_autograd``.)"""
    if mask is not None and mask.requires_grad:
        raise ValueError("the mask gets no gradient")
    return _autograd_functions()["attention"].apply(q, k, v, mask, key_lengths, scale)


def group_norm_autograd(x, groups: int, weight=None, bias=None, activation="none", eps: float = 1e-5):
    """``group_norm_forward`` as a differentiable function of x, weight and bias; the gradients are
    ``group_norm_backward``'s, computed only for the inputs that need them.  (In a HIP graph as
    for ``linear_autograd``.)"""
    return _autograd_functions()["group_norm"].apply(x, groups, weight, bias, activation, eps)


def dropout_autograd(x, p: float, seed, offset: int = 0, residual=None, scale: float = 1.0):
    """``dropout_forward`` as a differentiable function of x and residual.  The backward draws the
    same words again; a device tensor as the seed must not change before it.  (In a HIP graph
    as for ``linear_autograd``.)"""
    return _autograd_functions()["dropout"].apply(x, p, seed, offset, residual, scale)
