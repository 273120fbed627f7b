"""Plain float64 forms of attention, group norm and dropout, and how far off the kernels'
results may be (bounds counted from roundings, none of them measured)."""
import math

import torch

U32 = 2.0 ** -24   # half a step of float32


def half(dtype) -> float:
    """The largest relative error of one rounding to ``dtype``."""
    return torch.finfo(dtype).eps / 2


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def scores(q, k, scale, mask=None, key_lengths=None):
    """Masked scores [B, H, Lq, Lk] in float64."""
    q, k = q.detach().double().transpose(1, 2), k.detach().double().transpose(1, 2)
    share = q.shape[1] // max(1, k.shape[1])
    # keys that are left out altogether may hold anything
    out = torch.zeros((q.shape[0], 1, 1, k.shape[2]), dtype=torch.bool, device=q.device)
    if key_lengths is not None:
        ends = key_lengths.clamp(0, k.shape[2])[:, None, None, None]
        out = out | (torch.arange(k.shape[2], device=q.device) >= ends)
    if mask is not None and mask.dtype == torch.bool:
        out = out | ~mask
    k = k.repeat_interleave(share, 1)
    if out.shape[2] == 1:
        k = k.masked_fill(out.transpose(2, 3), 0.0)
    s = scale * torch.matmul(q, k.transpose(2, 3).contiguous())
    size = scale * torch.matmul(q.abs(), k.abs().transpose(2, 3).contiguous())
    if mask is not None and mask.dtype != torch.bool:
        s = s + mask.double()
        size = size + torch.where(mask.abs() < 1e30, mask.double().abs(), 0.0)
    return s.masked_fill(out, -math.inf), size, out


def attention(q, k, v, scale=None, mask=None, key_lengths=None, grad_out=None):
    """({name: float64 result}, {name: bound}) of out, and with ``grad_out`` of grad_q, grad_k and
    grad_v, for results in q's dtype."""
    D, h = q.shape[-1], half(q.dtype)
    scale = D ** -0.5 if scale is None else scale
    s, size, out_of = scores(q, k, scale, mask, key_lengths)
    v64 = v.detach().double().transpose(1, 2)
    share = q.shape[2] // max(1, k.shape[2])
    v64 = v64.repeat_interleave(share, 1)
    k64 = k.detach().double().transpose(1, 2).repeat_interleave(share, 1)
    if out_of.shape[2] == 1:
        v64 = v64.masked_fill(out_of.transpose(2, 3), 0.0)
        k64 = k64.masked_fill(out_of.transpose(2, 3), 0.0)
    top = s.amax(-1, keepdim=True) if s.shape[-1] else s.new_full((*s.shape[:-1], 1), -math.inf)
    seen = top > -math.inf
    p = torch.exp(s - torch.where(seen, top, 0.0)) * seen
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
    peak = p.amax(-1, keepdim=True) if p.shape[-1] else torch.zeros_like(top)
    o = torch.matmul(p, v64)
    n = max(2, s.shape[-1])
    # A score: D products and sums of magnitude `size` in float32 (a block of the matrix units
    # rounds at most once a product), its scaling, difference and exponential some 8 roundings more.
    # A weight's relative error is the scores' and the sum's; its rounding to 16 bits h, and as
    # much in the sum that it is divided by.
    ds = torch.where(p > 0, size, 0.0).amax(-1, keepdim=True) * (D + 4) * U32 * 2 if n else 0.0
    rel = 2 * (ds + 8 * U32) + (2 * h if q.dtype != torch.float32 else 0.0) + 2 * n * U32
    # float16 below its normal numbers: half a step is 2^-25, of weights whose largest is at
    # least one; of dS of a row over 8 |g|; of p and dS of all rows brought to at least 1 / 2 and 1 / 16
    tiny = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    size_o = torch.matmul(p, v64.abs())
    err_o = size_o * rel + n * tiny * peak * v64.abs().amax(-2, keepdim=True) if n and v64.shape[-2] else size_o * 0
    res = {"out": o.transpose(1, 2)}
    tol = {"out": (err_o + h * o.abs() + _floor(q.dtype)).transpose(1, 2)}
    if grad_out is None:
        return res, tol
    g = grad_out.detach().double().transpose(1, 2)
    dp = torch.matmul(g, v64.transpose(2, 3).contiguous())
    delta = (g * o).sum(-1, keepdim=True)
    d = p * (dp - delta)
    # errors of dp, of delta (out's error; with what its rounding took, no more) and of dS
    err_dp = torch.matmul(g.abs(), v64.abs().transpose(2, 3).contiguous()) * (D + 4) * U32
    err_delta = (g.abs() * err_o).sum(-1, keepdim=True) + (g * o).abs().sum(-1, keepdim=True) * ((D + 8) * U32 + h * h)
    norm = g.square().sum(-1, keepdim=True).sqrt()
    err_d = d.abs() * (rel + 2 * h + 8 * U32) + p * (err_dp + err_delta) * (1 + rel)
    rows = max(1, s.shape[2]) * share
    flat = (peak * norm).reshape(q.shape[0], k.shape[2], -1).amax(-1) if s.numel() else None

    def heads(t):
        return t.unflatten(1, (k.shape[2], share)).sum(2).transpose(1, 2)

    kt, gt = k64, g
    q64 = q.detach().double().transpose(1, 2)
    res["grad_q"] = scale * torch.matmul(d, kt)
    tol["grad_q"] = scale * (torch.matmul(err_d + n * U32 * d.abs(), kt.abs())
                             + n * tiny * 8 * peak * norm * kt.abs().amax(-2, keepdim=True))
    res["grad_k"] = scale * torch.matmul(d.transpose(2, 3).contiguous(), q64)
    tol["grad_k"] = scale * torch.matmul((err_d + rows * U32 * d.abs()).transpose(2, 3).contiguous(), q64.abs())
    res["grad_v"] = torch.matmul(p.transpose(2, 3).contiguous(), gt)
    tol["grad_v"] = torch.matmul((p * (rel + h + rows * U32)).transpose(2, 3).contiguous(), gt.abs())
    res["grad_q"], tol["grad_q"] = res["grad_q"].transpose(1, 2), tol["grad_q"].transpose(1, 2)
    for name in ("grad_k", "grad_v"):
        res[name], tol[name] = heads(res[name]), heads(tol[name])
    if tiny:   # the largest factors of the rows, at least an eighth of one after scaling by powers of two
        most = flat[:, None, :, None]
        tol["grad_k"] = tol["grad_k"] + scale * rows * tiny * 16 * most * q64.abs().amax()
        tol["grad_v"] = tol["grad_v"] + rows * tiny * 2 * peak.reshape(q.shape[0], k.shape[2], -1).amax(-1)[:, None, :, None] * gt.abs().amax()
    for name in ("grad_q", "grad_k", "grad_v"):
        tol[name] = tol[name] + h * res[name].abs() + _floor(q.dtype)
    return res, tol


def _floor(dtype):
    """Half the smallest step of ``dtype``."""
    return {torch.float16: 2.0 ** -25, torch.bfloat16: 1e-38, torch.float32: 1e-38}[dtype]


def check(got, want, tol, what=""):
    """Every element of got within tol of want."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = (got.detach().double() - want).abs()
    bad = ~(err <= tol)
    if bad.any():
        at = torch.nonzero(bad)[0].tolist()
        ratio = (err / tol).nan_to_num(math.inf).max().item()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {ratio:.3g} bounds; first at {at}: "
                             f"{got[tuple(at)].item()} for {want[tuple(at)].item()} +- {tol[tuple(at)].item()}")


# ---------------------------------------------------------------------------
# group norm
# ---------------------------------------------------------------------------
_ACTS = {"none": lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu,
         "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}


def group_norm(x, groups, weight, bias, act, eps=1e-5):
    """float64 by autograd's elementary functions (x, weight, bias float64 leaves or None)."""
    N, C = x.shape[0], x.shape[-1]
    t = x.reshape(N, -1, groups, C // groups)
    mean = t.mean((1, 3), keepdim=True)
    var = (t - mean).square().mean((1, 3), keepdim=True)
    y = ((t - mean) / (var + eps).sqrt()).reshape(x.shape)
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return _ACTS[act](y)


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
def philox_block(counter, key):
    """Philox 4x32-10 (Salmon et al., 2011) of one block, in Python's integers: counter and key as
    four and two 32-bit words."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [k[0] + 0x9E3779B9 & 0xFFFFFFFF, k[1] + 0xBB67AE85 & 0xFFFFFFFF]
    return c


def kept(n, p, seed, offset, first=0):
    """Whether elements first .. first + n - 1 are kept, by the generator in Python's integers."""
    low = 0xFFFFFFFF
    t, out, block, words = round(p * 2.0 ** 32), [], None, None
    for e in range(first, first + n):
        if e // 4 != block:
            block = e // 4
            words = philox_block([block & low, block >> 32, offset & low, offset >> 32 & low],
                                 [seed & low, seed >> 32 & low])
        out.append(words[e % 4] >= t)
    return torch.tensor(out, dtype=torch.bool)
