"""The performance cases of the operators that complete a layer of an encoder or a decoder
around FlashSCA and the linear and norm operators: attention of queries to the states of an
encoder of another length, group norm with an activation on channels-last maps, and dropout
from a counter-based generator onto a residual.

Six kinds of pass, each as a user's program makes it:

  attention         ``attention_forward``: out = softmax(scale q k^T + mask) v for each head
  attention_train   ``attention_autograd`` and its backward: the output and the gradients of
                    q, k and v
  group_norm        ``group_norm_forward``: act(N(x) weight + bias), N over each sample's
                    positions and each group of channels
  group_norm_train  ``group_norm_autograd`` and its backward: the output and the gradients of
                    the input, the weight and the bias
  dropout           ``dropout_forward``: residual + scale * x / (1 - p) where the element is kept
  dropout_train     ``dropout_autograd`` and its backward: the output and the gradients of the
                    input and the residual

The sizes are BEVFormer-base's (200 x 200 queries of 8 heads x 32 channels, six cameras' maps
on four levels), its small relative's (23 x 23 queries, 4 heads x 8), and generic ones.
``draw`` spreads sizes over the same ranges.

With ``own`` the passes call the framework; without it they are elementary torch operations in
float32 (the generator's words in whole numbers), rounded once at the end.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _attention(name, op, B, Lq, Lk, H, Hk, D, dtype, mask, packed=False):
    return {"name": name, "op": op, "B": B, "Lq": Lq, "Lk": Lk, "H": H, "Hk": Hk, "D": D,
            "dtype": dtype, "mask": mask, "packed": packed}


def _group_norm(name, op, N, R, C, groups, dtype, param_dtype, act, affine=True):
    return {"name": name, "op": op, "N": N, "R": R, "C": C, "groups": groups, "dtype": dtype,
            "param_dtype": param_dtype, "act": act, "affine": affine}


def _dropout(name, op, M, C, dtype, res_dtype, residual, p, scale=1.0):
    return {"name": name, "op": op, "M": M, "C": C, "dtype": dtype, "res_dtype": res_dtype,
            "residual": residual, "p": p, "scale": scale}


def listed():
    return [
        # 23 x 23 queries to every pixel of six small maps (8 x 22): latency of one call
        _attention("attention_small_f32", "attention", 1, 529, 1056, 4, 4, 8, "f32", "none"),
        # one new token of each of eight sequences to states of different lengths, four query
        # heads to a head of the states: serving
        _attention("attention_one_token_bf16", "attention", 8, 1, 8192, 32, 8, 128, "bf16", "lengths"),
        # 200 x 200 queries to every pixel of the third level of six maps (29 x 50), keys and
        # values from one projection: the largest
        _attention("attention_map_bf16", "attention", 1, 40000, 8700, 8, 8, 32, "bf16", "none", True),
        # a decoder's 900 queries to the 200 x 200 cells, a training step
        _attention("attention_train_decoder_bf16", "attention_train", 1, 900, 40000, 8, 8, 32, "bf16",
                   "none"),
        # wide heads, four query heads to a head of the states, padded batches, a training step
        _attention("attention_train_wide_bf16", "attention_train", 2, 2048, 4096, 16, 4, 128, "bf16",
                   "lengths"),
        # sizes that fit no tile, a bias with masked places and rows, a training step
        _attention("attention_train_ragged_f16", "attention_train", 3, 777, 1333, 6, 2, 72, "f16",
                   "bias"),
        # the small relative's six 16 x 44 maps: latency of one call
        _group_norm("group_norm_small_f32", "group_norm", 6, 704, 32, 8, "f32", "f32", "relu"),
        # six cameras' finest level, a training step: the largest
        _group_norm("group_norm_train_maps_bf16", "group_norm_train", 6, 23200, 256, 32, "bf16", "f32",
                    "relu"),
        # odd positions and groups of odd widths, a training step
        _group_norm("group_norm_train_ragged_f16", "group_norm_train", 3, 3331, 330, 30, "f16", "f16",
                    "silu"),
        # the output of the cross-attention at 200 x 200 queries onto the residual
        _dropout("dropout_queries_bf16", "dropout", 40000, 256, "bf16", "bf16", True, 0.1),
        # the inner activations of a wide feed-forward, without a residual: the largest
        _dropout("dropout_wide_bf16", "dropout", 16384, 8192, "bf16", "bf16", False, 0.1),
        # an odd width onto a float32 stream with a residual scale, a training step
        _dropout("dropout_train_ragged_f16", "dropout_train", 3331, 777, "f16", "f32", True, 0.25, 0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row's width: a multiple of eight mostly, any number else."""
    return 8 * _log_int(rng, lo // 8, hi // 8) if rng.random() < 0.75 else _log_int(rng, lo, hi)


def _draw_attention(rng, op, dtype):
    Hk = rng.choice([1, 2, 3, 4, 8])
    H = Hk * rng.choice([1, 1, 1, 2, 4])
    D = rng.choice([32, 64, 96, 128]) if rng.random() < 0.7 else rng.randint(1, 128)
    Lq = 1 if op == "attention" and rng.random() < 0.35 else _log_int(rng, 1, 40000)
    # (a softmax over a few states has next to no gradients to compare)
    B, Lk = _log_int(rng, 1, 16), _log_int(rng, 1 if op == "attention" else 16, 40000)
    masks = ["none", "none", "lengths", "keys"]
    if B * H * Lq * Lk <= 5e7:
        masks += ["pairs", "bias"]
    return _attention("", op, B, Lq, Lk, H, Hk, D, dtype, rng.choice(masks), rng.random() < 0.3)


def _draw_group_norm(rng, op, dtype):
    groups = rng.choice([1, 2, 4, 8, 16, 32, 32, rng.randint(1, 48)])
    C = groups * rng.choice([1, 2, 4, 8, 8, 16, rng.randint(1, 64)])
    return _group_norm("", op, rng.choice([1, 1, 2, 3, 6, 8]), _log_int(rng, 16, 140000), C, groups, dtype,
                       rng.choice([dtype, "f32"]), rng.choice(["none", "relu", "silu", "gelu"]),
                       rng.random() < 0.85)


def _draw_dropout(rng, op, dtype):
    residual = rng.random() < 0.6
    return _dropout("", op, _log_int(rng, 1, 60000), _width(rng, 32, 8192), dtype,
                    rng.choice([dtype, dtype, "f32"]) if residual else dtype, residual,
                    rng.choice([0.05, 0.1, 0.1, 0.25, 0.5]), rng.choice([1.0, 1.0, 0.5]))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    op = rng.choice(["attention", "attention", "attention_train", "attention_train", "group_norm",
                     "group_norm_train", "dropout", "dropout_train"])
    # (their largest listed cases are the other direction's)
    most["group_norm"], most["dropout_train"] = most["group_norm_train"] / 2, most["dropout"]
    make = {"a": _draw_attention, "g": _draw_group_norm, "d": _draw_dropout}[op[0]]
    while True:
        # all sizes anew until the case costs no more than the largest of its kind
        case = make(rng, op, rng.choice(["f32", "f16", "bf16", "bf16"]))
        if op[0] == "a" and case["B"] * case["H"] * case["Lq"] * case["Lk"] > (
                6e8 if op == "attention_train" else 2.8e9):
            continue   # scores that the plain form could not hold
        if _cost(case) <= most[op]:
            del case["name"]
            return case


# ---- inputs ----------------------------------------------------------------------------------


def _lengths(case):
    """The batch's lengths: full, then shorter by steps down to some 3/8."""
    B, Lk = case["B"], case["Lk"]
    return [Lk - (5 * b * Lk) // (8 * B) for b in range(B)]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt = _DTYPES[case["dtype"]]
    train = case["op"].endswith("train")

    def normal(*shape, dtype=dt, std=1.0, mean=0.0, leaf=True):
        t = torch.randn(shape, generator=g, device=dev).mul_(std).add_(mean).to(dtype)
        return t.requires_grad_(train and leaf)

    st = {"op": case["op"]}
    if case["op"].startswith("attention"):
        B, Lq, Lk, H, Hk, D = (case[k] for k in ("B", "Lq", "Lk", "H", "Hk", "D"))
        st["q"] = normal(B, Lq, H, D, std=1.25)
        if case["packed"]:   # one projection makes both
            kv = normal(B, Lk, 2, Hk, D, std=1.25, leaf=False)
            st["k"], st["v"] = kv[:, :, 0].requires_grad_(train), kv[:, :, 1].requires_grad_(train)
        else:
            st["k"], st["v"] = normal(B, Lk, Hk, D, std=1.25), normal(B, Lk, Hk, D)
        st["mask"] = st["key_lengths"] = None
        if case["mask"] == "lengths":
            order = torch.randperm(B, generator=g, device=dev)
            st["key_lengths"] = torch.tensor(_lengths(case), device=dev, dtype=torch.int32)[order].contiguous()
        elif case["mask"] == "keys":   # padding anywhere in a batch: three of four keys take part
            st["mask"] = torch.rand((B, 1, 1, Lk), generator=g, device=dev) < 0.75
        elif case["mask"] == "pairs":   # which queries see which states; some rows see none
            st["mask"] = (torch.rand((B, 1, Lq, Lk), generator=g, device=dev) < 0.6) \
                & (torch.rand((B, 1, Lq, 1), generator=g, device=dev) < 0.95)
        elif case["mask"] == "bias":
            # a penalty on the distance, a slope for each head; far places and a few whole
            # rows are masked, by -inf in even heads and by the type's lowest value in odd ones
            i = torch.arange(Lq, device=dev)[:, None] / Lq
            j = torch.arange(Lk, device=dev)[None, :] / Lk
            far = (i - j).abs()
            bias = -far * (2.0 ** torch.arange(H, device=dev))[:, None, None]
            out = (far > 0.6) | (torch.rand((Lq, 1), generator=g, device=dev) < 0.02)
            low = torch.where(torch.arange(H, device=dev) % 2 == 0, -math.inf,
                              torch.finfo(torch.float32).min)[:, None, None]
            st["mask"] = torch.where(out, low, bias)[None]
        if train:
            st["grad_out"] = normal(B, Lq, H, D, leaf=False)
    elif case["op"].startswith("group_norm"):
        N, R, C = case["N"], case["R"], case["C"]
        pdt = _DTYPES[case["param_dtype"]]
        # a convolution's output: each channel with an offset of its own
        x = torch.randn((N, R, C), generator=g, device=dev).add_(
            0.5 * torch.randn((C,), generator=g, device=dev))
        st.update(x=x.to(dt).requires_grad_(train), groups=case["groups"], act=case["act"],
                  weight=normal(C, dtype=pdt, std=0.1, mean=1.0) if case["affine"] else None,
                  bias=normal(C, dtype=pdt, std=0.1) if case["affine"] else None)
        if train:
            st["grad_out"] = normal(N, R, C, leaf=False)
    else:
        M, C = case["M"], case["C"]
        rdt = _DTYPES[case["res_dtype"]]
        st.update(x=normal(M, C), residual=normal(M, C, dtype=rdt) if case["residual"] else None,
                  p=case["p"], scale=case["scale"], seed=0x5DEECE66D + 7919 * int(seed), offset=int(seed) + 3)
        if train:
            st["grad_out"] = normal(M, C, dtype=rdt, leaf=False)
    return st


def run(st):
    if own:
        return _run_own(st)
    return {"a": _plain_attention, "g": _plain_group_norm, "d": _plain_dropout}[st["op"][0]](st)


# ---- the framework's calls -------------------------------------------------------------------


def _run_own(st):
    import paper_2607_10071_amd as fb

    op = st["op"]
    if op.startswith("attention"):
        call = fb.attention_autograd if op.endswith("train") else fb.attention_forward
        out = call(st["q"], st["k"], st["v"], mask=st["mask"], key_lengths=st["key_lengths"])
        names = ["q", "k", "v"]
    elif op.startswith("group_norm"):
        call = fb.group_norm_autograd if op.endswith("train") else fb.group_norm_forward
        out = call(st["x"], st["groups"], st["weight"], st["bias"], activation=st["act"])
        names = [n for n in ("x", "weight", "bias") if st[n] is not None]
    else:
        call = fb.dropout_autograd if op.endswith("train") else fb.dropout_forward
        out = call(st["x"], st["p"], st["seed"], st["offset"], residual=st["residual"], scale=st["scale"])
        names = [n for n in ("x", "residual") if st[n] is not None]
    if not op.endswith("train"):
        return out
    grads = torch.autograd.grad(out, [st[n] for n in names], st["grad_out"])
    return {"out": out.detach(), **{"grad_" + n: t for n, t in zip(names, grads)}}


# ---- the plain forms -------------------------------------------------------------------------


def _heads_first(t, share):
    """[B, L, heads, D] as float32 [B, heads * share, L, D]."""
    t = t.detach().float().transpose(1, 2)
    return (t.repeat_interleave(share, 1) if share > 1 else t).contiguous()


def _plain_attention(st):
    H, Hk = st["q"].shape[2], st["k"].shape[2]
    share = H // Hk
    q, k, v = _heads_first(st["q"], 1), _heads_first(st["k"], share), _heads_first(st["v"], share)
    scale = q.shape[-1] ** -0.5
    s = (q * scale) @ k.transpose(2, 3).contiguous()
    mask = st["mask"]
    if st["key_lengths"] is not None:
        mask = (torch.arange(k.shape[2], device=k.device) < st["key_lengths"][:, None])[:, None, None]
    if mask is not None:
        s = s.masked_fill_(~mask, -math.inf) if mask.dtype is torch.bool else s.add_(mask)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.mul_(torch.where(total > 0.0, 1.0 / total, 0.0))   # a row that sees nothing gives zeros
    out = (p @ v).transpose(1, 2).contiguous()
    if not st["op"].endswith("train"):
        return out.to(st["q"].dtype)
    go = _heads_first(st["grad_out"], 1)
    dv = p.transpose(2, 3).contiguous() @ go
    ds = go @ v.transpose(2, 3).contiguous()
    ds = ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = ds @ k
    dk = ds.transpose(2, 3).contiguous() @ q
    grads = {"out": out, "grad_q": dq.transpose(1, 2).contiguous()}
    grads["grad_k"], grads["grad_v"] = (t.unflatten(1, (Hk, share)).sum(2).transpose(1, 2).contiguous()
                                        for t in (dk, dv))
    return {n: t.to(st["q"].dtype) for n, t in grads.items()}


_SQRT_HALF = 0.7071067811865476
_INV_SQRT_2PI = 0.3989422804014327


def _act(a, v):
    if a == "relu":
        return v.clamp(min=0.0)
    if a == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * _SQRT_HALF))
    if a == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _act_slope(a, v):
    if a == "relu":
        return (v > 0.0).to(v.dtype)
    if a == "gelu":
        return 0.5 * (1.0 + torch.erf(v * _SQRT_HALF)) + v * _INV_SQRT_2PI * torch.exp(-0.5 * v * v)
    if a == "silu":
        p = 1.0 / (1.0 + torch.exp(-v))
        return p * (1.0 + v * (1.0 - p))
    return torch.ones_like(v)


def _plain_group_norm(st):
    x, G = st["x"].detach().float(), st["groups"]
    N, C = x.shape[0], x.shape[-1]
    w = torch.ones(C, device=x.device) if st["weight"] is None else st["weight"].detach().float()
    b = torch.zeros(C, device=x.device) if st["bias"] is None else st["bias"].detach().float()
    v = x.reshape(N, -1, G, C // G)
    v = v - v.mean((1, 3), keepdim=True)
    r = torch.rsqrt((v * v).mean((1, 3), keepdim=True) + 1e-5)
    xhat = (v * r).reshape(x.shape)
    pre = xhat * w + b
    out = _act(st["act"], pre).to(st["x"].dtype)
    if st["op"] == "group_norm":
        return out
    d = st["grad_out"].float() * _act_slope(st["act"], pre)
    dh, h = (d * w).reshape(v.shape), xhat.reshape(v.shape)
    dx = r * (dh - dh.mean((1, 3), keepdim=True) - h * (dh * h).mean((1, 3), keepdim=True))
    grads = {"out": out, "grad_x": dx.reshape(x.shape).to(st["x"].dtype)}
    if st["weight"] is not None:
        grads["grad_weight"] = (d * xhat).reshape(-1, C).sum(0).to(st["weight"].dtype)
        grads["grad_bias"] = d.reshape(-1, C).sum(0).to(st["bias"].dtype)
    return grads


_LOW = 0xFFFFFFFF


def _words(n, seed, offset, device):
    """The first n words of Philox 4x32-10 (Salmon et al., 2011): word i is number i % 4 of the
    block whose counter is (i / 4, offset) and whose key is the seed, 64 bits each."""
    i = torch.arange((n + 3) // 4, device=device)
    a, b = i & _LOW, i >> 32
    c, d = torch.full_like(i, offset & _LOW), torch.full_like(i, offset >> 32 & _LOW)
    k0, k1 = seed & _LOW, seed >> 32 & _LOW
    for _ in range(10):
        u, v = a * 0xD2511F53, c * 0xCD9E8D57   # the low 64 bits, in two's complement
        a, b, c, d = (v >> 32 & _LOW) ^ b ^ k0, v & _LOW, (u >> 32 & _LOW) ^ d ^ k1, u & _LOW
        k0, k1 = k0 + 0x9E3779B9 & _LOW, k1 + 0xBB67AE85 & _LOW
    return torch.stack((a, b, c, d), 1).reshape(-1)[:n]


def _plain_dropout(st):
    x, p = st["x"].detach(), st["p"]
    kept = (_words(x.numel(), st["seed"], st["offset"], x.device) >= round(p * 2.0 ** 32)).reshape(x.shape)
    factor = st["scale"] / (1.0 - p)
    out = torch.where(kept, x.float() * factor, 0.0)
    if st["residual"] is not None:
        out = st["residual"].detach().float() + out
    out = out.to(x.dtype if st["residual"] is None else st["residual"].dtype)
    if st["op"] == "dropout":
        return out
    grads = {"out": out, "grad_x": torch.where(kept, st["grad_out"].float() * factor, 0.0).to(x.dtype)}
    if st["residual"] is not None:
        grads["grad_residual"] = st["grad_out"].clone()
    return grads


# ---- what a pass cannot do without -----------------------------------------------------------


def work(case):
    es = _BYTES[case["dtype"]]
    train = case["op"].endswith("train")
    if case["op"].startswith("attention"):
        B, Lq, Lk, H, Hk, D = (case[k] for k in ("B", "Lq", "Lk", "H", "Hk", "D"))
        keys = sum(_lengths(case)) if case["mask"] == "lengths" else B * Lk
        rows, states = B * Lq * H * D * es, keys * Hk * D * es
        masks = {"none": 0, "lengths": 4 * B, "keys": B * Lk, "pairs": B * Lq * Lk, "bias": 4 * H * Lq * Lk}
        nbytes = 2 * rows + 2 * states + masks[case["mask"]]
        if train:   # the output's gradient in, the others' out
            nbytes += 2 * rows + 2 * B * Lk * Hk * D * es
        return {"bytes": nbytes, "flops": (14 if train else 4) * keys * Lq * H * D}
    if case["op"].startswith("group_norm"):
        n = case["N"] * case["R"] * case["C"]
        vectors = 2 * case["C"] * _BYTES[case["param_dtype"]] if case["affine"] else 0
        return {"bytes": (4 if train else 2) * n * es + (2 if train else 1) * vectors,
                "flops": n * (24 if train else 8)}
    n = case["M"] * case["C"]
    rs = _BYTES[case["res_dtype"]]
    nbytes = n * (es + rs * (2 if case["residual"] else 1))
    if train:
        nbytes += n * (rs * (2 if case["residual"] else 1) + es)
    return {"bytes": nbytes, "flops": n * (50 if train else 25)}


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (5e14 if case["dtype"] != "f32" else 5e13)


# ---- the same results in 64 bits -------------------------------------------------------------


def exact(case, seed):
    """The outputs by torch's own functions in float64, the gradients by its autograd; the
    generator in numpy's unsigned 64-bit words."""
    st = prepare(case, seed)
    return {"a": _exact_attention, "g": _exact_group_norm, "d": _exact_dropout}[st["op"][0]](st)


def _exact_attention(st):
    train = st["op"].endswith("train")
    q, k, v = (st[n].detach().double() for n in "qkv")
    share = q.shape[2] // k.shape[2]
    out, dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(q.shape[0]):
        for h in range(q.shape[2]):
            qi, ki, vi = (t.clone().requires_grad_(train)
                          for t in (q[b, :, h], k[b, :, h // share], v[b, :, h // share]))
            s = (qi @ ki.t()) * q.shape[-1] ** -0.5
            if st["key_lengths"] is not None:
                s = s.masked_fill(torch.arange(s.shape[1], device=s.device) >= st["key_lengths"][b], -math.inf)
            elif st["mask"] is not None:
                m = st["mask"][b % st["mask"].shape[0], h % st["mask"].shape[1]]
                s = s.masked_fill(~m, -math.inf) if m.dtype is torch.bool else s + m.double()
            seen = (s.detach() > -math.inf).any(1, keepdim=True)
            o = torch.softmax(s.masked_fill(~seen, 0.0), 1) * seen @ vi
            out[b, :, h] = o.detach()
            if train:
                gq, gk, gv = torch.autograd.grad(o, (qi, ki, vi), st["grad_out"][b, :, h].double())
                dq[b, :, h] = gq
                dk[b, :, h // share] += gk
                dv[b, :, h // share] += gv
    return {"out": out, "grad_q": dq, "grad_k": dk, "grad_v": dv} if train else out


def _exact_group_norm(st):
    F = torch.nn.functional
    names = [n for n in ("x", "weight", "bias") if st[n] is not None]
    train = st["op"].endswith("train")
    d = {n: st[n].detach().double().requires_grad_(train) for n in names}
    y = F.group_norm(d["x"].transpose(1, 2), st["groups"], d.get("weight"), d.get("bias"), 1e-5).transpose(1, 2)
    y = {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu}[st["act"]](y)
    if not train:
        return y
    grads = torch.autograd.grad(y, [d[n] for n in names], st["grad_out"].double())
    return {"out": y.detach(), **{"grad_" + n: t for n, t in zip(names, grads)}}


def _exact_dropout(st):
    x = st["x"].detach()
    u32, u64 = np.uint32, np.uint64
    i = np.arange((x.numel() + 3) // 4, dtype=u64)
    block = [(i & u64(_LOW)).astype(u32), (i >> u64(32)).astype(u32)]
    block += [np.full(i.shape, st["offset"] >> s & _LOW, dtype=u32) for s in (0, 32)]
    key = [st["seed"] & _LOW, st["seed"] >> 32 & _LOW]
    for _ in range(10):
        first = block[0].astype(u64) * u64(0xD2511F53)
        second = block[2].astype(u64) * u64(0xCD9E8D57)
        block = [(second >> u64(32)).astype(u32) ^ block[1] ^ u32(key[0]), second.astype(u32),
                 (first >> u64(32)).astype(u32) ^ block[3] ^ u32(key[1]), first.astype(u32)]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    dropped = np.stack([w < u64(round(st["p"] * 2.0 ** 32)) for w in block], 1).reshape(-1)[:x.numel()]
    dropped = torch.from_numpy(dropped).to(x.device).reshape(x.shape)
    factor = st["scale"] / (1.0 - st["p"])
    out = (x.double() * factor).masked_fill(dropped, 0.0)
    if st["residual"] is not None:
        out = out + st["residual"].detach().double()
    if st["op"] == "dropout":
        return out
    grads = {"out": out, "grad_x": (st["grad_out"].double() * factor).masked_fill(dropped, 0.0)}
    if st["residual"] is not None:
        grads["grad_residual"] = st["grad_out"].double()
    return grads
