"""The performance cases of the operators around FlashSCA in an encoder block: the
matrix product with bias, activation and residual in its epilogue, and the norms
before and after a block with its gate and residual scale.

Four kinds of pass, each as a user's program makes it:

  linear        ``linear_forward``: out = residual + scale * act(x W^T + bias)
  linear_train  ``linear_autograd`` and its backward: the output and the gradients of
                the input, the weight, the bias and the residual
  norm          ``norm_forward``: s = residual + scale * gate * N_post(x), y = N(s)
  norm_train    ``norm_autograd`` and its backward: both outputs and the gradients of
                the input, the residual, the gate and the norms' weights and biases

The sizes are BEVFormer-base's (200 x 200 queries, 256 channels, 8 heads x 4 levels x
8 points, six cameras' value maps on four levels), its small relative's (23 x 23
queries, 32 channels), and generic ones of wide blocks: one row, a few thousand
rows, odd sizes.  ``draw`` spreads sizes over the same ranges.

With ``own`` the passes call the framework; without it they are elementary torch
operations in float32, rounded once at the end.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _linear(name, op, M, K, N, dtype, out_dtype, act, bias, residual, scale=1.0):
    return {"name": name, "op": op, "M": M, "K": K, "N": N, "dtype": dtype, "out_dtype": out_dtype,
            "act": act, "bias": bias, "residual": residual, "scale": scale}


def _norm(name, op, G, R, C, dtype, res_dtype, kind, post, residual, gate, affine, scale=1.0):
    return {"name": name, "op": op, "G": G, "R": R, "C": C, "dtype": dtype, "res_dtype": res_dtype,
            "kind": kind, "post": post, "residual": residual, "gate": gate, "affine": affine,
            "scale": scale}


def listed():
    return [
        # the output projection of a small cross-attention (23 x 23 queries): latency of one call
        _linear("linear_small_f32", "linear", 529, 32, 32, "f32", "f32", "none", True, True),
        # one row through a wide block's down projection, onto the residual: serving latency
        _linear("linear_one_row_bf16", "linear", 1, 4096, 4096, "bf16", "bf16", "none", True, True),
        # FlashSCA's value projection: six cameras' pixels on four levels
        _linear("linear_value_bf16", "linear", 184950, 256, 256, "bf16", "bf16", "none", True, False),
        # FlashSCA's sampling offsets from the queries, in the float32 it reads
        _linear("linear_offsets_bf16", "linear", 40000, 256, 512, "bf16", "f32", "none", True, False),
        # a wide block's products over a batch of rows, activation and residual: the largest
        _linear("linear_large_bf16", "linear", 8192, 4096, 8192, "bf16", "bf16", "silu", True, True, 0.5),
        # sizes that fit no tile, half precision, a training step
        _linear("linear_train_ragged_f16", "linear_train", 3331, 515, 777, "f16", "f16", "relu", True,
                True),
        # the first product of an encoder block's feed-forward at 200 x 200 queries, a training step
        _linear("linear_train_ffn_bf16", "linear_train", 40000, 256, 1024, "bf16", "bf16", "gelu", True,
                False),
        # FlashSCA's output projection onto the queries at 200 x 200 in float32, a training step
        _linear("linear_train_output_f32", "linear_train", 40000, 256, 256, "f32", "f32", "none", True,
                True),
        # the norm after a small cross-attention: latency of one call
        _norm("norm_small_f32", "norm", 1, 529, 32, "f32", "f32", "layer", False, True, "none", True),
        # norms before and after a wide block, a gate for each sample, the largest rows
        _norm("norm_sandwich_wide_bf16", "norm", 4, 4096, 4096, "bf16", "bf16", "rms", True, True,
              "sample", True, 0.5),
        # the norm after the cross-attention at 200 x 200 queries with a gate for each channel, a
        # training step
        _norm("norm_train_queries_bf16", "norm_train", 1, 40000, 256, "bf16", "bf16", "layer", False,
              True, "channel", True),
        # an odd width, norms on both sides, gates for each sample, a training step
        _norm("norm_train_ragged_f16", "norm_train", 3, 2777, 771, "f16", "f16", "layer", True, True,
              "sample", True, 0.7071),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row's width: a multiple of eight mostly, any number else."""
    return 8 * _log_int(rng, lo // 8, hi // 8) if rng.random() < 0.75 else _log_int(rng, lo, hi)


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    op = rng.choice(["linear", "linear", "linear_train", "norm", "norm_train"])
    while True:
        # all sizes anew until the case costs no more than the largest of its kind
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        scale = rng.choice([1.0, 1.0, 0.5, 0.7071])
        if op.startswith("linear"):
            lo = 1 if op == "linear" else 64
            M = rng.randint(1, 64) if op == "linear" and rng.random() < 0.25 else _log_int(rng, lo, 190000)
            out_dtype = "f32" if rng.random() < 0.2 else dtype
            case = _linear("", op, M, _width(rng, 32, 8192), _width(rng, 32, 8192), dtype, out_dtype,
                           rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                           rng.random() < 0.75, rng.random() < 0.5, scale)
        else:
            G = rng.choice([1, 1, 2, 3, 4])
            R = _log_int(rng, 1, 60000) if op == "norm" else _log_int(rng, 32, 60000)
            post = rng.random() < 0.4
            case = _norm("", op, G, R, _width(rng, 32, 8192), dtype, dtype, rng.choice(["layer", "rms"]),
                         post, rng.random() < 0.75, rng.choice(["none", "channel", "sample"]),
                         rng.random() < 0.8, scale)
        if _cost(case) <= most[op]:
            del case["name"]
            return case


# ---- inputs ----------------------------------------------------------------------------------


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt = _DTYPES[case["dtype"]]
    train = case["op"].endswith("train")

    def normal(*shape, dtype=dt, std=1.0, mean=0.0, leaf=True):
        t = torch.randn(shape, generator=g, device=dev).mul_(std).add_(mean).to(dtype)
        return t.requires_grad_(train and leaf)

    st = {"op": case["op"], "scale": case["scale"]}
    if case["op"].startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        odt = _DTYPES[case["out_dtype"]]
        st.update(act=case["act"], out_dtype=odt, x=normal(M, K),
                  weight=normal(N, K, std=K ** -0.5),
                  bias=normal(N, std=0.1) if case["bias"] else None,
                  residual=normal(M, N, dtype=odt) if case["residual"] else None)
        if train:
            st["grad_out"] = normal(M, N, dtype=odt, leaf=False)
        return st
    G, R, C = case["G"], case["R"], case["C"]
    rdt = _DTYPES[case["res_dtype"]]
    affine, layer = case["affine"], case["kind"] == "layer"
    # a block's output has an offset and a scale of its own; weights lie around one
    st.update(kind=case["kind"], post=case["kind"] if case["post"] else None,
              eps=1e-5 if layer else 1e-6, x=normal(G, R, C, std=1.5, mean=0.25),
              residual=normal(G, R, C, dtype=rdt) if case["residual"] else None,
              gate={"none": lambda: None, "channel": lambda: normal(C, std=0.3, mean=0.5),
                    "sample": lambda: normal(G, C, std=0.3, mean=0.5)}[case["gate"]](),
              weight=normal(C, std=0.1, mean=1.0) if affine else None,
              bias=normal(C, std=0.1) if affine and layer else None,
              post_weight=normal(C, std=0.1, mean=1.0) if affine and case["post"] else None,
              post_bias=normal(C, std=0.1) if affine and case["post"] and layer else None)
    if train:
        st["grad_y"] = normal(G, R, C, leaf=False)
        st["grad_s"] = normal(G, R, C, dtype=rdt, leaf=False)
    return st


_LINEAR_LEAVES = ("x", "weight", "bias", "residual")
_NORM_LEAVES = ("x", "residual", "gate", "weight", "bias", "post_weight", "post_bias")


def run(st):
    return _run_own(st) if own else _run_plain(st)


# ---- the framework's calls -------------------------------------------------------------------


def _run_own(st):
    import paper_2607_10071_amd as fb

    op = st["op"]
    if op == "linear":
        return fb.linear_forward(st["x"], st["weight"], st["bias"], activation=st["act"],
                                 residual=st["residual"], scale=st["scale"],
                                 out_dtype=st["out_dtype"])
    if op == "linear_train":
        out = fb.linear_autograd(st["x"], st["weight"], st["bias"], activation=st["act"],
                                 residual=st["residual"], scale=st["scale"],
                                 out_dtype=st["out_dtype"])
        names = [k for k in _LINEAR_LEAVES if st[k] is not None]
        grads = torch.autograd.grad(out, [st[k] for k in names], st["grad_out"])
        return {"out": out.detach(), **{"grad_" + k: v for k, v in zip(names, grads)}}
    call = fb.norm_forward if op == "norm" else fb.norm_autograd
    y, s = call(st["x"], st["weight"], st["bias"], residual=st["residual"], gate=st["gate"],
                scale=st["scale"], norm=st["kind"], post_norm=st["post"],
                post_weight=st["post_weight"], post_bias=st["post_bias"], eps=st["eps"])
    if op == "norm":
        return {"y": y, "s": s}
    names = [k for k in _NORM_LEAVES if st[k] is not None]
    grads = torch.autograd.grad([y, s], [st[k] for k in names], [st["grad_y"], st["grad_s"]])
    return {"y": y.detach(), "s": s.detach(), **{"grad_" + k: v for k, v in zip(names, grads)}}


# ---- the plain forms -------------------------------------------------------------------------

_SQRT_HALF = 0.7071067811865476
_SQRT_2_OVER_PI = 0.7978845608028654
_INV_SQRT_2PI = 0.3989422804014327


def _act(a, v):
    if a == "relu":
        return v.clamp(min=0.0)
    if a == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * _SQRT_HALF))
    if a == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(_SQRT_2_OVER_PI * (v + 0.044715 * v * v * v)))
    if a == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _act_slope(a, v):
    if a == "relu":
        return (v > 0.0).to(v.dtype)
    if a == "gelu":
        return 0.5 * (1.0 + torch.erf(v * _SQRT_HALF)) + v * _INV_SQRT_2PI * torch.exp(-0.5 * v * v)
    if a == "gelu_tanh":
        t = torch.tanh(_SQRT_2_OVER_PI * (v + 0.044715 * v * v * v))
        return 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * _SQRT_2_OVER_PI * (1.0 + 0.134145 * v * v)
    if a == "silu":
        p = 1.0 / (1.0 + torch.exp(-v))
        return p * (1.0 + v * (1.0 - p))
    return torch.ones_like(v)


def _float(t):
    return None if t is None else t.detach().float()


def _normed(v, kind, eps):
    """The normalised rows and their factor."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)
    return v * r, r


def _affine(v, weight, bias):
    if weight is not None:
        v = v * weight
    return v if bias is None else v + bias


def _normed_grad(g, xhat, r, kind):
    g = g - xhat * (g * xhat).mean(-1, keepdim=True) - (g.mean(-1, keepdim=True) if kind == "layer" else 0.0)
    return g * r


def _run_plain(st):
    return _plain_linear(st) if st["op"].startswith("linear") else _plain_norm(st)


def _plain_linear(st):
    a, scale = st["act"], st["scale"]
    x, w, b, res = (_float(st[k]) for k in _LINEAR_LEAVES)
    pre = x @ w.t()
    if b is not None:
        pre = pre + b
    out = scale * _act(a, pre)
    if res is not None:
        out = res + out
    out = out.to(st["out_dtype"])
    if st["op"] == "linear":
        return out
    go = st["grad_out"].float()
    d = scale * go * _act_slope(a, pre)
    grads = {"out": out, "grad_x": (d @ w).to(st["x"].dtype), "grad_weight": (d.t() @ x).to(st["weight"].dtype)}
    if b is not None:
        grads["grad_bias"] = d.sum(0).to(st["bias"].dtype)
    if res is not None:
        grads["grad_residual"] = go.to(st["residual"].dtype)
    return grads


def _plain_norm(st):
    kind, post, eps, scale = st["kind"], st["post"], st["eps"], st["scale"]
    x, res, gate, w, b, pw, pb = (_float(st[k]) for k in _NORM_LEAVES)
    C = x.shape[-1]
    if gate is not None and gate.dim() == 2:
        gate = gate[:, None, :]
    u, xn, rx = x, None, None
    if post is not None:
        xn, rx = _normed(x, post, eps)
        u = _affine(xn, pw, pb)
    factor = scale if gate is None else scale * gate
    s = u * factor
    if res is not None:
        s = res + s
    # the stream that the caller keeps, in its type, is what the norm reads
    stored = s.to(st["x"].dtype if res is None else st["residual"].dtype)
    sn, rs = _normed(stored.float(), kind, eps)
    y = _affine(sn, w, b).to(st["x"].dtype)
    if st["op"] == "norm":
        return {"y": y, "s": stored}
    gy, gs = st["grad_y"].float(), st["grad_s"].float()
    ds = gs + _normed_grad(gy if w is None else gy * w, sn, rs, kind)
    du = ds * factor
    grads = {"y": y, "s": stored, "grad_x": du}
    if post is not None:
        grads["grad_x"] = _normed_grad(du if pw is None else du * pw, xn, rx, post)
    if res is not None:
        grads["grad_residual"] = ds
    if gate is not None:
        dg = scale * ds * u
        grads["grad_gate"] = dg.sum(1) if st["gate"].dim() == 2 else dg.reshape(-1, C).sum(0)
    if w is not None:
        grads["grad_weight"] = (gy * sn).reshape(-1, C).sum(0)
    if b is not None:
        grads["grad_bias"] = gy.reshape(-1, C).sum(0)
    if pw is not None:
        grads["grad_post_weight"] = (du * xn).reshape(-1, C).sum(0)
    if pb is not None:
        grads["grad_post_bias"] = du.reshape(-1, C).sum(0)
    return {k: v.to(st[k[5:]].dtype) if k.startswith("grad_") else v for k, v in grads.items()}


# ---- what a pass cannot do without -----------------------------------------------------------


def work(case):
    es = _BYTES[case["dtype"]]
    train = case["op"].endswith("train")
    if case["op"].startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        os_ = _BYTES[case["out_dtype"]]
        small = (N * K + (N if case["bias"] else 0)) * es
        nbytes = M * K * es + small + M * N * os_ * (2 if case["residual"] else 1)
        flops = 2 * M * N * K
        if train:   # the output's gradient in, the others' out
            nbytes += M * N * os_ * (2 if case["residual"] else 1) + M * K * es + small
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    n = case["G"] * case["R"] * case["C"]
    rs = _BYTES[case["res_dtype"]]
    layer = case["kind"] == "layer"
    vectors = ((2 if layer else 1) * (2 if case["post"] else 1) if case["affine"] else 0) \
        + {"none": 0, "channel": 1, "sample": case["G"]}[case["gate"]]
    nbytes = n * (2 * es + rs * (2 if case["residual"] else 1)) + vectors * case["C"] * es
    flops = n * (8 + (6 if case["post"] else 0))
    if train:
        nbytes += n * (2 * es + rs * (2 if case["residual"] else 1)) + vectors * case["C"] * es
        flops *= 3
    return {"bytes": nbytes, "flops": flops}


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (5e14 if case["dtype"] != "f32" else 5e13)


# ---- the same results in 64 bits -------------------------------------------------------------


def exact(case, seed):
    """The outputs by torch's own functions in float64, the gradients by its autograd."""
    st = prepare(case, seed)
    F = torch.nn.functional
    train = case["op"].endswith("train")
    leaves = _LINEAR_LEAVES if case["op"].startswith("linear") else _NORM_LEAVES
    d = {k: None if st[k] is None else st[k].detach().double().requires_grad_(train) for k in leaves}
    if case["op"].startswith("linear"):
        fn = {"none": lambda v: v, "relu": F.relu, "gelu": F.gelu, "silu": F.silu,
              "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}[case["act"]]
        out = fn(F.linear(d["x"], d["weight"], d["bias"])) * case["scale"]
        if d["residual"] is not None:
            out = out + d["residual"]
        if not train:
            return out
        outs, into = {"out": out}, [st["grad_out"].double()]
    else:
        C, eps = case["C"], st["eps"]

        def norm(v, kind, weight, bias):
            if kind == "layer":
                return F.layer_norm(v, (C,), weight, bias, eps)
            return F.rms_norm(v, (C,), weight, eps)

        u = norm(d["x"], st["post"], d["post_weight"], d["post_bias"]) if st["post"] else d["x"]
        if d["gate"] is not None:
            u = u * d["gate"].reshape(-1, 1, C)
        s = u * case["scale"] if d["residual"] is None else torch.add(d["residual"], u, alpha=case["scale"])
        stored = s.detach().to(_DTYPES[case["res_dtype" if case["residual"] else "dtype"]]).double()
        s = s + (stored - s.detach())   # rounded, with the gradient passed through
        outs = {"y": norm(s, st["kind"], d["weight"], d["bias"]), "s": s}
        if not train:
            return outs
        into = [st["grad_y"].double(), st["grad_s"].double()]
    names = [k for k in leaves if d[k] is not None]
    grads = torch.autograd.grad(list(outs.values()), [d[k] for k in names], into)
    return {**{k: v.detach() for k, v in outs.items()}, **{"grad_" + k: g for k, g in zip(names, grads)}}
