"""Attention, group norm and dropout in HIP graphs, under hooks on saved tensors, from several
threads, and together as a layer uses them."""
import threading

import pytest
import torch

import layer_ref as ref
import paper_2607_10071_amd as fb

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def randn(*shape, dtype=F32, seed=0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def noise():
    x = torch.randn(4096, device="cuda")
    return float((x * x).sum().item())


# ---- graphs ------------------------------------------------------------------------------------


def replayed(inputs, step):
    """``step`` captured, then replayed over new inputs with eager work between: each replay's results
    are the eager ones, bit for bit."""
    step()   # (what is allocated and looked up once)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for k in range(4):
        for n, t in enumerate(inputs):
            with torch.no_grad():
                if t.dtype == torch.bool:
                    t.copy_(randn(*t.shape, seed=100 * k + n) < 0.5)
                elif t.dtype == torch.int32:
                    t.copy_(torch.randint(0, 300, t.shape, device="cuda"))
                elif t.dtype == torch.int64:
                    t.copy_(torch.tensor([5 + k, 7]))
                else:
                    t.copy_(randn(*t.shape, dtype=t.dtype, seed=100 * k + n))
        for t in results:
            t.fill_(7)
        noise()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        noise()
        want = step()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (k, i)


@pytest.mark.parametrize("mask", ["none", "lengths", "keys", "bias"])
@pytest.mark.parametrize("lq,lk,d", [(1, 3000, 64), (200, 300, 32), (70, 260, 41)])
def test_attention_forward_and_backward(lq, lk, d, mask):
    q, k, v = randn(2, lq, 4, d, dtype=BF16), randn(2, lk, 2, d, dtype=BF16), randn(2, lk, 2, d, dtype=BF16, seed=1)
    g = randn(2, lq, 4, d, dtype=BF16, seed=2)
    kw, inputs = {}, [q, k, v, g]
    if mask == "lengths":
        kw["key_lengths"] = torch.tensor([lk, 17], dtype=torch.int32, device="cuda")
        inputs.append(kw["key_lengths"])
    elif mask == "keys":
        kw["mask"] = randn(2, 1, 1, lk) < 0.5
        inputs.append(kw["mask"])
    elif mask == "bias":
        kw["mask"] = randn(1, 4, lq, lk)
        inputs.append(kw["mask"])

    def step():
        stats = torch.empty((2, 4, lq, 2), device="cuda")
        rest = torch.empty_like(q)
        out = fb.attention_forward(q, k, v, stats=stats, rest=rest, **kw)
        r = fb.attention_backward(g, q, k, v, out, stats, rest=rest, **kw)
        return [out, stats, r["q"], r["k"], r["v"]]

    replayed(inputs, step)


@pytest.mark.parametrize("R", [30, 4000])
def test_group_norm_forward_and_backward(R):
    x, g = randn(2, R, 64, dtype=BF16), randn(2, R, 64, dtype=BF16, seed=1)
    w, b = randn(64), randn(64, seed=1)

    def step():
        stats = torch.empty((2, 8, 2), device="cuda")
        y = fb.group_norm_forward(x, 8, w, b, "silu", stats=stats)
        r = fb.group_norm_backward(g, x, stats, 8, w, b, "silu", want=("x", "weight", "bias"))
        return [y, *r.values()]

    replayed([x, g, w, b], step)


def test_training_steps_with_a_new_mask_each_replay():
    """The autograd forms captured together with their gradients; dropout's state in device memory."""
    q, k, v = (randn(1, n, 4, 32, dtype=BF16, seed=i).requires_grad_() for i, n in enumerate((50, 90, 90)))
    w = randn(128, 128, dtype=BF16, std=0.1).requires_grad_()
    r = randn(1, 50, 128, dtype=BF16, seed=5).requires_grad_()
    state = torch.tensor([1, 2], device="cuda")
    g = randn(1, 50, 128, dtype=BF16, seed=6)

    def step():
        a = fb.attention_autograd(q, k, v)
        y = fb.linear_autograd(a.reshape(1, 50, 128), w)
        out = fb.dropout_autograd(y, 0.3, state, residual=r)
        return [out.detach(), *torch.autograd.grad(out, [q, k, v, w, r], g)]

    replayed([q, k, v, w, state, g], lambda: [t.clone() for t in step()])


def test_two_graphs_share_no_workspace():
    """Two captured calls with workspaces of their own replay in any order."""
    ins = [(randn(1, 1, 8, 64, dtype=F16, seed=i), randn(1, 5000, 8, 64, dtype=F16, seed=i + 9)) for i in range(2)]
    want = [fb.attention_forward(q, k, k) for q, k in ins]
    graphs, outs = [], []
    for q, k in ins:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(fb.attention_forward(q, k, k))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in ins]
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


# ---- saved tensors -----------------------------------------------------------------------------


def wide_there(t):
    n = t.shape[-1]
    view = torch.full((*t.shape[:-1], n + 11), 1, dtype=t.dtype, device=t.device)[..., 3:n + 3]
    view.copy_(t)
    return view


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_hooks_that_give_back_slices(dtype):
    q, k, v = (randn(2, n, 4, 24, dtype=dtype, seed=i).requires_grad_() for i, n in enumerate((50, 90, 90)))
    mask, lengths = randn(1, 4, 50, 90), torch.tensor([90, 31], dtype=torch.int32, device="cuda")
    x = randn(3, 700, 48, dtype=dtype).requires_grad_()
    w, b = randn(48, dtype=dtype).requires_grad_(), randn(48, dtype=dtype, seed=1).requires_grad_()
    r = randn(3, 700, 48, dtype=dtype, seed=2).requires_grad_()
    state = torch.tensor([3, 4], device="cuda")

    def step():
        a = fb.attention_autograd(q, k, v, mask=mask, key_lengths=lengths)
        y = fb.group_norm_autograd(x, 6, w, b, "gelu")
        z = fb.dropout_autograd(y, 0.2, state, residual=r)
        return torch.autograd.grad([a, z], [q, k, v, x, w, b, r], [torch.ones_like(a), torch.ones_like(z)])

    want = step()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wide_there):
        got = step()
    assert all(torch.equal(a, c) for a, c in zip(want, got))


@pytest.mark.parametrize("change", [lambda t: t.double(), lambda t: t[..., :-1], lambda t: t.cpu()], ids=["type", "size", "device"])
def test_saved_tensors_that_came_back_as_something_else_are_refused(change):
    q = randn(1, 40, 2, 32).requires_grad_()
    x = randn(2, 50, 32).requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
        a, y = fb.attention_autograd(q, q, q), fb.group_norm_autograd(x, 4)
        for out, leaf in ((a, q), (y, x)):
            with pytest.raises(ValueError, match="came back as"):
                torch.autograd.grad(out.sum(), [leaf])


def test_second_derivatives_are_refused():
    q = randn(1, 40, 2, 32).requires_grad_()
    x = randn(2, 50, 32).requires_grad_()
    for out, leaf in ((fb.attention_autograd(q, q, q), q), (fb.group_norm_autograd(x, 4), x),
                      (fb.dropout_autograd(x, 0.5, 1), x)):
        (g,) = torch.autograd.grad((out * out).sum(), [leaf], create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.sum().backward()


def test_a_mask_that_wants_a_gradient_is_refused():
    q = randn(1, 4, 2, 32)
    mask = randn(1, 1, 4, 4).requires_grad_()
    for call in (fb.attention_forward, fb.attention_autograd):
        with pytest.raises(ValueError, match="gets no gradient"):
            call(q, q, q, mask=mask)


# ---- streams and threads -----------------------------------------------------------------------


def test_from_several_threads():
    """Each thread on a stream of its own, all entry points, the same bits as alone."""
    q, k = randn(2, 150, 4, 32, dtype=BF16), randn(2, 1000, 4, 32, dtype=BF16)
    x, w = randn(2, 3000, 64, dtype=BF16), randn(64)
    g = randn(2, 150, 4, 32, dtype=BF16, seed=3)

    def work():
        stats = torch.empty((2, 4, 150, 2), device="cuda")
        out = fb.attention_forward(q, k, k, stats=stats)
        r = fb.attention_backward(g, q, k, k, out, stats)
        y = fb.group_norm_forward(x, 8, w)
        z = fb.dropout_forward(y, 0.1, 5, residual=x)
        return [out, r["q"], r["k"], r["v"], y, z]

    want = work()
    torch.cuda.synchronize()
    bad = []

    def run():
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(10):
                got = work()
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    bad.append(1)

    threads = [threading.Thread(target=run) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_stream_argument():
    s = torch.cuda.Stream()
    q, k, x = randn(1, 5, 4, 32), randn(1, 4000, 4, 32), randn(2, 3000, 64)
    want = fb.attention_forward(q, k, k), fb.group_norm_forward(x, 8), fb.dropout_forward(x, 0.5, 1)
    s.wait_stream(torch.cuda.current_stream())
    got = (fb.attention_forward(q, k, k, stream=s), fb.group_norm_forward(x, 8, stream=s),
           fb.dropout_forward(x, 0.5, 1, stream=s))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- together ----------------------------------------------------------------------------------


def layer(ops, maps, queries, p):
    """A decoder's layer: group-normed maps to keys and values, the queries' attention to them, its
    projection dropped out onto the queries, a norm, a feed-forward with dropout."""
    B, M, C = maps.shape
    f = ops["group_norm"](maps, 8, p["gw"], p["gb"], "silu")
    kv = ops["linear"](f, p["wkv"])
    k, v = kv.reshape(B, M, 2, 4, C // 4).unbind(2)
    q = ops["linear"](queries, p["wq"]).reshape(B, -1, 4, C // 4)
    a = ops["attention"](q, k, v, p["lengths"]).reshape(B, -1, C)
    s = ops["dropout"](ops["linear"](a, p["wo"]), 11, queries)
    y = ops["norm"](s, p["nw"])
    h = ops["dropout"](ops["linear"](y, p["w1"], "gelu"), 12, None)
    return ops["linear"](h, p["w2"])


def test_a_layer_and_its_gradients():
    B, M, Q, C = 2, 600, 90, 64
    p = {"gw": 1 + randn(C, std=0.1), "gb": randn(C, std=0.1), "nw": 1 + randn(C, std=0.1, seed=1),
         "lengths": torch.tensor([600, 433], dtype=torch.int32, device="cuda")}
    for i, (n, o) in enumerate((("wkv", 2 * C), ("wq", C), ("wo", C), ("w1", 4 * C))):
        p[n] = randn(o, C, std=C ** -0.5, seed=i)
    p["w2"] = randn(C, 4 * C, std=(4 * C) ** -0.5, seed=9)
    maps, queries, g = randn(B, M, C), randn(B, Q, C, seed=1), randn(B, Q, C, seed=2)
    own = {"group_norm": fb.group_norm_autograd, "linear": lambda x, w, act="none": fb.linear_autograd(x, w, None, act),
           "attention": lambda q, k, v, n: fb.attention_autograd(q, k, v, key_lengths=n),
           "dropout": lambda x, seed, r: fb.dropout_autograd(x, 0.2, seed, residual=r),
           "norm": lambda s, w: fb.norm_autograd(s, w)[0]}
    leaves = [n for n in p if n != "lengths"]
    t = {n: v.clone().requires_grad_() if n in leaves else v for n, v in p.items()}
    ins = [maps.clone().requires_grad_(), queries.clone().requires_grad_()]
    out = layer(own, *ins, t)
    got = torch.autograd.grad(out, ins + [t[n] for n in leaves], g)

    def drop(x, seed, r):
        keep = ref.kept(x.numel(), 0.2, seed, 0).reshape(x.shape).cuda()
        y = torch.where(keep, x / 0.8, 0.0)
        return y if r is None else r + y

    def attend(q, k, v, lengths):
        s = torch.einsum("bihd,bjhd->bhij", q, k) * q.shape[-1] ** -0.5
        s = s.masked_fill(torch.arange(s.shape[-1], device="cuda") >= lengths[:, None, None, None], float("-inf"))
        return torch.einsum("bhij,bjhd->bihd", torch.softmax(s, -1), v)

    F = torch.nn.functional
    plain = {"group_norm": lambda x, n, w, b, act: F.silu(F.group_norm(x.transpose(1, 2), n, w, b).transpose(1, 2)),
             "linear": lambda x, w, act="none": F.gelu(x @ w.t()) if act == "gelu" else x @ w.t(), "attention": attend,
             "dropout": drop, "norm": lambda s, w: F.layer_norm(s, (C,), w)}
    t64 = {n: v.double().requires_grad_() if n in leaves else v for n, v in p.items()}
    ins64 = [maps.double().requires_grad_(), queries.double().requires_grad_()]
    want_out = layer(plain, *ins64, t64)
    want = torch.autograd.grad(want_out, ins64 + [t64[n] for n in leaves], g.double())
    # float32 through some ten operators of up to 600 terms, relative to each tensor's size
    for n, a, b in zip(["out", "maps", "queries", *leaves], (out, *got), (want_out, *want)):
        assert (a.detach().double() - b.detach()).norm() <= 2e-5 * b.detach().norm(), n
