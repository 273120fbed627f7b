"""The encoder block's operators as a program uses them: together with FlashSCA, on
side streams, in captured graphs, from several threads, and over random sizes."""
import random
import threading

import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

import block_ref as ref  # noqa: E402
import test_gpu_norm as tn  # noqa: E402
import test_gpu_sca as ts  # noqa: E402


@pytest.fixture(scope="module")
def fb():
    import paper_2607_10071_amd as m
    return m


def leaf(gen, *shape, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen) * std + mean).cuda().requires_grad_()


def test_a_block_around_flashsca(fb, device):
    """Norm, value projection, offsets and logits, FlashSCA, output projection onto
    the residual, norm with a gate, feed-forward: every product and norm of one
    forward and backward pass against float64, given what reached it."""
    inst = ts.small(77, C=64, heads=8, X=13, Y=11)
    wl = inst.wl
    value_in, l2i, off0, lg0 = ts._dev(inst, device)
    grid, img = fb.grid_of(wl), (wl.img_h, wl.img_w)
    B, Q, C = wl.B, wl.X * wl.Y, wl.C
    heads, L, P = off0.shape[2:5]
    gen = torch.Generator().manual_seed(5)
    q = leaf(gen, B, Q, C)
    feats = value_in.detach().clone().requires_grad_()
    w = {k: leaf(gen, n, c, std=c ** -0.5) for k, n, c in (
        ("value", C, C), ("offsets", heads * L * P * 2, C), ("logits", heads * L * P, C), ("out", C, C),
        ("up", 2 * C, C), ("down", C, 2 * C))}
    b = {k: leaf(gen, t.shape[0], std=0.1) for k, t in w.items()}
    n1, n2 = leaf(gen, C, std=0.1, mean=1.0), leaf(gen, C, std=0.1, mean=1.0)
    c1, c2 = leaf(gen, C, std=0.1), leaf(gen, C, std=0.1)
    gate = leaf(gen, B, C, std=0.3, mean=0.5)
    calls = []

    def linear(name, x, act="none", residual=None):
        out = fb.linear_autograd(x, w[name], b[name], act, residual)
        calls.append(("linear", x, w[name], b[name], act, residual, out))
        return out

    def norm(x, weight, bias, residual=None, gate=None):
        y, s = fb.norm_autograd(x, weight, bias, residual, gate)
        calls.append(("norm", x, weight, bias, residual, gate, y, s))
        return y, s

    y, stream = norm(q, n1, c1)
    value = linear("value", feats)
    offsets = linear("offsets", y).view_as(off0)
    logits = linear("logits", y).view_as(lg0)
    mixed = fb.sca_autograd(value, l2i, inst.z, grid, img, wl.levels, wl.heads, offsets, logits)
    attended = linear("out", mixed, residual=stream)
    y, stream = norm(attended, n2, c2, residual=q, gate=gate)
    out = linear("down", linear("up", y, act="gelu"), residual=stream)

    grads = {}
    for call in calls:
        for k, t in enumerate(call):
            if isinstance(t, torch.Tensor) and id(t) not in grads:
                grads[id(t)] = None
                if not t.is_leaf:
                    t.retain_grad()
    g = torch.randn(out.shape, generator=gen).cuda()
    out.backward(g)
    flat = lambda t: None if t is None else t.detach().reshape(-1, t.shape[-1]).cpu()
    for call in calls:
        if call[0] == "linear":
            _, x, wt, bias, act, residual, o = call
            want, pre, e, e_pre = ref.linear(flat(x), wt.detach().cpu(), bias.detach().cpu(), act,
                                             flat(residual), 1.0)
            ref.close(flat(o), want, e)
            # the backward reads the sums before the activation in float32
            exact = ref.linear_grads(flat(o.grad), flat(x), wt.detach().cpu(), pre, act, 1.0,
                                     torch.float32, act != "none")
            # an activation's second derivative is at most 0.8
            more = 0.8 * flat(o.grad).double().abs() * (e_pre + ref.F32 * pre.abs()) if act != "none" else 0
            v, e = exact["weight"]
            ref.close(wt.grad, v, e + (more.t() @ flat(x).double().abs() if act != "none" else 0))
            v, e = exact["bias"]
            ref.close(bias.grad, v, e + (more.sum(0) if act != "none" else 0))
        else:
            _, x, weight, bias, residual, gt, yy, ss = call
            want, e, _, _ = ref.stream(flat(x), flat(residual), None if gt is None else gt.detach().cpu(),
                                       1.0, None, None, None, 1e-5)
            ref.close(flat(ss), want, e)
            ref.close(flat(yy), *ref.normed(flat(ss), "layer", 1e-5, weight.detach().cpu(),
                                            bias.detach().cpu()))
            # without anything to add s is x, whose gradient holds this norm's share too
            gs = flat(ss.grad) if residual is not None else None
            exact = ref.norm_grads(flat(yy.grad), gs, flat(x), flat(ss),
                                   None if gt is None else gt.detach().cpu(), 1.0, "layer",
                                   weight.detach().cpu(), None, None, None, 1e-5)
            ref.close(weight.grad, *exact["weight"])
            ref.close(bias.grad, *exact["bias"])
            if gt is not None:
                ref.close(gt.grad, *exact["gate"])
                # the norm alone reads `attended`
                ref.close(flat(x.grad), *exact["x"])
    assert all(torch.isfinite(t.grad).all() and t.grad.abs().max() > 0 for t in (q, feats))


def test_saved_tensors_moved_by_hooks(fb, device):
    """Inputs that are rows inside wider tensors, packed to contiguous copies: the
    backward goes by the strides of what it gets."""
    gen = torch.Generator().manual_seed(3)
    big, w = leaf(gen, 50, 90), leaf(gen, 64, 40)
    gate = leaf(gen, 64)
    g = torch.randn(50, 64, generator=gen).cuda()

    def step():
        x = big[:, 5:45]
        h = fb.linear_autograd(x, w, None, "silu")
        y, s = fb.norm_autograd(big[:, 20:84], gate, None, h, gate, post_norm="rms")
        return torch.autograd.grad([y, s], [big, w, gate], [g, g])

    want = step()
    with torch.autograd.graph.save_on_cpu():
        got = step()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def passes(fb, seed=0, dtype=torch.bfloat16, M=600, C=256):
    """A few calls of each kind with workspaces among them, as functions of inputs
    that stay where they are."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    ins = {"x": rand(M, C), "w": rand(512, C), "b": rand(512), "g": rand(M, 512), "pre": rand(M, 512),
           "r": rand(M, C), "gate": rand(C), "n": rand(C), "long": rand(96, 8192), "wl": rand(64, 8192),
           "one": rand(1, C), "many": rand(4096, 512), "wide": rand(4096, 512)}

    def run():
        i = ins
        out = [fb.linear_forward(i["x"], i["w"], i["b"], "gelu"),
               fb.linear_forward(i["long"], i["wl"]), fb.linear_forward(i["one"], i["w"], i["b"])]
        out.append(fb.linear_forward(i["many"], i["wide"]))   # 256 x 256 tiles
        out += fb.linear_backward(i["g"], i["x"], i["w"], i["pre"], "gelu", 0.5).values()
        y, s = fb.norm_forward(i["x"], i["n"], None, i["r"], i["gate"], 0.5, "rms", "layer")
        out += [y, s]
        out += fb.norm_backward(i["r"], i["x"], i["x"], s, i["n"], i["gate"], 0.5, "rms", "layer",
                                want=("x", "residual", "gate", "weight")).values()
        return out

    return ins, run


def refill(ins, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for t in ins.values():
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))


def test_side_streams(fb, device):
    ins, run = passes(fb)
    want = [t.clone() for t in run()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(4):   # calls on several streams at once, each with workspaces of its own
        for st in streams:
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


def test_stream_arguments(fb, device):
    """stream= with a Stream and with its raw handle, on tensors of the default one."""
    ins, _ = passes(fb)
    want = fb.linear_forward(ins["long"], ins["wl"])
    wb = fb.linear_backward(ins["g"], ins["x"], ins["w"], ins["pre"], "silu")
    wy, wsum = fb.norm_forward(ins["x"], ins["n"], None, ins["r"])
    wn = fb.norm_backward(ins["r"], None, ins["x"], wsum, ins["n"], want=("x", "weight"))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for handle in (st, st.cuda_stream, 0):
        out = torch.empty_like(want)
        fb.linear_forward(ins["long"], ins["wl"], out=out, stream=handle)
        b = fb.linear_backward(ins["g"], ins["x"], ins["w"], ins["pre"], "silu", stream=handle)
        y, s = fb.norm_forward(ins["x"], ins["n"], None, ins["r"], stream=handle)
        n = fb.norm_backward(ins["r"], None, ins["x"], s, ins["n"], want=("x", "weight"), stream=handle)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(y, wy) and torch.equal(s, wsum)
        assert all(torch.equal(b[k], wb[k]) for k in wb) and all(torch.equal(n[k], wn[k]) for k in wn)


def test_graphs(fb, device):
    """Two captured graphs, replayed in turns with new inputs, eager work and
    synchronizations between the replays."""
    ins, run = passes(fb)
    run()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out))
    for k in range(4):
        refill(ins, 100 + k)
        want = [t.clone() for t in run()]
        for g, out in graphs if k % 2 else graphs[::-1]:
            for t in out:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_a_training_pass_in_a_graph(fb, device):
    gen = torch.Generator().manual_seed(1)
    x, w, b, r, n, gate = (leaf(gen, *s) for s in ((300, 128), (128, 128), (128,), (300, 128), (128,),
                                                  (128,)))
    leaves = [x, w, b, r, n, gate]
    g = torch.randn(300, 128, generator=gen).cuda()

    def step():
        h = fb.linear_autograd(x, w, b, "gelu_tanh", r)
        y, s = fb.norm_autograd(h, n, None, r, gate, norm="rms")
        return [y, s, *torch.autograd.grad([y, s], leaves, [g, g])]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [t.detach() for t in step()]
    for k in range(3):
        with torch.no_grad():
            for t in leaves:
                t.copy_(torch.randn(t.shape, generator=gen))
        graph.replay()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b.detach()) for a, b in zip(got, want)), k


def test_prepared_calls(fb, device):
    """The same calls again on the same tensors, with new values in them, on their
    stream and in a graph."""
    ins, _ = passes(fb)
    i = ins
    outs = {"long": torch.empty(96, 64, dtype=torch.bfloat16, device=device),
            "one": torch.empty(1, 512, device=device), "y": torch.empty_like(i["x"]),
            "s": torch.empty_like(i["x"]), "n": torch.empty_like(i["x"])}
    calls = [fb.prepare_linear_forward(i["long"], i["wl"], out=outs["long"]),
             fb.prepare_linear_forward(i["one"], i["w"], i["b"], "silu", out=outs["one"]),
             fb.prepare_norm_forward(i["x"], i["n"], None, i["r"], i["gate"], 0.5, "rms", out=outs["y"],
                                     out_s=outs["s"]),
             fb.prepare_norm_forward(i["x"], i["n"], out=outs["n"])]

    def want():
        y, s = fb.norm_forward(i["x"], i["n"], None, i["r"], i["gate"], 0.5, "rms")
        return {"long": fb.linear_forward(i["long"], i["wl"]),
                "one": fb.linear_forward(i["one"], i["w"], i["b"], "silu", out_dtype=torch.float32),
                "y": y, "s": s, "n": fb.norm_forward(i["x"], i["n"])[0]}

    for k in range(3):
        refill(ins, k)
        for call in calls:
            call()
        torch.cuda.synchronize()
        w = want()
        assert all(torch.equal(outs[n], w[n]) for n in w)
    with pytest.raises(ValueError):
        fb.prepare_linear_forward(i["x"], i["w"])
    with pytest.raises(ValueError):
        fb.prepare_norm_forward(i["x"], i["n"], residual=i["r"], out=outs["y"])


def test_threads(fb, device):
    ins, run = passes(fb)
    want = [t.clone() for t in run()]
    torch.cuda.synchronize()
    bad = []

    def work():
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            for _ in range(5):
                got = run()
                st.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    bad.append(1)

    ts_ = [threading.Thread(target=work) for _ in range(3)]
    for t in ts_:
        t.start()
    for t in ts_:
        t.join()
    assert not bad


@pytest.mark.parametrize("M,K,N", [(600, 256, 256), (70000, 512, 256), (96, 8192, 64), (20, 264, 72)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_places_that_are_no_multiple_of_16_bytes(fb, device, M, K, N, dtype):
    """Widths that the streamed kernel takes at addresses and strides it does not: the
    checked one takes the same plan, workspace and all."""
    dt = ref.DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(M)
    big = torch.randn(M, K + 3, generator=gen, device=device).to(dt)
    x = big[:, 1:K + 1]
    w = torch.randn(N, K, generator=gen, device=device).to(dt)
    g = torch.randn(M, N, generator=gen, device=device).to(dt)
    got, want = fb.linear_forward(x, w), fb.linear_forward(x.contiguous(), w)
    mag = x.abs().double() @ w.abs().double().t()
    # the same exact sum in two orders, each rounded
    lim = 2 * ((K + 2) * ref.F32 * mag + ref.u(dt) * (want.double().abs() + K * ref.F32 * mag))
    assert ((got.double() - want.double()).abs() <= lim).all()
    a = fb.linear_backward(g, x, w)
    b = fb.linear_backward(g, x.contiguous(), w)
    assert torch.equal(a["bias"], b["bias"])
    mag = g.abs().double().t() @ x.abs().double()
    lim = 2 * ((M + 2) * ref.F32 * mag + ref.u(dt) * (b["weight"].double().abs() + M * ref.F32 * mag))
    assert ((a["weight"].double() - b["weight"].double()).abs() <= lim).all()


def test_random_linears(fb, device):
    rng = random.Random(11)
    gen = torch.Generator().manual_seed(11)
    for _ in range(40):
        dtype = rng.choice(list(ref.DTYPES))
        dt = ref.DTYPES[dtype]
        M, K, N = (max(1, int(2 ** rng.uniform(0, hi))) for hi in (10, 11, 10))
        if rng.random() < 0.5:
            K, N = -(-K // 8) * 8, -(-N // 8) * 8
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        odt = torch.float32 if rng.random() < 0.3 else dt
        x = torch.randn(M, K, generator=gen).to(dt)
        w = (torch.randn(N, K, generator=gen) * K ** -0.5).to(dt)
        b = torch.randn(N, generator=gen).to(dt) if rng.random() < 0.7 else None
        r = torch.randn(M, N, generator=gen).to(odt) if rng.random() < 0.5 else None
        print("linear", M, K, N, dtype, act, flush=True)
        cuda = lambda t: None if t is None else t.cuda()
        pre = torch.empty(M, N, dtype=dt, device=device)
        want, _, e, _ = ref.linear(x, w, b, act, r, 0.75)
        ref.close(fb.linear_forward(cuda(x), cuda(w), cuda(b), act, cuda(r), 0.75, out_dtype=odt, pre=pre),
                  want, e)
        g = torch.randn(M, N, generator=gen).to(odt)
        got = fb.linear_backward(g.cuda(), cuda(x), cuda(w), pre, act, 0.75)
        exact = ref.linear_grads(g, x, w, pre.cpu(), act, 0.75, dt, act != "none" or odt != dt)
        for k in got:
            ref.close(got[k], *exact[k])


def test_random_norms(fb, device):
    rng = random.Random(12)
    for n in range(40):
        types = rng.choice(tn.TYPES)
        G = rng.choice([1, 1, 2, 3, 5])
        M = G * max(1, int(2 ** rng.uniform(0, 8)))
        C = max(1, int(2 ** rng.uniform(0, 12)))
        kind, post = rng.choice([("layer", None), ("rms", None), ("layer", "layer"), ("rms", "rms"),
                                 (None, "rms")])
        gate = rng.choice([None, "channel", "sample"])
        t, gy, gs = tn.make(n, M, C, types, kind or "layer", post, rng.random() < 0.7, gate,
                            rng.random() < 0.8, G)
        if not kind:
            t["weight"] = t["bias"] = None
        print("norm", M, C, types, kind, post, gate, G, flush=True)
        tn.check_forward(fb, t, kind, post, 0.75, 1e-5, G)
        tn.check_backward(fb, t, gy, gs, kind, post, 0.75, 1e-5, G)
