"""The block operators together, as a residual block of a model calls them: norm, one projection to q, k and v, linear attention over strided parts
of its result, a norm for each head, the projection back with the residual, then norm, a projection with GeLU and one back; forward, backward,
a token after a prompt, in workspaces full of what is no number, and captured.  Every stage is held to its bound at the inputs that it had."""
import pytest
import torch

import block_oracle as bo
from test_gpu_linear import forward_bounds

pytestmark = pytest.mark.gpu
DT = dict(bf16=torch.bfloat16, f32=torch.float32)
B, H, DH, D, U = 2, 3, 64, 200, 328
A = H * DH


def params(io):
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = lambda n, k: (rnd(n, k) * k ** -0.5).to(DT[io])  # noqa: E731
    return dict(w1=1 + 0.1 * rnd(D), wqkv=w(3 * A, D), bqkv=0.1 * rnd(3 * A), ld=torch.tensor([-0.3, -0.02, -0.001], device="cuda"), wh=1 + 0.1 * rnd(DH),
                wo=w(D, A), w3=1 + 0.1 * rnd(D), b3=0.1 * rnd(D), wu=w(U, D), bu=0.1 * rnd(U), wd=w(D, U))


def inputs(T, io, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return rnd(B, T, D).to(DT[io]), rnd(B, H, DH, DH), rnd(B, T, D).to(DT[io])


def heads(qkv):
    return [qkv[..., i * A:(i + 1) * A].unflatten(-1, (H, DH)) for i in range(3)]


def forward(p, x, s0, ws):
    from paper_2402_19427_b200 import binding
    f = {}
    f["h"], _, f["r1"] = binding.layer_norm(x, p["w1"], center=False, stats=True)
    f["qkv"] = binding.linear(f["h"], p["wqkv"], p["bqkv"], workspace=ws)
    f["o"], f["s"] = binding.linear_attention_prefill(*heads(f["qkv"]), p["ld"], s0=s0, workspace=ws)
    f["oh"], _, f["r2"] = binding.layer_norm(f["o"], p["wh"], center=False, stats=True)
    f["y"] = binding.linear(f["oh"].flatten(-2), p["wo"], residual=x, workspace=ws)
    f["n"], f["m3"], f["r3"] = binding.layer_norm(f["y"], p["w3"], p["b3"], stats=True)
    f["u"], f["z"] = binding.linear(f["n"], p["wu"], p["bu"], "gelu", keep_preact=True, workspace=ws)
    f["out"] = binding.linear(f["u"], p["wd"], residual=f["y"], workspace=ws)
    return f


def backward(p, x, s0, f, dout, ws):
    from paper_2402_19427_b200 import binding
    g = {}
    g["d"] = binding.linear_backward(dout, f["u"], p["wd"], need=("x", "weight"), workspace=ws)
    g["u"] = binding.linear_backward(g["d"]["x"], f["n"], p["wu"], preact=f["z"], activation="gelu", workspace=ws)
    g["n3"] = binding.layer_norm_backward(g["u"]["x"], f["y"], f["r3"], mean=f["m3"], weight=p["w3"], workspace=ws)
    g["dy"] = g["n3"]["x"] + dout
    g["o"] = binding.linear_backward(g["dy"], f["oh"].flatten(-2), p["wo"], need=("x", "weight"), workspace=ws)
    g["nh"] = binding.layer_norm_backward(g["o"]["x"].unflatten(-1, (H, DH)), f["o"], f["r2"], weight=p["wh"], workspace=ws)
    dqkv = torch.empty_like(f["qkv"])
    dq, dk, dv = heads(dqkv)
    g["mix"] = binding.linear_attention_backward(*heads(f["qkv"]), p["ld"], g["nh"]["x"], s0=s0, state_grads=True, dq=dq, dk=dk, dv=dv, workspace=ws)
    g["qkv"] = binding.linear_backward(dqkv, f["h"], p["wqkv"], workspace=ws)
    g["n1"] = binding.layer_norm_backward(g["qkv"]["x"], x, f["r1"], weight=p["w1"], workspace=ws)
    g["dx"] = g["n1"]["x"] + g["dy"]
    return g


def flat(results):
    return [t for v in results.values() for t in (v.values() if isinstance(v, dict) else [v]) if t is not None]


def workspace():
    return torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")   # NaN in every type, and no number of anything


def check_norm(name, got, x, w, b, center, dt):
    ref, mu, r = bo.norm(x, w, b, 1e-5, center)
    bo.assert_within(name, got, ref, bo.norm_bound(x, w, b, mu, r, dt, ref))


def check_linear(name, got, x, w, bias, kind, res, dt):
    ref, z, mag = bo.linear(x, w, bias, kind, res)
    bo.assert_within(name, got, ref, forward_bounds(res, kind, ref, z, mag, dt, x.shape[-1])[1])


def check_forward(p, x, s0, f, dt):
    check_norm("h", f["h"], x, p["w1"], None, False, dt)
    check_linear("qkv", f["qkv"], f["h"], p["wqkv"], p["bqkv"], "none", None, dt)
    o, s, om, sm = bo.attention(*heads(f["qkv"]), p["ld"], s0, DH ** -0.5)
    T = x.shape[1]
    bo.assert_within("o", f["o"], o, bo.attention_bound(om, o, dt, T))
    bo.assert_within("s", f["s"], s, bo.state_bound(sm, T))
    check_norm("oh", f["oh"], f["o"], p["wh"], None, False, dt)
    check_linear("y", f["y"], f["oh"].flatten(-2), p["wo"], None, "none", x, dt)
    check_norm("n", f["n"], f["y"], p["w3"], p["b3"], True, dt)
    check_linear("u", f["u"], f["n"], p["wu"], p["bu"], "gelu", None, dt)
    check_linear("out", f["out"], f["u"], p["wd"], None, "none", f["y"], dt)


def check_linear_backward(name, got, dy, x, w, pre, kind, dt):
    dy, x = dy.flatten(0, -2).double(), x.flatten(0, -2).double()
    w, M, N = w.double(), x.shape[0], w.shape[0]
    dz = dy * (bo.act_slope(pre.flatten(0, -2).double(), kind) if pre is not None else 1.0)
    near = 0.0 if kind == "none" else 1.01 * bo.half_step(dt)   # dz rounded to the io type, the slope off by its terms: as in the projection's own tests
    slope = 0.0 if kind == "none" else 20 * bo.U32 * dy.abs()
    term = lambda n: (near + 2 * n * bo.U32) * dz.abs() + slope  # noqa: E731
    dx, dw = dz @ w, dz.T @ x
    bo.assert_within(name + " dx", got["x"].flatten(0, -2), dx, term(N) @ w.abs() + bo.half_step(dt) * dx.abs())
    bo.assert_within(name + " dw", got["weight"], dw, term(M).T @ x.abs() + bo.half_step(dt) * dw.abs())
    if "bias" in got:
        bo.assert_within(name + " db", got["bias"], dz.sum(0), ((24 + M) * bo.U32 * dz.abs() + slope).sum(0) + 1e-30)


def check_norm_backward(name, got, dy, x, mean, r, w, dt):
    ref = bo.norm_backward(dy, x, mean, r, w, mean is not None)
    bo.assert_within(name + " dx", got["x"], ref[0], 80 * bo.U32 * ref[3] + bo.half_step(dt) * ref[0].abs())
    bo.assert_within(name + " dw", got["weight"], ref[1], 64 * bo.U32 * ref[4] + 1e-30)
    bo.assert_within(name + " db", got["bias"], ref[2], 64 * bo.U32 * ref[5] + 1e-30)


def check_backward(p, x, s0, f, dout, g, dt):
    check_linear_backward("d", g["d"], dout, f["u"], p["wd"], None, "none", dt)
    check_linear_backward("u", g["u"], g["d"]["x"], f["n"], p["wu"], f["z"], "gelu", dt)
    check_norm_backward("n3", g["n3"], g["u"]["x"], f["y"], f["m3"], f["r3"], p["w3"], dt)
    check_linear_backward("o", g["o"], g["dy"], f["oh"].flatten(-2), p["wo"], None, "none", dt)
    check_norm_backward("nh", g["nh"], g["o"]["x"].unflatten(-1, (H, DH)), f["o"], None, f["r2"], p["wh"], dt)
    ref, mag = bo.attention_backward(*heads(f["qkv"]), p["ld"], g["nh"]["x"], s0, None, DH ** -0.5)
    T = x.shape[1]
    for n in "qkv":
        bo.assert_within("d" + n, g["mix"][n], ref[n], bo.attention_bound(mag[n], ref[n], dt, T))
    bo.assert_within("ds0", g["mix"]["s0"], ref["s0"], bo.state_bound(mag["s0"], T))
    dqkv = torch.cat([g["mix"][n].flatten(-2) for n in "qkv"], -1)
    check_linear_backward("qkv", g["qkv"], dqkv, f["h"], p["wqkv"], None, "none", dt)
    check_norm_backward("n1", g["n1"], g["qkv"]["x"], x, None, f["r1"], p["w1"], dt)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 150, 260])
def test_forward_and_backward(T, io):
    p, ws = params(io), workspace()
    x, s0, dout = inputs(T, io)
    f = forward(p, x, s0, ws)
    check_forward(p, x, s0, f, DT[io])
    g = backward(p, x, s0, f, dout, ws)
    check_backward(p, x, s0, f, dout, g, DT[io])
    ws.fill_(255)
    assert all(torch.equal(a, b) for a, b in zip(flat(f), flat(forward(p, x, s0, ws))))
    assert all(torch.equal(a, b) for a, b in zip(flat(g), flat(backward(p, x, s0, f, dout, ws))))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_tokens_after_a_prompt(io):
    """Each stage of a step at its own inputs; the mixer over the whole of what the prompt and the steps fed it."""
    from paper_2402_19427_b200 import binding
    p, ws, dt, T, N = params(io), workspace(), DT[io], 140, 4
    x, s0, _ = inputs(T + N, io)
    f = forward(p, x[:, :T].contiguous(), s0, ws)
    fed, outs, s = [f["qkv"]], [f["o"]], f["s"]
    for t in range(T, T + N):
        xt = x[:, t].contiguous()
        h = binding.layer_norm(xt, p["w1"], center=False)
        check_norm("h", h, xt, p["w1"], None, False, dt)
        qkv = binding.linear(h, p["wqkv"], p["bqkv"], workspace=ws)
        check_linear("qkv", qkv, h, p["wqkv"], p["bqkv"], "none", None, dt)
        o = binding.linear_attention_decode_step(*(a.contiguous() for a in heads(qkv)), p["ld"], s)
        oh = binding.layer_norm(o, p["wh"], center=False)
        check_norm("oh", oh, o, p["wh"], None, False, dt)
        y = binding.linear(oh.flatten(-2), p["wo"], residual=xt, workspace=ws)
        check_linear("y", y, oh.flatten(-2), p["wo"], None, "none", xt, dt)
        fed.append(qkv[:, None])
        outs.append(o[:, None])
    o, sr, om, sm = bo.attention(*heads(torch.cat(fed, 1)), p["ld"], s0, DH ** -0.5)
    bo.assert_within("o", torch.cat(outs, 1), o, bo.attention_bound(om, o, dt, T + N))
    bo.assert_within("s", s, sr, bo.state_bound(sm, T + N))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_two_graphs_in_one_workspace(io):
    """Captured forward and backward of two inputs that share a workspace, replayed in turn, and again after the inputs have changed"""
    p, ws = params(io), workspace()
    runs = []
    for T, seed in ((150, 1), (33, 2)):
        x, s0, dout = inputs(T, io, seed)
        step = lambda x=x, s0=s0, dout=dout: (lambda f: (f, backward(p, x, s0, f, dout, ws)))(forward(p, x, s0, ws))  # noqa: E731
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f, g = step()
        runs.append((graph, step, x, f, g))
    for change in range(2):
        for graph, step, x, f, g in runs:
            if change:
                x.copy_(-0.5 * x)
            graph.replay()
        for graph, step, x, f, g in runs[::-1]:
            graph.replay()
            fe, ge = step()
            assert all(torch.equal(a, b) for a, b in zip(flat(f) + flat(g), flat(fe) + flat(ge)))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_two_streams_at_once(io):
    """Two users' blocks on streams of their own, each with its workspace, while the default stream idles"""
    p = params(io)
    users = [(inputs(T, io, seed), workspace(), torch.cuda.Stream()) for T, seed in ((260, 4), (150, 5))]
    step = lambda x, s0, dout, ws: (lambda f: flat(f) + flat(backward(p, x, s0, f, dout, ws)))(forward(p, x, s0, ws))  # noqa: E731
    alone = [step(*data, ws) for data, ws, _ in users]
    torch.cuda.synchronize()
    results = [[], []]
    for _ in range(5):
        for i, (data, ws, stream) in enumerate(users):
            with torch.cuda.stream(stream):
                results[i].append(step(*data, ws))
    torch.cuda.synchronize()
    for runs, want in zip(results, alone):
        assert all(torch.equal(a, b) for run in runs for a, b in zip(run, want))
