"""rglru_linear and its backward against fp64: sizes around the tiles' borders, single tokens, odd sizes, each activation and type."""
import pytest
import torch

import block_oracle as bo
from util import Guarded

pytestmark = pytest.mark.gpu
DT = dict(bf16=torch.bfloat16, f32=torch.float32)


def make(M, K, N, io, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + M + 3 * K + 5 * N)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[io]
    return dict(x=rnd(M, K).to(dt), weight=(rnd(N, K) * K ** -0.5).to(dt), bias=0.3 * rnd(N), residual=rnd(M, N).to(dt), dy=rnd(M, N).to(dt), preact=(1.5 * rnd(M, N)).to(dt))


def forward_bounds(t, kind, y, z, mag, dt, K):
    """A sum of K products in fp32, in any order and whichever way it rounds: 2 K half steps of the terms' magnitude.  The activations'
    slopes are below 1.13, their own arithmetic takes some ten roundings of values up to |z|."""
    off = (2 * K + 4) * bo.U32 * mag
    r = 0.0 if t is None else t.double().abs()
    return off + bo.half_step(dt) * z.abs(), 1.13 * off + 16 * bo.U32 * (z.abs() + r) + bo.half_step(dt) * y.abs()


def run_forward(M, K, N, io, kind, with_bias=True, with_residual=True, flags=0):
    from paper_2402_19427_b200 import binding
    t = make(M, K, N, io)
    bias, res = (t["bias"] if with_bias else None), (t["residual"] if with_residual else None)
    g = Guarded()
    y = g.empty((M, N), DT[io])
    got, pre = binding.linear(t["x"], t["weight"], bias, kind, res, y=y, keep_preact=True, flags=flags)
    g.check()
    yr, z, mag = bo.linear(t["x"], t["weight"], bias, kind, res)
    zb, yb = forward_bounds(res, kind, yr, z, mag, DT[io], K)
    bo.assert_within("preact", pre, z, zb)
    bo.assert_within("y", got, yr, yb)
    plain = binding.linear(t["x"], t["weight"], bias, kind, res, flags=flags)
    assert torch.equal(plain, got)


def run_backward(M, K, N, io, kind, flags=0):
    from paper_2402_19427_b200 import binding
    t, dt = make(M, K, N, io), DT[io]
    pre = t["preact"] if kind != "none" else None
    got = binding.linear_backward(t["dy"], t["x"], t["weight"], preact=pre, activation=kind, flags=flags)
    dz = t["dy"].double() * (bo.act_slope(pre.double(), kind) if pre is not None else 1.0)
    x, w = t["x"].double(), t["weight"].double()
    # dz goes into the products in the io type: half a step of each term; sums as in the forward.  The slope is a sum of two terms of up to
    # 1.2 that cancel near its zero (z = -0.75 for GeLU): what is left is off by some 16 half steps of the terms, not of itself
    near = 0.0 if kind == "none" else 1.01 * bo.half_step(dt)
    dx, dw, db = dz @ w, dz.T @ x, dz.sum(0)
    slope = 0.0 if kind == "none" else 20 * bo.U32 * t["dy"].double().abs()
    term = lambda n: (near + 2 * n * bo.U32) * dz.abs() + slope  # noqa: E731
    bo.assert_within("dx", got["x"], dx, term(N) @ w.abs() + bo.half_step(dt) * dx.abs())
    bo.assert_within("dweight", got["weight"], dw, term(M).T @ x.abs() + bo.half_step(dt) * dw.abs())
    bo.assert_within("dbias", got["bias"], db, ((24 + M) * bo.U32 * dz.abs() + slope).sum(0) + 1e-30)
    again = binding.linear_backward(t["dy"], t["x"], t["weight"], preact=pre, activation=kind, flags=flags)
    assert all(torch.equal(got[k], again[k]) for k in got)
    some = binding.linear_backward(t["dy"], t["x"], t["weight"], preact=pre, activation=kind, need=("weight",), flags=flags)
    assert set(some) == {"weight"} and torch.equal(some["weight"], got["weight"])


SIZES = [(1, 2560, 2560), (1, 64, 8), (2, 256, 512), (3, 1000, 136), (8, 2560, 512), (16, 512, 2560), (17, 384, 1024), (33, 2560, 320), (64, 1536, 264),
         (65, 512, 512), (100, 264, 1032), (127, 136, 96), (129, 192, 520), (255, 1024, 256), (257, 2568, 264), (640, 512, 1000), (1500, 800, 640), (4096, 256, 256)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward(M, K, N, io):
    run_forward(M, K, N, io, "none")
    run_forward(M, K, N, io, "gelu", with_residual=False)
    run_forward(M, K, N, io, "silu", with_bias=False)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (5, 3, 7), (70, 65, 33), (130, 257, 129), (300, 1001, 77), (9, 4095, 11)])
def test_forward_and_backward_of_odd_sizes(M, K, N, io):
    for kind in ("none", "gelu"):
        run_forward(M, K, N, io, kind)
        run_backward(M, K, N, io, kind)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_backward(M, K, N, io):
    for kind in ("none", "gelu", "silu"):
        run_backward(M, K, N, io, kind)


def test_forced_generic():
    run_forward(200, 264, 136, "bf16", "gelu", flags=1)
    run_backward(200, 264, 136, "bf16", "gelu", flags=1)


def test_residual_stream_in_place_and_leading_dimensions():
    from paper_2402_19427_b200 import binding
    for M in (3, 300):
        t = make(M, 512, 512, "bf16")
        y = binding.linear(t["x"], t["weight"], residual=t["residual"])
        stream = t["residual"].clone()
        assert binding.linear(t["x"], t["weight"], residual=stream, y=stream).data_ptr() == stream.data_ptr()
        assert torch.equal(stream, y)
        assert torch.equal(binding.linear(t["x"].view(M, 1, 512), t["weight"], residual=t["residual"].view(M, 1, 512)), y.view(M, 1, 512))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("M", [4, 200])
def test_values_that_are_no_numbers_stay_in_their_row(M, io):
    from paper_2402_19427_b200 import binding
    t = make(M, 256, 264, io)
    clean = binding.linear(t["x"], t["weight"], t["bias"], "gelu")
    x = t["x"].clone(); x[1, 5] = float("nan"); x[2, 200] = float("inf")
    y = binding.linear(x, t["weight"], t["bias"], "gelu")
    keep = [i for i in range(M) if i not in (1, 2)]
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[1]).all()
    up = t["weight"][:, 200] > 0   # inf in, GeLU: inf where the weight is positive, 0 where it is negative
    assert torch.isinf(y[2][up]).all() and (y[2][t["weight"][:, 200] < 0] == 0).all()
    # slopes at infinity are 1 and 0
    pre = t["preact"].clone(); pre[0] = float("inf"); pre[1] = float("-inf")
    for kind in ("gelu", "silu"):
        dx = binding.linear_backward(t["dy"], t["x"], t["weight"], preact=pre, activation=kind)["x"]
        straight = binding.linear_backward(t["dy"], t["x"], t["weight"])["x"]
        assert torch.equal(dx[0], straight[0]) and (dx[1] == 0).all()


def test_gradients_against_differences():
    from paper_2402_19427_b200 import binding
    t = make(6, 40, 24, "f32")
    for kind in ("none", "gelu", "silu"):
        _, pre = binding.linear(t["x"], t["weight"], t["bias"], kind, keep_preact=True)
        got = binding.linear_backward(t["dy"], t["x"], t["weight"], preact=pre if kind != "none" else None, activation=kind)
        loss = lambda **a: float((bo.linear(a["x"], a["weight"], a["bias"], kind, None)[0] * t["dy"].double()).sum())  # noqa: E731
        args = {n: t[n].double() for n in ("x", "weight", "bias")}
        for name in args:
            for i in (0, 11, t[name].numel() - 1):
                e = torch.zeros_like(args[name]); e.view(-1)[i] = 1e-5
                diff = (loss(**{**args, name: args[name] + e}) - loss(**{**args, name: args[name] - e})) / 2e-5
                # third derivatives times 1e-10, 1e-16 / 1e-5 of the loss, fp32 roundings of sums of at most 40 terms below 4
                assert abs(diff - float(got[name].view(-1)[i])) <= 5e-5, (kind, name, i)


def test_graph_replay_and_two_streams():
    from paper_2402_19427_b200 import binding
    t = make(384, 512, 640, "bf16")
    call = lambda: (binding.linear(t["x"], t["weight"], t["bias"], "gelu", t["residual"]),  # noqa: E731
                    binding.linear_backward(t["dy"], t["x"], t["weight"], preact=t["preact"], activation="gelu"))
    y, g = call()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s in side:
            with torch.cuda.stream(s):
                got.append(call())
    torch.cuda.synchronize()
    for y1, g1 in got:
        assert torch.equal(y1, y) and all(torch.equal(g1[k], g[k]) for k in g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, g2 = call()
    graph.replay(); graph.replay(); torch.cuda.synchronize()
    assert torch.equal(y2, y) and all(torch.equal(g2[k], g[k]) for k in g)
