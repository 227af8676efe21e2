"""rglru_layer_norm and its backward against fp64, at widths on both sides of every layout, with and without centring, weights and sums."""
import pytest
import torch

import block_oracle as bo
from util import Guarded

pytestmark = pytest.mark.gpu
DT = dict(bf16=torch.bfloat16, f32=torch.float32)


def make(rows, N, io, seed=0, shift=0.3):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + (sum(rows) if isinstance(rows, tuple) else rows) + 7 * N)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = rnd(*(rows if isinstance(rows, tuple) else (rows,)), N) * 1.5 + shift
    return x.to(DT[io]), (1 + 0.2 * rnd(N)), 0.3 * rnd(N), torch.randn(x.shape, generator=g, device="cuda").to(DT[io])


# bf16: eight values a load (8, 16, 32 lanes, a block, 1024 threads, the long kernels), one a load (odd widths); fp32 likewise with four
WIDTHS = [1, 7, 8, 64, 65, 96, 128, 129, 256, 264, 257, 512, 520, 1000, 1531, 2560, 4096, 8191, 8192, 8200, 16384, 16392, 8193]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("N", WIDTHS)
def test_forward_and_backward(N, center, io):
    from paper_2402_19427_b200 import binding
    rows = 37 if N > 512 else 301
    x, w, b, dy = make(rows, N, io)
    g = Guarded()
    y = g.empty((rows, N), DT[io])
    out, mean, rstd = binding.layer_norm(x, w, b, center=center, stats=True, y=y)
    assert out.data_ptr() == y.data_ptr()
    yr, mu, r = bo.norm(x, w, b, 1e-5, center)
    bo.assert_within("y", y, yr, bo.norm_bound(x, w, b, mu, r, DT[io], yr))
    bo.assert_within("rstd", rstd, r, 200 * bo.U32 * r * (1 + (x.double().abs().amax(-1) * r) ** 2 / 8))
    if center:
        bo.assert_within("mean", mean, mu, 40 * bo.U32 * x.double().abs().mean(-1) + bo.U32)
    else:
        assert mean is None
    dx = g.empty((rows, N), DT[io])
    got = binding.layer_norm_backward(dy, x, rstd, mean=mean, weight=w, dx=dx)
    ref = bo.norm_backward(dy, x, mean, rstd, w, center)
    # two sums over a row (27 half steps of their terms, as above) and ten roundings
    bo.assert_within("dx", got["x"], ref[0], 80 * bo.U32 * ref[3] + bo.half_step(DT[io]) * ref[0].abs())
    # xh rounded twice, the sums of a thread's rows, of a block and of the blocks in fp32
    bo.assert_within("dweight", got["weight"], ref[1], 64 * bo.U32 * ref[4] + 1e-30)
    bo.assert_within("dbias", got["bias"], ref[2], 64 * bo.U32 * ref[5] + 1e-30)
    g.check()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 5, 100, 5000])
def test_rows(rows, io):
    from paper_2402_19427_b200 import binding
    for N in (128, 2560):
        x, w, b, dy = make(rows, N, io, seed=3)
        y, mean, rstd = binding.layer_norm(x, None, b, stats=True)
        yr, mu, r = bo.norm(x, None, b, 1e-5, True)
        bo.assert_within("y", y, yr, bo.norm_bound(x, None, b, mu, r, DT[io], yr))
        got = binding.layer_norm_backward(dy, x, rstd, mean=mean)
        ref = bo.norm_backward(dy, x, mean, rstd, None, True)
        bo.assert_within("dx", got["x"], ref[0], 80 * bo.U32 * ref[3] + bo.half_step(DT[io]) * ref[0].abs())
        # up to 5000 rows: 5000 / 592 rows a group, 32 groups a block, 592 blocks
        bo.assert_within("dweight", got["weight"], ref[1], 128 * bo.U32 * ref[4] + 1e-30)
        bo.assert_within("dbias", got["bias"], ref[2], 128 * bo.U32 * ref[5] + 1e-30)
        only = binding.layer_norm_backward(dy, x, rstd, mean=mean, param_grads=False)
        assert set(only) == {"x"} and torch.equal(only["x"], got["x"])
        again = binding.layer_norm_backward(dy, x, rstd, mean=mean)
        assert all(torch.equal(got[k], again[k]) for k in got)


def test_heads_of_a_batch_and_large_means():
    from paper_2402_19427_b200 import binding
    x, w, b, _ = make((2, 33, 5), 64, "bf16", shift=0.0)
    y = binding.layer_norm(x, w, center=False)
    assert torch.equal(y.view(-1, 64), binding.layer_norm(x.view(-1, 64), w, center=False))
    x, w, b, _ = make(9, 1024, "f32", shift=1000.0)   # deviations are taken from the mean, not out of a difference of squares
    yr, mu, r = bo.norm(x, w, b, 1e-5, True)
    bo.assert_within("y", binding.layer_norm(x, w, b), yr, bo.norm_bound(x, w, b, mu, r, torch.float32, yr))


@pytest.mark.parametrize("N", [64, 1531, 4096, 20001])
def test_a_row_that_is_no_number_touches_no_other(N):
    from paper_2402_19427_b200 import binding
    x, w, b, dy = make(50, N, "bf16")
    clean, mean, rstd = binding.layer_norm(x, w, b, stats=True)
    bad = x.clone(); bad[7, N // 2] = float("inf"); bad[23, 0] = float("nan"); bad[31] = 0
    y, m2, r2 = binding.layer_norm(bad, w, b, stats=True)
    keep = [i for i in range(50) if i not in (7, 23, 31)]
    assert torch.equal(y[keep], clean[keep]) and torch.equal(r2[keep], rstd[keep])
    assert torch.isnan(y[23]).all() and not torch.isfinite(y[7]).all()
    bo.assert_within("a row of zeros", y[31], b.double(), bo.half_step(torch.bfloat16) * b.double().abs())
    dx = binding.layer_norm_backward(dy, bad, r2, mean=m2, weight=w)["x"]
    assert torch.equal(dx[keep], binding.layer_norm_backward(dy, x, rstd, mean=mean, weight=w)["x"][keep])


def test_gradients_against_differences():
    from paper_2402_19427_b200 import binding
    x, w, b, dy = make(4, 96, "f32", seed=5)
    for center in (True, False):
        _, mean, rstd = binding.layer_norm(x, w, b, center=center, stats=True)
        got = binding.layer_norm_backward(dy, x, rstd, mean=mean, weight=w)
        loss = lambda x, w, b: float((bo.norm(x, w, b, 1e-5, center)[0] * dy.double()).sum())  # noqa: E731
        for name, t in (("x", x), ("weight", w), ("bias", b)):
            for i in (0, 17, t.numel() - 1):
                e = torch.zeros_like(t, dtype=torch.float64); e.view(-1)[i] = 1e-5
                args = dict(x=x.double(), w=w.double(), b=b.double()); key = dict(x="x", weight="w", bias="b")[name]
                hi = loss(**{**args, key: args[key] + e}); lo = loss(**{**args, key: args[key] - e})
                # the differences are off by h^2 (1e-10 of third derivatives) and 1e-16 / 1e-5 of the loss, the kernel by fp32 roundings
                assert abs((hi - lo) / 2e-5 - float(got[name].view(-1)[i])) <= 2e-5, (name, i)


def test_graph_replay_and_another_stream():
    from paper_2402_19427_b200 import binding
    x, w, b, dy = make(333, 2560, "bf16")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            y, mean, rstd = binding.layer_norm(x, w, b, stats=True); g = binding.layer_norm_backward(dy, x, rstd, mean=mean, weight=w)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, mean2, rstd2 = binding.layer_norm(x, w, b, stats=True); g2 = binding.layer_norm_backward(dy, x, rstd2, mean=mean2, weight=w)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(g[k], g2[k]) for k in g)
    x.copy_(x.flip(0)); dy.copy_(dy.flip(0))
    graph.replay(); torch.cuda.synchronize()
    assert torch.equal(y2, y.flip(0)) and torch.equal(g2["x"], g["x"].flip(0))
