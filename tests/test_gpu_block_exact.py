"""The block operators on small whole numbers, whose sums every kernel has to give exactly: a token, a border row or a stretch that were dropped, taken
twice or put in another's place would show at any length, where bounds on rounding grow with it."""
import pytest
import torch

import block_oracle as bo
from test_gpu_linear import SIZES
from test_gpu_linear_attention import SHAPES

pytestmark = pytest.mark.gpu
DT = dict(bf16=torch.bfloat16, f32=torch.float32)


def whole(g, *shape):
    """-1 and 1, an eighth of the values each, and 0.  A sum of n products of two has a variance of n / 16: for up to 20000 of them (35 squared) all entries of a matrix
    stay below 256 (seven times that), so that bf16 holds them exactly.  Larger results are rounded once, from the exact sum."""
    r = torch.randint(0, 8, shape, generator=g, device="cuda", dtype=torch.int8)
    return (r == 0).float() - (r == 1).float()


def rounded(t, dt):
    return t.float().to(dt)   # whole numbers below 2^24: exact in fp32


# besides: more terms than one accumulator takes, in tiles that are a CTA pair's alone
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SIZES + [(1, 1, 1), (5, 3, 7), (70, 65, 33), (130, 257, 129), (300, 1001, 77), (9, 4095, 11), (4097, 130, 260), (17001, 2312, 2304), (256, 17000, 264)])
def test_projection(M, K, N, io):
    from paper_2402_19427_b200 import binding
    dt = DT[io]
    g = torch.Generator(device="cuda").manual_seed(M + 3 * K + 5 * N)
    x, w, dy, bias, res = whole(g, M, K).to(dt), whole(g, N, K).to(dt), whole(g, M, N).to(dt), whole(g, N), whole(g, M, N).to(dt)
    xd, wd, dyd = x.double(), w.double(), dy.double()
    y = xd @ wd.T + bias.double()
    got, pre = binding.linear(x, w, bias, residual=res, keep_preact=True)
    assert torch.equal(pre, rounded(y, dt)) and torch.equal(got, rounded(y + res.double(), dt))
    grads = binding.linear_backward(dy, x, w)
    assert torch.equal(grads["x"], rounded(dyd @ wd, dt)), "dx"
    assert torch.equal(grads["weight"], rounded(dyd.T @ xd, dt)), "dweight"
    assert torch.equal(grads["bias"], dyd.sum(0).float()), "dbias"


# besides: one sequence over all SMs; whole sequences for every block and stretches of those left over
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,dk,dv", SHAPES + [(1, 150, 2, 33, 7), (1, 19300, 2, 128, 128), (8, 2000, 20, 64, 32), (3, 1400, 99, 24, 64), (1, 1000, 2, 200, 136)])
def test_linear_attention(B, T, H, dk, dv, io):
    """Without decay, and (every third head) without memory"""
    from paper_2402_19427_b200 import binding
    dt = DT[io]
    g = torch.Generator(device="cuda").manual_seed(B + 3 * T + 5 * H + 7 * dk + 11 * dv)
    q, k, v, do = (whole(g, B, T, H, w).to(dt) for w in (dk, dk, dv, dv))
    s0, ds_T = whole(g, B, H, dk, dv), whole(g, B, H, dk, dv)
    ld = torch.zeros(H, device="cuda"); ld[2::3] = float("-inf")
    o, s_T, _, _ = bo.attention(q, k, v, ld, s0, 1.0)
    got, got_s = binding.linear_attention_prefill(q, k, v, ld, s0=s0, scale=1.0)
    assert float(s_T.abs().max()) <= 256
    assert torch.equal(got_s, s_T.float()) and torch.equal(got, rounded(o, dt))
    ref, _ = bo.attention_backward(q, k, v, ld, do, s0, ds_T, 1.0)
    grads = binding.linear_attention_backward(q, k, v, ld, do, s0=s0, ds_T=ds_T, scale=1.0, state_grads=True)
    for n in "qkv":
        assert torch.equal(grads[n], rounded(ref[n], dt)), n
    assert torch.equal(grads["s0"], ref["s0"].float())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("rows,N", [(1, 64), (301, 128), (5000, 128), (5000, 2560), (700, 1531), (60000, 72), (2500, 16392)])
def test_norm_gradients_of_weight_and_bias(rows, N, io):
    """mean 0 and rstd 1 as given: the deviations are x itself"""
    from paper_2402_19427_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(rows + N)
    x, dy = whole(g, rows, N).to(DT[io]), whole(g, rows, N).to(DT[io])
    for center in (True, False):
        got = binding.layer_norm_backward(dy, x, torch.ones(rows, device="cuda"), mean=torch.zeros(rows, device="cuda") if center else None)
        assert torch.equal(got["weight"], (dy.double() * x.double()).sum(0).float()) and torch.equal(got["bias"], dy.double().sum(0).float())
