"""The block operators where their arithmetic or their bookkeeping could go wrong and the other tests' bounds would not show it."""
import pytest
import torch

import block_oracle as bo

pytestmark = pytest.mark.gpu
DT = dict(bf16=torch.bfloat16, f32=torch.float32)


def test_a_recorded_timeout_survives_calls_that_share_the_workspace():
    """The first word of a workspace is the status of all calls in it until it is queried: no operator puts anything else there"""
    from paper_2402_19427_b200 import binding
    timeout = 0x52474C00 | binding.ERR_TIMEOUT   # as a kernel records it
    x = torch.randn(40, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(64, 64, device="cuda", dtype=torch.bfloat16)
    _, mean, rstd = binding.layer_norm(x, stats=True)
    q = x.view(1, 40, 1, 64)
    ld = torch.zeros(1, device="cuda")
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    for name, call in dict(norm=lambda: binding.layer_norm_backward(x, x, rstd, mean=mean, workspace=ws),
                           linear=lambda: binding.linear(x, w, workspace=ws), few=lambda: binding.linear(x[:1], w, workspace=ws),
                           linear_backward=lambda: binding.linear_backward(x, x, w, preact=x, activation="gelu", workspace=ws),
                           mix=lambda: binding.linear_attention_prefill(q, q, q, ld, workspace=ws),
                           mix_backward=lambda: binding.linear_attention_backward(q, q, q, ld, q, workspace=ws)).items():
        ws.zero_()
        ws[:4].view(torch.int32).fill_(timeout)
        call()
        assert binding.query_status(ws) == binding.ERR_TIMEOUT, name
        call()
        assert binding.query_status(ws) == binding.OK, name


@pytest.mark.parametrize("product", ["forward", "dweight"])
def test_sums_over_many_terms_are_as_exact_as_fp32(product):
    """All terms of one sign, half a million of them: an accumulator that adds up by cutting off must not take them all."""
    from paper_2402_19427_b200 import binding
    terms, rows, cols = 1 << 19, 2560, 2048   # 80 tiles of 256 x 256: most of them are one CTA pair's, with all of their terms
    g = torch.Generator(device="cuda").manual_seed(5)
    a = (0.5 + torch.rand(terms, rows, generator=g, device="cuda", dtype=torch.bfloat16)) * (1 + torch.rand(rows, generator=g, device="cuda")).bfloat16()
    b = 0.5 + torch.rand(terms, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    if product == "dweight":
        got = binding.linear_backward(a, b, torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16), need=("weight",))["weight"]
    else:
        got = binding.linear(a.T.contiguous(), b.T.contiguous())
    for m in (0, 1024, rows - 64):
        ref = a[:, m:m + 64].double().T @ b[:, :64].double()
        # 16384 terms an accumulator, 16 an instruction, each of which cuts off less than two steps of the sum (2^-23 relative); the
        # accumulators' sum takes 32 roundings.  Then one rounding to bf16: half a step of the result's own binade
        half = torch.exp2(torch.floor(torch.log2(ref)) - 8)
        bo.assert_within(product, got[m:m + 64, :64], ref, half + (2 * 1024 * 2 + 32) * bo.U32 * ref)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 4, 5, 12, 264, 2565])
def test_norm_of_large_means_and_widths_that_leave_threads_idle(N, io):
    """Rows of one large value, (0 - mean) r beyond fp32's range: what lies behind a row's end takes no part"""
    from paper_2402_19427_b200 import binding
    x = torch.full((9, N), 2.0 ** 122, device="cuda", dtype=DT[io])
    g = torch.Generator(device="cuda").manual_seed(N)
    dy, w = torch.randn(9, N, generator=g, device="cuda").to(DT[io]), 1 + 0.1 * torch.randn(N, generator=g, device="cuda")
    mean, rstd = torch.full((9,), 2.0 ** 122, device="cuda"), torch.full((9,), 300.0, device="cuda")
    got = binding.layer_norm_backward(dy, x, rstd, mean=mean, weight=w)
    ref = bo.norm_backward(dy, x, mean, rstd, w, True)
    bo.assert_within("dx", got["x"], ref[0], 80 * bo.U32 * ref[3] + bo.half_step(DT[io]) * ref[0].abs())
    assert (got["weight"] == 0).all()
    bo.assert_within("dbias", got["bias"], ref[2], 64 * bo.U32 * ref[5])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [5, 8, 33])
def test_an_infinite_value_of_v_is_infinite_in_later_outputs(dk, io):
    """Widths that no tensor-core kernel takes: an infinity in v is one in its column from its token on, also where dk is no multiple of four"""
    from paper_2402_19427_b200 import binding
    T, dv, at, col = 150, 6, 3, 2
    g = torch.Generator(device="cuda").manual_seed(dk)
    q, k, v = ((0.5 + torch.rand(1, T, 2, w, generator=g, device="cuda")).to(DT[io]) for w in (dk, dk, dv))
    ld = torch.tensor([-0.01, -0.1], device="cuda")
    clean, s = binding.linear_attention_prefill(q, k, v, ld)
    v = v.clone(); v[0, at, 1, col] = float("inf")
    o, sT = binding.linear_attention_prefill(q, k, v, ld)
    assert torch.isposinf(o[0, at:, 1, col]).all() and torch.isposinf(sT[0, 1, :, col]).all()
    o[0, at:, 1, col] = clean[0, at:, 1, col]
    sT[0, 1, :, col] = s[0, 1, :, col]
    assert torch.equal(o, clean) and torch.equal(sT, s)
