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
