"""rglru_linear_attention_*: prefill, decode step and backward against the recurrence in fp64, token by token; lengths around the chunks'
borders, widths on and off the tiles, strided and time-major tensors, decays from none to total."""
import pytest
import torch

import block_oracle as bo
from util import Guarded

pytestmark = pytest.mark.gpu
DT = dict(bf16=torch.bfloat16, f32=torch.float32)


def make(B, T, H, dk, dv, io, seed=0, state=True, decay=None):
    g = torch.Generator(device="cuda").manual_seed(seed + B + 3 * T + 5 * H + 7 * dk + 11 * dv)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[io]
    ld = torch.log1p(-torch.exp2(-torch.linspace(1.0, 9.0, H, device="cuda", dtype=torch.float64))).float() if decay is None else torch.tensor(decay, device="cuda")
    return dict(q=rnd(B, T, H, dk).to(dt), k=rnd(B, T, H, dk).to(dt), v=rnd(B, T, H, dv).to(dt), do=rnd(B, T, H, dv).to(dt), ld=ld,
                s0=2 * rnd(B, H, dk, dv) if state else None, ds_T=rnd(B, H, dk, dv) if state else None)


def check_forward(t, o, s_T, scale):
    T, dt = t["q"].shape[1], t["q"].dtype
    orr, sr, om, sm = bo.attention(t["q"], t["k"], t["v"], t["ld"], t["s0"], scale)
    bo.assert_within("o", o, orr, bo.attention_bound(om, orr, dt, T))
    bo.assert_within("s_T", s_T, sr, bo.state_bound(sm, T))


def check_backward(t, got, scale):
    T, dt = t["q"].shape[1], t["q"].dtype
    ref, mag = bo.attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], t["s0"], t["ds_T"], scale)
    for n in "qkv":
        bo.assert_within("d" + n, got[n], ref[n], bo.attention_bound(mag[n], ref[n], dt, T))
    if "s0" in got:
        bo.assert_within("ds0", got["s0"], ref["s0"], bo.state_bound(mag["s0"], T))


SHAPES = [(1, 1, 1, 16, 16), (2, 1, 3, 128, 128), (1, 31, 2, 64, 64), (2, 33, 2, 64, 128), (1, 64, 1, 128, 64), (1, 127, 2, 128, 128), (2, 128, 2, 128, 128),
          (1, 129, 3, 128, 128), (3, 200, 2, 96, 96), (1, 257, 2, 80, 112), (1, 300, 2, 24, 40), (2, 700, 3, 128, 128), (1, 1500, 1, 128, 128), (1, 2050, 2, 64, 64)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,dk,dv", SHAPES)
def test_prefill_and_backward(B, T, H, dk, dv, io):
    from paper_2402_19427_b200 import binding
    for state in (True, False):
        t = make(B, T, H, dk, dv, io, state=state)
        g = Guarded()
        o, s_T = g.empty((B, T, H, dv), DT[io]), g.empty((B, H, dk, dv), torch.float32)
        binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"], o=o, s_T=s_T)
        check_forward(t, o, s_T, dk ** -0.5)
        dq, dk_, dv_ = g.empty((B, T, H, dk), DT[io]), g.empty((B, T, H, dk), DT[io]), g.empty((B, T, H, dv), DT[io])
        got = binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True, dq=dq, dk=dk_, dv=dv_)
        check_backward(t, got, dk ** -0.5)
        g.check()
        again = binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True)
        assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 70, 2, 33, 7), (2, 40, 1, 1, 1), (1, 150, 2, 200, 256), (1, 90, 1, 256, 136), (2, 65, 2, 12, 100)])
def test_other_widths(B, T, H, dk, dv, io):
    from paper_2402_19427_b200 import binding
    t = make(B, T, H, dk, dv, io)
    o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"], scale=0.7)
    check_forward(t, o, s_T, 0.7)
    got = binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], scale=0.7, state_grads=True)
    check_backward(t, got, 0.7)


def test_forced_generic():
    from paper_2402_19427_b200 import binding
    t = make(2, 150, 2, 64, 64, "bf16")
    o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"], flags=1)
    check_forward(t, o, s_T, 64 ** -0.5)
    check_backward(t, binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True, flags=1), 64 ** -0.5)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_decays_from_none_to_total(io):
    from paper_2402_19427_b200 import binding
    # no memory at all, almost none, a strong decay whose powers underflow, plain linear attention, a growing state
    t = make(1, 300, 6, 64, 64, io, decay=[float("-inf"), -200.0, -1.0, -1e-3, 0.0, 2e-3])
    o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"])
    check_forward(t, o, s_T, 64 ** -0.5)
    check_backward(t, binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True), 64 ** -0.5)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_parts_of_one_projection_and_time_major_batches(io):
    from paper_2402_19427_b200 import binding
    B, T, H, w = 2, 150, 3, 64
    t = make(B, T, H, w, w, io)
    o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"])
    g = binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True)
    qkv = torch.stack([t["q"], t["k"], t["v"]], 2)
    parts = [qkv[:, :, i] for i in range(3)]
    o2, s2 = binding.linear_attention_prefill(*parts, t["ld"], s0=t["s0"])
    assert torch.equal(o, o2) and torch.equal(s_T, s2)
    dqkv = torch.full_like(qkv, float("nan"))
    g2 = binding.linear_attention_backward(*parts, t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True, **{"d" + n: dqkv[:, :, i] for i, n in enumerate("qkv")})
    assert torch.equal(dqkv, torch.stack([g["q"], g["k"], g["v"]], 2)) and torch.equal(g["s0"], g2["s0"])
    major = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (t["q"], t["k"], t["v"])]
    out = torch.empty(T, B, H, w, dtype=DT[io], device="cuda").transpose(0, 1)
    o3, s3 = binding.linear_attention_prefill(*major, t["ld"], s0=t["s0"], o=out)
    assert torch.equal(o, o3) and torch.equal(s_T, s3)
    # distances that are no multiple of 16 bytes
    odd = torch.zeros(B, T, 3 * H * w + 1, dtype=DT[io], device="cuda")
    views = [odd[:, :, i * H * w:(i + 1) * H * w].unflatten(-1, (H, w)) for i in range(3)]
    for dst, src in zip(views, (t["q"], t["k"], t["v"])):
        dst.copy_(src)
    o4, s4 = binding.linear_attention_prefill(*views, t["ld"], s0=t["s0"])
    check_forward(t, o4, s4, w ** -0.5)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 8, 8), (1, 16, 128, 128), (3, 5, 96, 80), (2, 3, 33, 7), (64, 20, 128, 128), (2, 2, 300, 260), (700, 2, 16, 64)])
def test_decode_steps(B, H, dk, dv, io):
    from paper_2402_19427_b200 import binding
    steps = 3
    t = make(B, steps, H, dk, dv, io)
    g = Guarded()
    s, o = g.empty((B, H, dk, dv), torch.float32), g.empty((B, H, dv), DT[io])
    s.copy_(t["s0"])
    outs = []
    for i in range(steps):
        q, k, v = (t[n][:, i].contiguous() for n in "qkv")
        assert binding.linear_attention_decode_step(q, k, v, t["ld"], s, o=o).data_ptr() == o.data_ptr()
        outs.append(o.clone())
    g.check()
    orr, sr, om, sm = bo.attention(t["q"], t["k"], t["v"], t["ld"], t["s0"], dk ** -0.5)
    # fp32 sums over dk rows, three roundings of the state a step, one of the result
    bo.assert_within("o", torch.stack(outs, 1), orr, (dk + 32) * bo.U32 * om + bo.half_step(DT[io]) * orr.abs())
    bo.assert_within("s", s, sr, 4 * steps * bo.U32 * sm)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_prefill_continues_and_decode_follows(io):
    from paper_2402_19427_b200 import binding
    t = make(2, 300, 2, 128, 128, io)
    cut = lambda a, b: (t[n][:, a:b].contiguous() for n in "qkv")  # noqa: E731
    o1, s = binding.linear_attention_prefill(*cut(0, 170), t["ld"], s0=t["s0"])
    o2, s_in_place = binding.linear_attention_prefill(*cut(170, 297), t["ld"], s0=s, s_T=s)
    assert s_in_place.data_ptr() == s.data_ptr()
    outs = [o1, o2]
    for i in range(297, 300):
        outs.append(binding.linear_attention_decode_step(*(t[n][:, i].contiguous() for n in "qkv"), t["ld"], s)[:, None])
    check_forward(t, torch.cat(outs, 1), s, 128 ** -0.5)
    # gradients of two segments chain through the carried state
    o1, s1 = binding.linear_attention_prefill(*cut(0, 170), t["ld"], s0=t["s0"])
    late = binding.linear_attention_backward(*cut(170, 300), t["ld"], t["do"][:, 170:].contiguous(), s0=s1, ds_T=t["ds_T"], state_grads=True)
    early = binding.linear_attention_backward(*cut(0, 170), t["ld"], t["do"][:, :170].contiguous(), s0=t["s0"], ds_T=late["s0"], state_grads=True)
    check_backward(t, dict({n: torch.cat([early[n], late[n]], 1) for n in "qkv"}, s0=early["s0"]), 128 ** -0.5)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_later_tokens_that_are_no_numbers_touch_no_earlier_one(bad, io):
    from paper_2402_19427_b200 import binding
    t = make(2, 200, 2, 128, 128, io)
    o, _ = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"])
    for name in "qkv":
        x = {n: t[n].clone() for n in "qkv"}
        x[name][0, 77, 1, 3] = bad
        got, _ = binding.linear_attention_prefill(x["q"], x["k"], x["v"], t["ld"], s0=t["s0"])
        assert torch.equal(got[0, :77], o[0, :77]) and torch.equal(got[1], o[1]) and torch.equal(got[0, :, 0], o[0, :, 0]), name
        assert not torch.isfinite(got[0, 77, 1]).all(), name
        if name == "q":
            assert torch.equal(got[0, 78:], o[0, 78:])


def test_gradients_against_differences():
    from paper_2402_19427_b200 import binding
    t = make(1, 12, 2, 6, 5, "f32")
    got = binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True)

    def loss(**a):
        o, s, _, _ = bo.attention(a["q"], a["k"], a["v"], t["ld"], a["s0"], 6 ** -0.5)
        return float((o * t["do"].double()).sum() + (s * t["ds_T"].double()).sum())
    args = {n: t[n].double() for n in ("q", "k", "v", "s0")}
    for name in args:
        for i in (0, 13, t[name].numel() - 1):
            e = torch.zeros_like(args[name]); e.view(-1)[i] = 1e-4
            diff = (loss(**{**args, name: args[name] + e}) - loss(**{**args, name: args[name] - e})) / 2e-4
            # the loss is linear in each: the differences are off by 1e-16 / 1e-4 of it, the kernel by fp32 roundings of sums below 100
            assert abs(diff - float(got[name].view(-1)[i])) <= 2e-4, (name, i)


def test_graph_replay_and_two_streams():
    from paper_2402_19427_b200 import binding
    t = make(1, 1100, 2, 128, 128, "bf16")
    call = lambda: (*binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"]),  # noqa: E731
                    *binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True).values())
    ref = call()
    side, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s in side:
            with torch.cuda.stream(s):
                got.append(call())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got.append(call())
    graph.replay(); graph.replay(); torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, ref))


@pytest.mark.parametrize("io,B,T,H,dk,dv", [("f32", 1, 1100, 2, 64, 128), ("f32", 2, 700, 3, 33, 200), ("bf16", 1, 19300, 2, 128, 128), ("bf16", 1, 900, 1, 136, 256)])
def test_cut_sequences_whose_state_is_updated_in_place(io, B, T, H, dk, dv):
    """Sequences long enough to be shared by several blocks, all of which start from s0: it may be where s_T goes"""
    from paper_2402_19427_b200 import binding
    t = make(B, T, H, dk, dv, io)
    o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"])
    s = t["s0"].clone()
    o2, _ = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=s, s_T=s)
    assert torch.equal(o, o2) and torch.equal(s, s_T)
    # the last tokens, and the state, against the walk over those tokens alone from the state before them
    cut = T - 150
    _, before = binding.linear_attention_prefill(*(t[n][:, :cut].contiguous() for n in "qkv"), t["ld"], s0=t["s0"])
    tail = dict(t, **{n: t[n][:, cut:].contiguous() for n in "qkv"}, s0=before)
    orr, sr, om, sm = bo.attention(tail["q"], tail["k"], tail["v"], t["ld"], before, dk ** -0.5)
    # both states have come by their own cuts: each is off by fp32 sums of what lies in it, a few half steps of its magnitude a chunk
    off = 2 * bo.state_bound(sm, T)
    bo.assert_within("s_T", s_T, sr, off)
    bo.assert_within("o", o[:, cut:], orr, 2 * bo.attention_bound(om, orr, DT[io], T) + bo.U32 * (512 + T / 8) * om)


@pytest.mark.parametrize("B,T,H,dk,dv", [(8, 2000, 20, 64, 32), (3, 1400, 99, 24, 64)])
def test_more_heads_than_fit_at_once(B, T, H, dk, dv):
    """Whole sequences for every block and a stretch of those left over, forward and backward"""
    from paper_2402_19427_b200 import binding
    t = make(B, T, H, dk, dv, "bf16")
    o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"])
    check_forward(t, o, s_T, dk ** -0.5)
    got = binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True)
    check_backward(t, got, dk ** -0.5)
    s = t["s0"].clone()
    o2, _ = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=s, s_T=s)
    assert torch.equal(o, o2) and torch.equal(s, s_T)
