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


@pytest.mark.parametrize("which", ["linear", "linear_split", "linear_few", "linear_f32", "linear_long", "linear_backward", "mix", "mix_cut", "mix_many", "mix_backward"])
def test_waits_that_run_out_are_reported_and_the_next_call_is_clean(which):
    """One operand's copies are held back, so that the products wait for them; the limit is a millisecond: the kernels give up, drain and return, the status
    says so, once, and the next call in the same workspace gives what it gave before."""
    from paper_2402_19427_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    ws = torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")
    if which.startswith("linear"):
        M, K, N = dict(linear=(2000, 320, 1100), linear_split=(300, 2560, 512), linear_few=(20, 512, 2560), linear_f32=(500, 512, 512), linear_long=(2304, 17000, 2304)).get(which, (700, 512, 640))
        x, w, dy = rnd(M, K), rnd(N, K), rnd(M, N)
        if which == "linear_f32":
            x, w, dy = x.float(), w.float(), dy.float()
        if which == "linear_backward":
            call = lambda flags: list(binding.linear_backward(dy, x, w, preact=dy, activation="gelu", flags=flags, workspace=ws).values())  # noqa: E731
        else:
            call = lambda flags: [binding.linear(x, w, activation="gelu", residual=dy, flags=flags, workspace=ws)]  # noqa: E731
    else:
        B, T, H = dict(mix=(1, 300, 4), mix_cut=(1, 9000, 2), mix_many=(8, 2000, 20)).get(which, (1, 2100, 3))
        q, k, v, do = (rnd(B, T, H, 64) for _ in range(4))
        ld = torch.full((H,), -0.01, device="cuda")
        if which == "mix_backward":
            call = lambda flags: list(binding.linear_attention_backward(q, k, v, ld, do, state_grads=True, flags=flags, workspace=ws).values())  # noqa: E731
        else:
            call = lambda flags: list(binding.linear_attention_prefill(q, k, v, ld, flags=flags, workspace=ws))  # noqa: E731
    want = call(0)
    torch.cuda.synchronize()
    assert binding.query_status(ws) == binding.OK
    prev = binding.set_wait_limit_ns(1_000_000)
    try:
        call(binding.FLAG_TEST_CARRY_NEVER_ARRIVES)
        torch.cuda.synchronize()
        assert binding.query_status(ws) == binding.ERR_TIMEOUT
        assert binding.query_status(ws) == binding.OK
    finally:
        binding.set_wait_limit_ns(prev)
    assert all(torch.equal(a, b) for a, b in zip(call(0), want))
    torch.cuda.synchronize()
    assert binding.query_status(ws) == binding.OK


@pytest.mark.parametrize("io,T", [("bf16", 9000), ("f32", 1100)])
def test_a_captured_prompt_of_a_cut_sequence_updates_its_state_in_place(io, T):
    """The copy of s0 that such a call makes for its blocks is captured with it, and made again on every replay"""
    from paper_2402_19427_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k, v = (torch.randn(1, T, 2, 64, generator=g, device="cuda").to(DT[io]) for _ in range(3))
    ld, s0 = torch.tensor([-0.001, -0.0001], device="cuda"), torch.randn(1, 2, 64, 64, generator=g, device="cuda")
    o1, s1 = binding.linear_attention_prefill(q, k, v, ld, s0=s0)
    o2, s2 = binding.linear_attention_prefill(q, k, v, ld, s0=s1)
    s = s0.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, _ = binding.linear_attention_prefill(q, k, v, ld, s0=s, s_T=s)
    for want_o, want_s in ((o1, s1), (o2, s2)):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want_o) and torch.equal(s, want_s)


@pytest.mark.parametrize("dk,dv", [(8, 8), (8, 128), (128, 8), (72, 8), (16, 120)])
def test_the_narrowest_heads_of_the_tensor_core_walk(dk, dv):
    from paper_2402_19427_b200 import binding
    from test_gpu_linear_attention import check_backward, check_forward, make
    for B, T, H in ((1, 1, 3), (2, 200, 3)):
        t = make(B, T, H, dk, dv, "bf16")
        o, s_T = binding.linear_attention_prefill(t["q"], t["k"], t["v"], t["ld"], s0=t["s0"])
        check_forward(t, o, s_T, dk ** -0.5)
        check_backward(t, binding.linear_attention_backward(t["q"], t["k"], t["v"], t["ld"], t["do"], s0=t["s0"], ds_T=t["ds_T"], state_grads=True), dk ** -0.5)


def test_two_host_threads_call_at_once():
    """Each with its stream; attributes of kernels and plans of a device are set up by whoever comes first"""
    import threading
    from paper_2402_19427_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn(300, 264, generator=g, device="cuda").bfloat16(), torch.randn(520, 264, generator=g, device="cuda").bfloat16()
    q = x.view(1, 300, 3, 88)
    ld = torch.full((3,), -0.01, device="cuda")

    def work():
        y, pre = binding.linear(x, w, activation="gelu", keep_preact=True)
        grads = binding.linear_backward(y, x, w, preact=pre, activation="gelu")
        n, mean, rstd = binding.layer_norm(y, stats=True)
        return [y, *grads.values(), n, binding.layer_norm_backward(y, n, rstd, mean=mean)["weight"], *binding.linear_attention_prefill(q, q, q, ld),
                *binding.linear_attention_backward(q, q, q, ld, q, state_grads=True).values()]

    want, got, errors = work(), [[], []], []
    torch.cuda.synchronize()

    def run(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i].append(work())
                torch.cuda.current_stream().synchronize()
        except Exception as e:   # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert all(torch.equal(a, b) for runs in got for r in runs for a, b in zip(r, want))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H", [(1, 300, 3), (1, 19300, 3), (60, 1400, 3)])
def test_growing_states_and_tokens_of_zeros(B, T, H, io):
    """Powers of a decay above one that leave fp32's range take nothing from a state that is 0: sequences that are zeros but for their last tokens (forward) or
    their first (backward) give what those tokens give alone"""
    from paper_2402_19427_b200 import binding
    from test_gpu_linear_attention import check_backward, check_forward, make
    n, w = 90, 64
    ld = [0.01, 0.3, 0.6][:H]
    part = make(B, n, H, w, w, io, state=False, decay=ld)
    zero = torch.zeros(B, T - n, H, w, dtype=DT[io], device="cuda")
    late = {x: torch.cat([zero, part[x]], 1) for x in "qkv"}
    o, s_T = binding.linear_attention_prefill(*(late[x] for x in "qkv"), part["ld"])
    assert (o[:, :T - n] == 0).all()
    check_forward(part, o[:, T - n:], s_T, w ** -0.5)
    early = {x: torch.cat([part[x], zero], 1) for x in ("q", "k", "v", "do")}
    got = binding.linear_attention_backward(early["q"], early["k"], early["v"], part["ld"], early["do"], state_grads=True)
    for x in "kv":
        assert (got[x][:, n:] == 0).all(), x
    check_backward(part, {x: got[x][:, :n] if x != "s0" else got[x] for x in got}, w ** -0.5)


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_activations_to_bf16_are_good_to_their_last_place(kind):
    """As far into the negative tail as bf16's normal numbers go: half a step of the result's own binade, and a tenth of that"""
    from paper_2402_19427_b200 import binding
    z = torch.cat([torch.linspace(-12.8, 12.8, 1 << 16, device="cuda"), torch.linspace(-1, 1, 1 << 12, device="cuda")]).bfloat16().unique()
    one = torch.ones(1, 1, device="cuda", dtype=torch.bfloat16)
    zd = z.double()
    ref = zd * (0.5 * torch.special.erfc(-zd * 0.5 ** 0.5) if kind == "gelu" else torch.sigmoid(zd))
    half = torch.exp2(torch.floor(torch.log2(ref.abs().clamp_min(2.0 ** -126))) - 8)
    # Phi is good to 2e-7 and, relative to itself, to 1e-4; the exponential's and the reciprocal's arguments are rounded in fp32 (up to 122 half steps); both below 0.1
    # of half a step, which is at least 2^-9 of the result
    for rows in (z.numel(), 5):   # products on the tensor cores; few rows
        x = z[:rows, None].contiguous() if rows > 5 else z[::max(1, z.numel() // 5)][:5, None].contiguous()
        i = torch.arange(z.numel(), device="cuda") if rows > 5 else torch.arange(z.numel(), device="cuda")[::max(1, z.numel() // 5)][:5]
        y = binding.linear(x, one, activation=kind)[:, 0]
        bo.assert_within(kind, y, ref[i], 1.1 * half[i])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_tensors_of_more_than_2_31_elements(io):
    """The last rows and tokens of each operator are those of a call on them alone"""
    from paper_2402_19427_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(9)
    rows, N, n = (1 << 31) // 1024 + 77, 1024, 5   # 2.1 10^9 elements and some
    x = torch.empty(rows, N, device="cuda", dtype=DT[io])
    x.fill_(0.25)
    x[-200:] = torch.randn(200, N, generator=g, device="cuda").to(DT[io])
    tail = x[-200:].clone()
    y, mean, rstd = binding.layer_norm(x, stats=True)
    assert torch.equal(y[-200:], binding.layer_norm(tail))
    dx = binding.layer_norm_backward(y, x, rstd, mean=mean)["x"]
    assert torch.equal(dx[-200:], binding.layer_norm_backward(y[-200:].clone(), tail, rstd[-200:].clone(), mean=mean[-200:].clone())["x"])
    del y, dx
    w = torch.randn(N, N, generator=g, device="cuda").to(DT[io])
    y = binding.linear(x, w, residual=x)
    ref, z, mag = bo.linear(tail, w, None, "none", tail)
    bound = (2 * N + 4) * bo.U32 * mag + 16 * bo.U32 * (z.abs() + tail.double().abs()) + bo.half_step(DT[io]) * ref.abs()
    bo.assert_within("y", y[-200:], ref, bound)
    del y
    got = binding.linear_backward(x, x, w, need=("x", "bias"))
    dxr = tail.double() @ w.double()
    bo.assert_within("dx", got["x"][-200:], dxr, 2 * N * bo.U32 * (tail.double().abs() @ w.double().abs()) + bo.half_step(DT[io]) * dxr.abs())
    del got
    # one sequence of 8 heads of 128: a decay that has forgotten all but the last 300 tokens (exp(-150) of what was before)
    q = x.view(1, rows, 8, 128)
    ld = torch.full((8,), -0.5, device="cuda")
    o, s = binding.linear_attention_prefill(q, q, q, ld)
    t = x[-300:].clone().view(1, 300, 8, 128)
    orr, sr, om, sm = bo.attention(t, t, t, ld, None, 128 ** -0.5)
    bo.assert_within("o", o[:, -n:], orr[:, -n:], bo.attention_bound(om[:, -n:], orr[:, -n:], DT[io], 300))
    bo.assert_within("s_T", s, sr, bo.state_bound(sm, 300))
    assert torch.isfinite(o[:, ::100003].float()).all()
    del o
    grads = binding.linear_attention_backward(q, q, q, ld, q)
    ref, mag = bo.attention_backward(t, t, t, ld, t, None, None, 128 ** -0.5)
    for name in "qkv":
        bo.assert_within("d" + name, grads[name][:, -n:], ref[name][:, -n:], bo.attention_bound(mag[name][:, -n:], ref[name][:, -n:], DT[io], 300))
