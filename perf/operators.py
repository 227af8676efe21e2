"""The operators that stand around the temporal core, as cases that can be timed and compared.

A case is one pass through one of

* ``norm`` / ``norm_backward`` / ``norm_step`` -- the normalisation in front of a block (``center``: layer norm, else the root mean
  square alone) or of each head behind a mixer, its gradients, and one after the other;
* ``linear`` / ``linear_backward`` -- a projection of the block with bias, activation and skip connection in its epilogue, and its gradients;
* ``mix`` / ``mix_step`` / ``mix_backward`` -- linear attention with a decay for each head: whole sequences, one token for each of B
  sequences with the state updated in place, and the gradients.

With ``own`` false ``run`` is their plain form, elementary operations in fp32; with ``own`` true it calls
``paper_2402_19427_b200.binding``.  ``exact`` is their definition in fp64.

Widths and head counts are those of ``inputs.CONFIGS``, ``bench.py`` and the tests: 2560 (10, 16 or 20 heads), 4096 (16 or 32), 1536 and 2048
(16), 1024 (8).  Sequence lengths likewise: 2048 for training, 4096 for the backward, 65536 for long documents, 197 for a prompt.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = [(8, 128), (16, 128), (20, 128), (32, 128), (16, 96), (32, 64), (10, 64)]   # (heads, head width) of bf16 layers
MOST_ELEMENTS = 1 << 26
DEVICE = "cuda"


def _norm(op, rows, N, io="bf16", center=True, bias=True):
    return dict(op=op, rows=rows, N=N, io=io, center=center, bias=bias)


def _linear(op, M, K, N, io="bf16", act="none", bias=True, residual=False):
    return dict(op=op, M=M, K=K, N=N, io=io, act=act, bias=bias, residual=residual)


def _mix(op, B, T, H, dk, dv, io="bf16", state=False, fused=False):
    return dict(op=op, B=B, T=T, H=H, dk=dk, dv=dv, io=io, state=state, fused=fused)


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # the norm in front of a block for one user's next token: latency
        named("norm_token", _norm("norm", 1, 2560)),
        # the norm of every head behind the mixer, training batch (8 x 2048 tokens, 20 heads)
        named("norm_heads", _norm("norm", 8 * 2048 * 20, 128, center=False, bias=False)),
        # gradients of the norm in front of a block, training batch of 4 x 4096 tokens
        named("norm_backward", _norm("norm_backward", 4 * 4096, 4096)),
        # forward and backward of a small exact run, an odd width and a ragged number of rows
        named("norm_f32_step", _norm("norm_step", 1213, 1531, io="f32")),
        # output projection of one user's next token, added to the residual stream: reads the weights once
        named("linear_token", _linear("linear", 1, 2560, 2560, residual=True)),
        # the branch with the GeLU, training batch; its input to the activation is kept for the backward
        named("linear_train", _linear("linear", 8 * 2048, 2560, 2560, act="gelu")),
        # gradients of the same
        named("linear_backward", _linear("linear_backward", 8 * 2048, 2560, 2560, act="gelu")),
        # one token for each sequence of a full serving batch
        named("mix_step", _mix("mix_step", 64, 1, 20, 128, 128)),
        # one user's prompt, q, k and v side by side as one projection leaves them
        named("mix_prompt", _mix("mix", 1, 197, 20, 128, 128, fused=True)),
        # training batch
        named("mix_train", _mix("mix", 8, 2048, 20, 128, 128)),
        # one long document that continues a carried state
        named("mix_long", _mix("mix", 1, 65536, 16, 128, 128, state=True)),
        # gradients of a training batch
        named("mix_backward", _mix("mix_backward", 4, 4096, 16, 128, 128)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "linear", "linear", "mix", "mix", "mix"])
    io = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "norm":
        op = rng.choice(["norm", "norm_backward", "norm_step"])
        N = rng.choice([64, 96, 128, 160, 256, 1024, 1536, 2048, 2560, 4096, 5632]) if rng.random() < 0.6 else _log_int(rng, 33, 8191)
        most = max(1, MOST_ELEMENTS // (2 if op == "norm_step" else 1) // N)
        return _norm(op, _log_int(rng, 1, min(most, 8 * 2048 * 20)), N, io, rng.random() < 0.6, rng.random() < 0.6)
    if kind == "linear":
        op = rng.choice(["linear", "linear", "linear_backward"])
        if rng.random() < 0.75:
            K, N = (rng.choice([512, 1024, 1536, 2048, 2560, 4096]) for _ in range(2))
        else:
            K, N = (_log_int(rng, 65, 2047) for _ in range(2))
        most = 8 * 2048 * 2560 * 2560 // (K * N * (8 if io == "f32" else 2 if op == "linear_backward" else 1))
        return _linear(op, _log_int(rng, 1, max(1, min(most, 8 * 2048))), K, N, io, rng.choice(["none", "gelu", "silu"]), rng.random() < 0.7,
                       op == "linear" and rng.random() < 0.4)
    op = rng.choice(["mix", "mix", "mix_backward", "mix_step"])
    if io == "f32":
        H, dk, dv = rng.choice([2, 4, 8]), _log_int(rng, 16, 128), _log_int(rng, 16, 128)
    elif rng.random() < 0.7:
        H, dk = rng.choice(HEADS)
        dv = dk
    else:
        H, dk, dv = rng.choice([4, 8, 16]), 8 * rng.randint(4, 16), 8 * rng.randint(4, 16)
    fused = op == "mix" and dk == dv and dk % 8 == 0 and rng.random() < 0.4
    if op == "mix_step":
        return _mix(op, _log_int(rng, 1, max(1, 64 * 20 * 128 * 128 // (H * dk * dv))), 1, H, dk, dv, io)
    tokens = MOST_ELEMENTS // 2 // (H * max(dk, dv)) // (16 if io == "f32" else 2 if op == "mix_backward" else 1)
    T = _log_int(rng, 1, min(tokens, 65536))
    return _mix(op, _log_int(rng, 1, max(1, min(16, tokens // T))), T, H, dk, dv, io, rng.random() < 0.5, fused)


def _dtype(case):
    return torch.bfloat16 if case["io"] == "bf16" else torch.float32


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    dt = _dtype(case)

    def normal(*shape, dtype=dt, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device=DEVICE) * scale + shift).to(dtype)

    s, op, f32 = dict(case=dict(case)), case["op"], torch.float32
    if op.startswith("norm"):
        rows, N = case["rows"], case["N"]
        s["x"] = normal(rows, N, scale=1.5, shift=0.25)
        s["weight"] = normal(N, dtype=f32, scale=0.2, shift=1.0)
        s["bias"] = normal(N, dtype=f32, scale=0.2) if case["bias"] else None
        if op != "norm":
            s["dy"] = normal(rows, N)
        if op == "norm_backward":   # what the forward left: the mean and the reciprocal deviation of every row
            xd = s["x"].float()
            mean = xd.mean(-1) if case["center"] else torch.zeros(rows, device=DEVICE)
            s["mean"] = mean if case["center"] else None
            s["rstd"] = torch.rsqrt((xd - mean[:, None]).square().mean(-1) + 1e-5)
    elif op.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = normal(M, K)
        s["weight"] = normal(N, K, scale=K ** -0.5)
        s["bias"] = normal(N, dtype=f32, scale=0.3) if case["bias"] else None
        s["residual"] = normal(M, N) if case["residual"] else None
        if op == "linear_backward":
            s["dy"] = normal(M, N)
            s["preact"] = normal(M, N) if case["act"] != "none" else None
    else:
        B, T, H, dk, dv = (case[k] for k in ("B", "T", "H", "dk", "dv"))
        tok = (B, H) if op == "mix_step" else (B, T, H)
        if case["fused"]:
            qkv = normal(B, T, 3, H, dk)
            s["q"], s["k"], s["v"] = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        else:
            s["q"], s["k"], s["v"] = normal(*tok, dk), normal(*tok, dk), normal(*tok, dv)
        # a memory of 32 tokens for the first head up to 4096 for the last
        s["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(5.0, 12.0, H, device=DEVICE, dtype=torch.float64))).float()
        state = op == "mix_step" or case["state"]
        s["s0"] = normal(B, H, dk, dv, dtype=f32, scale=4.0) if state else None
        if op == "mix_backward":
            s["do"] = normal(B, T, H, dv)
            s["ds_T"] = normal(B, H, dk, dv, dtype=f32) if state else None
    return s


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2402_19427_b200 import binding
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        return binding.layer_norm(s["x"], s["weight"], s["bias"], center=c["center"])
    if op == "norm_backward":
        return binding.layer_norm_backward(s["dy"], s["x"], s["rstd"], mean=s["mean"], weight=s["weight"])
    if op == "norm_step":
        y, mean, rstd = binding.layer_norm(s["x"], s["weight"], s["bias"], center=c["center"], stats=True)
        return dict(binding.layer_norm_backward(s["dy"], s["x"], rstd, mean=mean, weight=s["weight"]), y=y)
    if op == "linear":
        if c["act"] == "none":
            return binding.linear(s["x"], s["weight"], s["bias"], residual=s["residual"])
        return binding.linear(s["x"], s["weight"], s["bias"], activation=c["act"], residual=s["residual"], keep_preact=True)
    if op == "linear_backward":
        return binding.linear_backward(s["dy"], s["x"], s["weight"], preact=s["preact"], activation=c["act"])
    if op == "mix":
        return binding.linear_attention_prefill(s["q"], s["k"], s["v"], s["log_decay"], s0=s["s0"])
    if op == "mix_step":
        return binding.linear_attention_decode_step(s["q"], s["k"], s["v"], s["log_decay"], s["s0"]), s["s0"]
    return binding.linear_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["do"], s0=s["s0"], ds_T=s["ds_T"], state_grads=c["state"])


# ------------------------------------------------------------------ plain forms
def _plain_norm(x, weight, bias, center, dt):
    x = x.float()
    mean = x.mean(-1, keepdim=True) if center else torch.zeros_like(x[:, :1])
    rstd = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + 1e-5)
    y = (x - mean) * rstd * weight
    return (y if bias is None else y + bias).to(dt), mean, rstd


def _plain_norm_backward(dy, x, mean, rstd, weight, center, dt):
    dy, xhat = dy.float(), (x.float() - mean) * rstd
    g = dy * weight
    dx = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if center:
        dx = dx - g.mean(-1, keepdim=True)
    return dict(x=(dx * rstd).to(dt), weight=(dy * xhat).sum(0), bias=dy.sum(0))


def _plain_act(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _plain_act_grad(z, act):
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _powers(log_decay, n):
    """decay ** n for each head: [H, *n.shape], the exponents in fp64."""
    return torch.exp(log_decay.double().reshape(-1, *[1] * n.dim()) * n.double()).float()


def _plain_mix(q, k, v, log_decay, s0, first, chunk=64):
    """o_t = sum_{s <= t} d^(t-s) (q_t k_s) v_s + d^(t+first) q_t S_0 and S_T = d^T S_0 + sum_s d^(T-s-first) k_s v_s^T over [B,T,H,*] in
    fp32: products within chunks of tokens, the states at their borders as one product over the chunks."""
    q, k, v = (x.float().transpose(1, 2) for x in (q, k, v))
    B, H, T, dk = q.shape
    dv, n = v.shape[-1], -(-T // chunk)
    at = torch.arange(n * chunk, device=q.device)
    s_T = (k * _powers(log_decay, T - first - at[:T])[..., None]).transpose(-1, -2) @ v
    if s0 is not None:
        s_T = s_T + _powers(log_decay, at.new_full((1, 1), T)) * s0
    q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, n * chunk - T)).reshape(B, H, n, chunk, -1) for x in (q, k, v))
    i = at[:chunk]
    apart = i[:, None] - i
    near = torch.where(apart >= 0, _powers(log_decay, apart.clamp(min=0)), 0.0)
    o = (q @ k.transpose(-1, -2) * near[:, None]) @ v
    local = (k * _powers(log_decay, chunk - first - i)[:, None, :, None]).transpose(-1, -2) @ v
    c = at[:n]
    before = c[:, None] - 1 - c
    far = torch.where(before >= 0, _powers(log_decay, chunk * before.clamp(min=0)), 0.0)
    states = (far @ local.reshape(B, H, n, dk * dv)).reshape(B, H, n, dk, dv)
    if s0 is not None:
        states = states + _powers(log_decay, chunk * c)[..., None, None] * s0[:, :, None]
    o = o + (q @ states) * _powers(log_decay, i + first)[:, None, :, None]
    return o.reshape(B, H, n * chunk, dv)[:, :, :T].transpose(1, 2), s_T


def run(state):
    if own:
        return _own(state)
    s, c, dt = state, state["case"], _dtype(state["case"])
    op = c["op"]
    if op == "norm":
        return _plain_norm(s["x"], s["weight"], s["bias"], c["center"], dt)[0]
    if op == "norm_backward":
        return _plain_norm_backward(s["dy"], s["x"], s["mean"][:, None] if c["center"] else 0.0, s["rstd"][:, None], s["weight"], c["center"], dt)
    if op == "norm_step":
        y, mean, rstd = _plain_norm(s["x"], s["weight"], s["bias"], c["center"], dt)
        return dict(_plain_norm_backward(s["dy"], s["x"], mean, rstd, s["weight"], c["center"], dt), y=y)
    if op == "linear":
        z = s["x"].float() @ s["weight"].float().T
        z = z if s["bias"] is None else z + s["bias"]
        y = _plain_act(z, c["act"])
        y = (y if s["residual"] is None else y + s["residual"].float()).to(dt)
        return y if c["act"] == "none" else (y, z.to(dt))
    if op == "linear_backward":
        dz = s["dy"].float()
        dz = dz if c["act"] == "none" else dz * _plain_act_grad(s["preact"].float(), c["act"])
        return dict(x=(dz @ s["weight"].float()).to(dt), weight=(dz.T @ s["x"].float()).to(dt), bias=dz.sum(0))
    scale = c["dk"] ** -0.5
    if op == "mix":
        o, s_T = _plain_mix(s["q"], s["k"], s["v"], s["log_decay"], s["s0"], 1)
        return (o * scale).to(dt), s_T
    if op == "mix_step":
        q, k, v = (s[n].float() for n in "qkv")
        s["s0"].mul_(_powers(s["log_decay"], torch.ones(1, 1, device=q.device))).add_(k[..., :, None] * v[..., None, :])
        return ((q[..., None, :] @ s["s0"])[..., 0, :] * scale).to(dt), s["s0"]
    back = lambda t: t.flip(1)  # noqa: E731
    turned = lambda t: None if t is None else t.transpose(-1, -2)  # noqa: E731
    do = s["do"].float() * scale
    dq, _ = _plain_mix(do, s["v"], s["k"], s["log_decay"], turned(s["s0"]), 1)
    dk, _ = _plain_mix(back(s["v"]), back(do), back(s["q"]), s["log_decay"], turned(s["ds_T"]), 0)
    dv, ds0 = _plain_mix(back(s["k"]), back(s["q"]), back(do), s["log_decay"], s["ds_T"], 0)
    out = dict(q=dq.to(dt), k=back(dk).to(dt), v=back(dv).to(dt))
    return dict(out, s0=ds0) if c["state"] else out


# ------------------------------------------------------------------ definitions in 64 bits
def exact(case, seed):
    s, c, f64 = prepare(case, seed), case, torch.float64
    op, d = c["op"], {}
    for name, t in s.items():
        d[name] = t.to(f64) if isinstance(t, torch.Tensor) else t
    if op.startswith("norm"):
        x, N = d["x"], c["N"]
        if op == "norm_backward":
            mu, inv = (d["mean"] if c["center"] else torch.zeros_like(d["rstd"])), d["rstd"]
        else:
            mu = x.sum(1) / N if c["center"] else torch.zeros_like(x[:, 0])
            inv = ((x - mu[:, None]).pow(2).sum(1) / N + 1e-5).pow(-0.5)
        h = torch.einsum("rn,r->rn", x - mu[:, None], inv)
        y = h * d["weight"] + (d["bias"] if d["bias"] is not None else 0.0)
        if op == "norm":
            return y
        w, dy = d["weight"], d["dy"]
        along = torch.einsum("rn,n,rn->r", dy, w, h) / N
        level = torch.einsum("rn,n->r", dy, w) / N if c["center"] else torch.zeros_like(along)
        out = dict(x=torch.einsum("rn,r->rn", dy * w - level[:, None] - h * along[:, None], inv), weight=torch.einsum("rn,rn->n", dy, h),
                   bias=torch.einsum("rn->n", dy))
        return out if op == "norm_backward" else dict(out, y=y)
    if op.startswith("linear"):
        phi = lambda z: torch.special.ndtr(z)  # noqa: E731
        if op == "linear":
            z = torch.einsum("mk,nk->mn", d["x"], d["weight"]) + (d["bias"] if d["bias"] is not None else 0.0)
            y = z * phi(z) if c["act"] == "gelu" else z * torch.sigmoid(z) if c["act"] == "silu" else z
            y = y + (d["residual"] if d["residual"] is not None else 0.0)
            return y if c["act"] == "none" else (y, z)
        dz = d["dy"]
        if c["act"] != "none":
            z = d["preact"]
            sig = torch.sigmoid(z)
            slope = phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if c["act"] == "gelu" else sig + z * sig * (1 - sig)
            dz = dz * slope
        return dict(x=torch.einsum("mn,nk->mk", dz, d["weight"]), weight=torch.einsum("mn,mk->nk", dz, d["x"]), bias=torch.einsum("mn->n", dz))
    # token by token, as the recurrence is written
    decay = torch.exp(d["log_decay"])[None, :, None, None]
    scale, q, k, v = 1.0 / math.sqrt(c["dk"]), d["q"], d["k"], d["v"]
    if op == "mix_step":
        st = decay * d["s0"] + torch.einsum("bhd,bhe->bhde", k, v)
        return torch.einsum("bhd,bhde->bhe", q, st) * scale, st
    B, T, H, dk, dv = (c[n] for n in ("B", "T", "H", "dk", "dv"))
    if T * B * H * dk * dv > 4e11:
        return None
    st = torch.zeros(B, H, dk, dv, dtype=f64, device=q.device) if d["s0"] is None else d["s0"].clone()
    rows, keep = [], op == "mix"
    for t in range(T):
        st.mul_(decay).addcmul_(k[:, t, :, :, None], v[:, t, :, None, :])
        rows.append(torch.matmul(q[:, t, :, None, :], st)[:, :, 0] if keep else torch.matmul(st, d["do"][:, t, :, :, None])[..., 0])
    first = torch.stack(rows, 1) * scale
    if keep:
        return first, st
    g = torch.zeros_like(st) if d["ds_T"] is None else d["ds_T"].clone()
    dks, dvs = [], []
    for t in reversed(range(T)):
        g.addcmul_(q[:, t, :, :, None] * scale, d["do"][:, t, :, None, :])
        dks.append(torch.matmul(g, v[:, t, :, :, None])[..., 0])
        dvs.append(torch.matmul(k[:, t, :, None, :], g)[:, :, 0])
        g.mul_(decay)
    out = dict(q=first, k=torch.stack(dks[::-1], 1), v=torch.stack(dvs[::-1], 1))
    return dict(out, s0=g) if c["state"] else out


def work(case):
    op, e = case["op"], 2 if case["io"] == "bf16" else 4
    if op.startswith("norm"):
        n, N = case["rows"] * case["N"], case["N"]
        passes = {"norm": 2, "norm_backward": 3, "norm_step": 4}[op]   # x, y; dy, x, dx; x, dy, y, dx
        vectors = 4 * N * {"norm": 1 + case["bias"], "norm_backward": 3, "norm_step": 3 + case["bias"]}[op]
        stats = 4 * case["rows"] * (1 + case["center"]) if op == "norm_backward" else 0
        return {"bytes": passes * n * e + vectors + stats, "flops": n * {"norm": 7, "norm_backward": 12, "norm_step": 19}[op]}
    if op.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        if op == "linear":
            outs = M * N * (1 + (case["act"] != "none") + case["residual"])
            return {"bytes": (M * K + N * K + outs) * e + 4 * N * case["bias"], "flops": 2 * M * N * K}
        return {"bytes": (2 * M * K + 2 * N * K + M * N * (1 + (case["act"] != "none"))) * e + 4 * N, "flops": 4 * M * N * K}
    B, T, H, dk, dv = (case[k] for k in ("B", "T", "H", "dk", "dv"))
    tok, mat = B * T * H, 4 * B * H * dk * dv
    if op == "mix_step":
        return {"bytes": tok * 2 * (dk + dv) * e + 2 * mat + 4 * H, "flops": tok * 5 * dk * dv}
    if op == "mix":   # the recurrence's products: state and output
        return {"bytes": tok * 2 * (dk + dv) * e + mat * (1 + case["state"]) + 4 * H, "flops": tok * 4 * dk * dv}
    return {"bytes": tok * (4 * dk + 3 * dv) * e + mat * 3 * case["state"] + 4 * H, "flops": tok * 10 * dk * dv}
