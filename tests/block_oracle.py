"""Plain fp64 forms of the operators around the temporal core (torch, on whatever device the inputs are), and beside each result the sum of
the absolute values of its terms, from which the tests derive how far a correct kernel can be off."""
import torch

U32 = 2.0 ** -24   # half a step of fp32, relative
SMALLEST = 2.0 ** -126   # fp32 keeps no relative accuracy below: a term that has decayed this far may be lost


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def d(t):
    return None if t is None else t.double()


def assert_within(name, got, ref, bound):
    got, ref, bound = got.double(), ref.double(), bound.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{name}: values that are not finite"
    over = (got - ref).abs() - bound
    i = int(over.argmax())
    assert float(over.max()) <= 0, (f"{name}: {int((over > 0).sum())} of {over.numel()} outside; worst: got {float(got.flatten()[i]):.9e}, "
                                    f"ref {float(ref.flatten()[i]):.9e}, allowed {float(bound.flatten()[i]):.2e}")


# ---- norm
def norm(x, weight, bias, eps, center):
    x = d(x)
    mu = x.mean(-1, keepdim=True) if center else torch.zeros_like(x[..., :1])
    r = ((x - mu) ** 2).mean(-1, keepdim=True).add(eps).rsqrt()
    h = (x - mu) * r
    y = h * (1.0 if weight is None else d(weight)) + (0.0 if bias is None else d(bias))
    return y, mu[..., 0], r[..., 0]


def norm_bound(x, weight, bias, mu, r, dtype, y):
    """A sum in fp32 over at most 16 values a thread and eleven levels of a tree is off by at most 27 half steps of the sum of the
    magnitudes; the mean, the deviation and the mean square take one such sum each, and some ten roundings follow."""
    big = d(x).abs().amax(-1, keepdim=True) + mu[..., None].abs()
    off = 80 * U32 * (big * r[..., None] * (1.0 if weight is None else d(weight).abs())) * (1 + big * r[..., None])
    return off + (0.0 if bias is None else 2 * U32 * d(bias).abs()) + half_step(dtype) * y.abs()


def norm_backward(dy, x, mu, r, weight, center):
    dy, h = d(dy), (d(x) - (d(mu)[..., None] if center else 0.0)) * d(r)[..., None]
    g = dy * (1.0 if weight is None else d(weight))
    dx = g - h * (g * h).mean(-1, keepdim=True) - (g.mean(-1, keepdim=True) if center else 0.0)
    dx = dx * d(r)[..., None]
    rows = tuple(range(dy.dim() - 1))
    mag = g.abs() + h.abs() * (g * h).abs().mean(-1, keepdim=True) + g.abs().mean(-1, keepdim=True)
    return dx, (dy * h).sum(rows), dy.sum(rows), mag * d(r)[..., None].abs(), (dy * h).abs().sum(rows), dy.abs().sum(rows)


# ---- projection
def act(z, kind):
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    return z * torch.sigmoid(z) if kind == "silu" else z


def act_slope(z, kind):
    if kind == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    s = torch.sigmoid(z)
    return s + z * s * (1 - s) if kind == "silu" else torch.ones_like(z)


def linear(x, weight, bias, kind, residual):
    z = d(x) @ d(weight).T + (0.0 if bias is None else d(bias))
    mag = d(x).abs() @ d(weight).abs().T + (0.0 if bias is None else d(bias).abs())
    return act(z, kind) + (0.0 if residual is None else d(residual)), z, mag


# ---- linear attention, token by token as it is written
def attention(q, k, v, log_decay, s0, scale):
    """o, s_T, and the sums of magnitudes behind both"""
    q, k, v = d(q), d(k), d(v)
    B, T, H, dk = q.shape
    decay = torch.exp(d(log_decay)).reshape(1, H, 1, 1)
    s = torch.zeros(B, H, dk, v.shape[-1], dtype=torch.float64, device=q.device) if s0 is None else d(s0).clone()
    m = s.abs()
    o, om = [], []
    for t in range(T):
        s = decay * s + k[:, t, :, :, None] * v[:, t, :, None, :]
        m = decay * m + (k[:, t, :, :, None] * v[:, t, :, None, :]).abs()
        o.append((q[:, t, :, None, :] @ s)[:, :, 0] * scale)
        om.append((q[:, t, :, None, :].abs() @ m)[:, :, 0] * abs(scale))
    return torch.stack(o, 1), s, torch.stack(om, 1), m


def attention_backward(q, k, v, log_decay, do, s0, ds_T, scale):
    q, k, v, do = d(q), d(k), d(v), d(do)
    B, T, H, dk = q.shape
    decay = torch.exp(d(log_decay)).reshape(1, H, 1, 1)
    s = torch.zeros(B, H, dk, v.shape[-1], dtype=torch.float64, device=q.device) if s0 is None else d(s0).clone()
    m = s.abs()
    dq, dqm = [], []
    for t in range(T):
        s = decay * s + k[:, t, :, :, None] * v[:, t, :, None, :]
        m = decay * m + (k[:, t, :, :, None] * v[:, t, :, None, :]).abs()
        dq.append((s @ do[:, t, :, :, None])[..., 0] * scale)
        dqm.append((m @ do[:, t, :, :, None].abs())[..., 0] * abs(scale))
    g = torch.zeros_like(s) if ds_T is None else d(ds_T).clone()
    m = g.abs()
    dk_, dv_, dkm, dvm = [], [], [], []
    for t in reversed(range(T)):
        new = scale * q[:, t, :, :, None] * do[:, t, :, None, :]
        g, m = g + new, m + new.abs()
        dk_.append((g @ v[:, t, :, :, None])[..., 0]); dkm.append((m @ v[:, t, :, :, None].abs())[..., 0])
        dv_.append((k[:, t, :, None, :] @ g)[:, :, 0]); dvm.append((k[:, t, :, None, :].abs() @ m)[:, :, 0])
        g, m = decay * g, decay * m
    back = lambda xs: torch.stack(xs[::-1], 1)  # noqa: E731
    return (dict(q=torch.stack(dq, 1), k=back(dk_), v=back(dv_), s0=g), dict(q=torch.stack(dqm, 1), k=back(dkm), v=back(dvm), s0=m))


def attention_bound(mag, ref, dtype, T):
    """What an output or a gradient may be off by.  bf16: a product of q and k or a state is rounded once (half a step of a term's
    magnitude, two for the decay factor beside it in fp32), the result once.  fp32: sums of at most 256 terms in any order, and one rounding per
    32 tokens for the state that a term has travelled through."""
    terms = U32 * (512 + T / 8)
    if dtype == torch.bfloat16:
        terms = terms + 1.01 * half_step(dtype)
    return terms * mag + half_step(dtype) * ref.abs() + SMALLEST


def state_bound(mag, T):
    """fp32 sums over chunks of at most 128 tokens, and one rounding per 32 tokens"""
    return U32 * (512 + T / 8) * mag + SMALLEST
