"""The entry points around the temporal core refuse what they cannot serve: every call below fails validation before any CUDA work."""
import ctypes

import pytest
import torch

vp = ctypes.c_void_p
GOOD = 0x7F0000000000   # aligned, never dereferenced
FAR = 1 << 32           # between buffers that must not meet


@pytest.fixture(scope="module")
def b():
    from paper_2402_19427_b200 import binding, build
    build.build()
    binding.load()
    return binding


def at(i, off=0):
    return vp(GOOD + i * FAR + off)


def test_norm(b):
    lib, S = b.load(), b.NormShape

    def fwd(shape=S(4, 64, b.BF16, 1, 1e-5), x=at(0), w=at(1), bias=at(2), y=at(3), mean=at(4), rstd=at(5)):
        return lib.rglru_layer_norm(ctypes.byref(shape) if shape else None, x, w, bias, y, mean, rstd, None)

    assert fwd(shape=None) == b.ERR_NULL and fwd(x=None) == b.ERR_NULL and fwd(y=None) == b.ERR_NULL
    for bad in (S(0, 64, 1, 1, 1e-5), S(4, 0, 1, 1, 1e-5), S(-1, 64, 1, 1, 1e-5), S(4, 64, 1, 1, -1.0), S(4, 64, 1, 1, float("nan")), S(4, (1 << 30) + 1, 1, 1, 0), S(1 << 60, 64, 1, 1, 0)):
        assert fwd(shape=bad) == b.ERR_SHAPE
    assert fwd(shape=S(4, 64, 2, 1, 1e-5)) == b.ERR_UNSUPPORTED
    for name in ("x", "w", "bias", "y", "mean", "rstd"):
        assert fwd(**{name: at(0, 4)}) == b.ERR_ALIGN, name
    assert fwd(y=at(0)) == b.ERR_ALIAS and fwd(y=at(0, 496)) == b.ERR_ALIAS

    def bwd(shape=S(4, 64, b.BF16, 1, 0.0), dy=at(0), x=at(1), mean=at(2), rstd=at(3), w=at(4), dx=at(5), dw=at(6), db=at(7), ws=at(8), n=1 << 20):
        return lib.rglru_layer_norm_backward(ctypes.byref(shape), dy, x, mean, rstd, w, dx, dw, db, ws, n, None)

    for name in ("dy", "x", "mean", "rstd", "dx", "ws"):
        assert bwd(**{name: None}) == b.ERR_NULL, name
    assert bwd(ws=at(8, 16)) == b.ERR_ALIGN and bwd(dw=at(6, 4)) == b.ERR_ALIGN
    assert bwd(n=16) == b.ERR_WORKSPACE and bwd(dx=at(0)) == b.ERR_ALIAS and bwd(dx=at(1, 16)) == b.ERR_ALIAS
    assert lib.rglru_layer_norm_workspace_bytes(ctypes.byref(S(4, 64, 1, 1, 0.0))) >= 2 * 64 * 4
    assert lib.rglru_layer_norm_workspace_bytes(ctypes.byref(S(4, 0, 1, 1, 0.0))) == 0


def test_linear(b):
    lib, S = b.load(), b.LinearShape
    ok = S(8, 64, 32, b.BF16, 1, 0)

    def fwd(shape=ok, x=at(0), w=at(1), bias=at(2), res=at(3), y=at(4), pre=at(5), ws=at(6), n=1 << 30):
        return lib.rglru_linear(ctypes.byref(shape) if shape else None, x, w, bias, res, y, pre, ws, n, None)

    for name in ("x", "w", "y", "ws", "shape"):
        assert fwd(**{name: None}) == b.ERR_NULL, name
    for bad in (S(0, 64, 32, 1, 0, 0), S(8, 0, 32, 1, 0, 0), S(8, 64, -1, 1, 0, 0), S(1 << 31, 64, 32, 1, 0, 0)):
        assert fwd(shape=bad) == b.ERR_SHAPE
    assert fwd(shape=S(8, 64, 32, 3, 0, 0)) == b.ERR_UNSUPPORTED and fwd(shape=S(8, 64, 32, 1, 3, 0)) == b.ERR_UNSUPPORTED and fwd(shape=S(8, 64, 32, 1, -1, 0)) == b.ERR_UNSUPPORTED
    for name in ("x", "w", "bias", "res", "y", "pre", "ws"):
        assert fwd(**{name: at(9, 8)}) == b.ERR_ALIGN, name
    assert fwd(n=16) == b.ERR_WORKSPACE
    assert fwd(y=at(0)) == b.ERR_ALIAS and fwd(y=at(1)) == b.ERR_ALIAS and fwd(y=at(3, 16)) == b.ERR_ALIAS and fwd(y=at(5)) == b.ERR_ALIAS
    assert fwd(pre=at(3)) == b.ERR_ALIAS and fwd(pre=at(0)) == b.ERR_ALIAS

    def bwd(shape=ok, dy=at(0), x=at(1), w=at(2), pre=at(3), dx=at(4), dw=at(5), db=at(6), ws=at(7), n=1 << 30):
        return lib.rglru_linear_backward(ctypes.byref(shape), dy, x, w, pre, dx, dw, db, ws, n, None)

    for name in ("dy", "x", "w", "pre", "ws"):
        assert bwd(**{name: None}) == b.ERR_NULL, name
    assert bwd(db=at(6, 4)) == b.ERR_ALIGN and bwd(n=300) == b.ERR_WORKSPACE
    assert bwd(dx=at(0)) == b.ERR_ALIAS and bwd(dw=at(2)) == b.ERR_ALIAS and bwd(dw=at(4)) == b.ERR_ALIAS and bwd(db=at(5, 64)) == b.ERR_ALIAS
    assert lib.rglru_linear_workspace_bytes(ctypes.byref(ok), b.OP_DECODE) == 0 and lib.rglru_linear_workspace_bytes(ctypes.byref(ok), b.OP_PREFILL) >= 256


def test_linear_attention(b):
    lib, S, St = b.load(), b.LinearAttentionShape, b.LinearAttentionStrides
    ok = S(2, 16, 2, 64, 32, b.BF16, 0.125, 0)

    def fwd(shape=ok, st=None, q=at(0), k=at(1), v=at(2), ld=at(3), s0=at(4), o=at(5), sT=at(6), ws=at(7), n=1 << 30):
        return lib.rglru_linear_attention_prefill(ctypes.byref(shape) if shape else None, ctypes.byref(st) if st else None, q, k, v, ld, s0, o, sT, ws, n, None)

    for name in ("q", "k", "v", "ld", "o", "sT", "ws", "shape"):
        assert fwd(**{name: None}) == b.ERR_NULL, name
    for i, bad in enumerate([0, -1, 0, 0, 0]):
        dims = [2, 16, 2, 64, 32]; dims[i] = bad
        assert fwd(shape=S(*dims, b.BF16, 0.125, 0)) == b.ERR_SHAPE
    assert fwd(shape=S(2, 16, 2, 64, 32, b.BF16, float("nan"), 0)) == b.ERR_SHAPE
    for bad in (S(2, 16, 2, 264, 32, 1, 1.0, 0), S(2, 16, 2, 64, 257, 1, 1.0, 0), S(2, 16, 2, 64, 32, 4, 1.0, 0), S(1 << 20, 16, 1 << 10, 64, 32, 1, 1.0, 0)):
        assert fwd(shape=bad) == b.ERR_UNSUPPORTED
    for name in ("q", "k", "v", "ld", "s0", "o", "sT", "ws"):
        assert fwd(**{name: at(9, 8)}) == b.ERR_ALIGN, name
    assert fwd(n=16) == b.ERR_WORKSPACE
    for name in ("q", "k", "v", "s0"):
        assert fwd(**{name: at(5)}) == b.ERR_ALIAS, name
    assert fwd(sT=at(4, 16)) == b.ERR_ALIAS and fwd(sT=at(0)) == b.ERR_ALIAS
    for token, batch in ((64, 2048), (128, 64), (-128, 2048), (128, 1920 - 1), (0, 2048)):   # tokens over one another
        st = St(); st.q[0], st.q[1] = token, batch
        assert fwd(st=st) == b.ERR_SHAPE, (token, batch)
    st = St(); st.o[0], st.o[1] = 64 * 3, 64 * 3 * 16      # reaches further than a dense tensor: into s_T
    assert fwd(st=st, sT=at(5, 4096)) == b.ERR_ALIAS

    def step(shape=ok, q=at(0), k=at(1), v=at(2), ld=at(3), s=at(4), o=at(5)):
        return lib.rglru_linear_attention_decode_step(ctypes.byref(shape) if shape else None, q, k, v, ld, s, o, None)

    for name in ("q", "k", "v", "ld", "s", "o", "shape"):
        assert step(**{name: None}) == b.ERR_NULL, name
    assert step(shape=S(2, 0, 0, 64, 32, 1, 1.0, 0)) == b.ERR_SHAPE and step(shape=S(2, 0, 2, 5000, 32, 1, 1.0, 0)) == b.ERR_UNSUPPORTED
    assert step(s=at(4, 4)) == b.ERR_ALIGN and step(o=at(0)) == b.ERR_ALIAS and step(o=at(4)) == b.ERR_ALIAS and step(s=at(2)) == b.ERR_ALIAS

    def bwd(shape=ok, st=None, q=at(0), k=at(1), v=at(2), ld=at(3), s0=at(4), do=at(5), dsT=at(6), dq=at(7), dk=at(8), dv=at(9), ds0=at(10), ws=at(11), n=1 << 30):
        return lib.rglru_linear_attention_backward(ctypes.byref(shape), ctypes.byref(st) if st else None, q, k, v, ld, s0, do, dsT, dq, dk, dv, ds0, ws, n, None)

    for name in ("q", "k", "v", "ld", "do", "dq", "dk", "dv", "ws"):
        assert bwd(**{name: None}) == b.ERR_NULL, name
    assert bwd(dsT=at(6, 4)) == b.ERR_ALIGN and bwd(n=16) == b.ERR_WORKSPACE
    for out in ("dq", "dk", "dv", "ds0"):
        for i in (0, 1, 2, 4, 5, 6):
            assert bwd(**{out: at(i)}) == b.ERR_ALIAS, (out, i)
    assert bwd(dk=at(7)) == b.ERR_ALIAS and bwd(ds0=at(9)) == b.ERR_ALIAS
    assert lib.rglru_linear_attention_workspace_bytes(ctypes.byref(ok), b.OP_PREFILL) >= 256 and lib.rglru_linear_attention_workspace_bytes(ctypes.byref(ok), b.OP_DECODE) == 0


def test_binding_names_the_wrong_argument(b):
    """CPU tensors and wrong arguments are refused before anything is allocated on a device."""
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="no CPU fallback"):
        b.layer_norm(x)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        b.layer_norm(x.half())
    with pytest.raises(TypeError, match="x: expected a tensor"):
        b.layer_norm(None)
    with pytest.raises(TypeError, match="weight: expected a tensor or None"):
        b.layer_norm(x, 3.0)
    with pytest.raises(ValueError, match="no CPU fallback"):
        b.linear(x, torch.zeros(8, 64))
    with pytest.raises(ValueError, match="activation"):
        b.linear(x, torch.zeros(8, 64), activation="tanh")
    with pytest.raises(ValueError, match="need"):
        b.linear_backward(x, x, x, need=("x", "y"))
    q = torch.zeros(1, 4, 2, 16)
    with pytest.raises(ValueError, match="no CPU fallback"):
        b.linear_attention_prefill(q, q, q, torch.zeros(2))
    with pytest.raises(TypeError, match="log_decay"):
        b.linear_attention_decode_step(q[:, 0], q[:, 0], q[:, 0], None, q)


def test_gradients_side_by_side(b):
    """dq, dk and dv may be parts of one row (the GPU tests run them so), but no byte of one may lie in another"""
    lib, S, St = b.load(), b.LinearAttentionShape, b.LinearAttentionStrides
    for token, batch in ((2 * 128 + 64, 16 * 320), (2 * 320, 320)):   # [B,T,320] and [T,B,320]
        st = St()
        for name in ("dq", "dk", "dv"):
            getattr(st, name)[0], getattr(st, name)[1] = token, batch

        def bwd(dq, dk, dv, n, st=st):
            shape = S(2, 16, 2, 64, 32, b.BF16, 0.125, 0)
            return lib.rglru_linear_attention_backward(ctypes.byref(shape), ctypes.byref(st), at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7, dq), at(7, dk), at(7, dv),
                                                       at(10), at(11), n, None)

        big = 1 << 30
        for dq, dk, dv in ((0, 240, 512), (0, 256, 496), (0, 256, 528), (0, 0, 512), (256, 0, 256), (0, 256, 256), (0, 256, 640 * 3 + 512 - 16), (512 + 16, 0, 256)):
            assert bwd(dq, dk, dv, big) == b.ERR_ALIAS, (dq, dk, dv)
    other = St()
    for name, token in (("dq", 320), ("dk", 320), ("dv", 640)):
        getattr(other, name)[0], getattr(other, name)[1] = token, 32 * token
    assert bwd(0, 256, 512, big, other) == b.ERR_ALIAS


def test_gradients_side_by_side_in_sequences_without_a_gap(b):
    """A sequence's last token row and the next sequence's first may not share bytes either, when the distance between sequences is no multiple
    of the one between tokens"""
    lib, S, St = b.load(), b.LinearAttentionShape, b.LinearAttentionStrides
    B, T = 2, 16
    shape = S(B, T, 2, 64, 32, b.BF16, 0.125, 0)

    def bwd(token, batch, offsets):
        st = St()
        for name in ("dq", "dk", "dv"):
            getattr(st, name)[0], getattr(st, name)[1] = token, batch
        return lib.rglru_linear_attention_backward(ctypes.byref(shape), ctypes.byref(st), at(0), at(1), at(2), at(3), at(4), at(5), at(6),
                                                   *(at(7, 2 * o) for o in offsets), at(10), at(11), 1 << 30, None)

    # rows of 128 (dq), 128 (dk) and 64 (dv) elements, 320 from row to row; the outer distance ends behind the first of them
    for outer_of in ((lambda n: (320, (n - 1) * 320 + 128)), (lambda n: ((n - 1) * 320 + 128, 320))):   # [B,T,...] and [T,B,...]
        inner = T if outer_of(2)[0] == 320 else B
        assert bwd(*outer_of(inner), (0, 128, 256)) == b.ERR_ALIAS


def test_every_workspace_has_room_for_the_status(b):
    """256 bytes in front of what a call puts there: the partial sums of the norm's gradients [blocks][2][N] fp32 (one row: one block)"""
    assert b.load().rglru_layer_norm_workspace_bytes(ctypes.byref(b.NormShape(1, 64, b.BF16, 1, 0.0))) == 256 + 2 * 64 * 4


def test_sizes_behind_which_indices_would_not_fit(b):
    """A row of nearly 2^31 elements fits the memory, but not the kernels' 32-bit columns: refused, as the header says"""
    lib, big, r = b.load(), (1 << 31) - 1016, ctypes.byref
    assert lib.rglru_linear(r(b.LinearShape(1, 8, big, b.BF16, 0, 0)), at(0), at(1), None, None, at(2), None, at(3), 1 << 40, None) == b.ERR_SHAPE
    assert lib.rglru_linear_backward(r(b.LinearShape(1, 8, big, b.BF16, 0, 0)), at(0), at(1), at(2), None, None, None, at(3), at(4), 1 << 40, None) == b.ERR_SHAPE
    assert lib.rglru_linear(r(b.LinearShape(1, big, 8, b.BF16, 0, 0)), at(0), at(1), None, None, at(2), None, at(3), 1 << 40, None) == b.ERR_SHAPE
    assert lib.rglru_linear_attention_decode_step(r(b.LinearAttentionShape(1, 0, 1, 1, big, b.F32, 1.0, 0)), at(0), at(1), at(2), at(3), at(4), at(5 + 4), None) == b.ERR_UNSUPPORTED
    assert lib.rglru_linear_attention_decode_step(r(b.LinearAttentionShape(1, 0, 1, 4104, 8, b.F32, 1.0, 0)), at(0), at(1), at(2), at(3), at(4), at(5), None) == b.ERR_UNSUPPORTED
    # sizes are computed without overflow up to there
    assert lib.rglru_linear_workspace_bytes(r(b.LinearShape(8, 1 << 30, 1 << 30, b.F32, 0, 0)), b.OP_PREFILL) == 256


def test_outputs_over_vectors(b):
    """No output may lie over a vector that other blocks still read, or over another output"""
    lib, r = b.load(), ctypes.byref
    n = b.NormShape(40, 64, b.BF16, 1, 1e-5)

    def fwd(x=at(0), w=at(1), bias=at(2), y=at(3), mean=at(4), rstd=at(5)):
        return lib.rglru_layer_norm(r(n), x, w, bias, y, mean, rstd, None)

    for bad in (dict(w=at(3)), dict(bias=at(3, 5104)), dict(mean=at(3)), dict(rstd=at(3, 16)), dict(mean=at(0)), dict(rstd=at(0, 5104)), dict(mean=at(1)), dict(rstd=at(2, 240)),
                dict(mean=at(5, 144))):
        assert fwd(**bad) == b.ERR_ALIAS, bad

    def bwd(dy=at(0), x=at(1), mean=at(2), rstd=at(3), w=at(4), dx=at(5), dw=at(6), db=at(7)):
        return lib.rglru_layer_norm_backward(r(n), dy, x, mean, rstd, w, dx, dw, db, at(8), 1 << 30, None)

    for bad in (dict(mean=at(5)), dict(rstd=at(5, 16)), dict(w=at(5, 5104)), dict(dw=at(5)), dict(db=at(5, 16)), dict(db=at(6, 240))):
        assert bwd(**bad) == b.ERR_ALIAS, bad
    lin = b.LinearShape(40, 64, 96, b.BF16, 1, 0)

    def linear(x=at(0), w=at(1), bias=at(2), res=at(3), y=at(4), pre=at(5)):
        return lib.rglru_linear(r(lin), x, w, bias, res, y, pre, at(6), 1 << 30, None)

    for bad in (dict(bias=at(4)), dict(bias=at(5, 16))):
        assert linear(**bad) == b.ERR_ALIAS, bad
    mix = b.LinearAttentionShape(2, 16, 2, 64, 32, b.BF16, 0.125, 0)
    for o, sT in ((at(3), at(6)), (at(5), at(3))):
        assert lib.rglru_linear_attention_prefill(r(mix), None, at(0), at(1), at(2), at(3), at(4), o, sT, at(7), 1 << 30, None) == b.ERR_ALIAS
        assert lib.rglru_linear_attention_decode_step(r(mix), at(0), at(1), at(2), at(3), sT, o, None) == b.ERR_ALIAS
    for i in range(4):
        outs = [at(3) if i == j else at(7 + j) for j in range(4)]
        assert lib.rglru_linear_attention_backward(r(mix), None, at(0), at(1), at(2), at(3), at(4), at(5), at(6), *outs, at(11), 1 << 30, None) == b.ERR_ALIAS


def test_truth_values_that_have_none(b):
    """An argument whose truth cannot be told is named, instead of counting as False with an error left behind"""
    x, q = torch.zeros(4, 64), torch.zeros(1, 4, 2, 16)
    both = torch.tensor([True, False])
    with pytest.raises(TypeError, match="center"):
        b.layer_norm(x, center=both)
    with pytest.raises(TypeError, match="stats"):
        b.layer_norm(x, stats=both)
    with pytest.raises(TypeError, match="param_grads"):
        b.layer_norm_backward(x, x, x[:, 0], param_grads=both)
    with pytest.raises(TypeError, match="keep_preact"):
        b.linear(x, torch.zeros(8, 64), keep_preact=both)
    with pytest.raises(TypeError, match="state_grads"):
        b.linear_attention_backward(q, q, q, torch.zeros(2), q, state_grads=both)
