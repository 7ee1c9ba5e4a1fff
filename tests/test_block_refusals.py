"""What the layer norm, linear and rotary entry points refuse, before any HIP
call: through the C ABI with addresses that are never read, and through the
binding with CPU tensors."""
import ctypes
import math

import pytest
import torch

from paper_2406_08552_amd import dfa

INVALID, UNSUPPORTED = dfa.DFA_ERR_INVALID_ARG, dfa.DFA_ERR_UNSUPPORTED
X, W, BIAS, GATE, RES, Y, M1, M2, WS = (0x10000000 * (i + 1) for i in range(9))


@pytest.fixture(scope="module")
def L():
    return dfa.lib()


def norm(L, X=X, w=W, b=BIAS, Y=Y, mean=M1, rstd=M2, xt=dfa.BF16, B=2, l=8, C=64, ws=0, bs=0, off=0.0, eps=1e-6):
    return L.dfa_layer_norm(X, w, b, Y, mean, rstd, xt, B, l, C, ws, bs, off, eps, None)


@pytest.mark.parametrize("kw,status,message", [
    (dict(X=None), INVALID, "X is NULL"),
    (dict(Y=None), INVALID, "Y is NULL"),
    (dict(X=X + 8), INVALID, "aligned"),
    (dict(w=W + 2), INVALID, "aligned"),
    (dict(mean=M1 + 2), INVALID, "aligned"),
    (dict(xt=2), INVALID, "x_type"),
    (dict(B=0), INVALID, "positive"),
    (dict(l=0), INVALID, "positive"),
    (dict(C=0), INVALID, "positive"),
    (dict(C=16385), UNSUPPORTED, "16384"),
    (dict(B=1 << 16, l=1 << 15), INVALID, "too large"),
    (dict(ws=-1), INVALID, "stride"),
    (dict(bs=1 << 41), INVALID, "stride"),
    (dict(eps=-1.0), INVALID, "eps"),
    (dict(eps=math.nan), INVALID, "eps"),
    (dict(Y=X), INVALID, "overlaps"),
    (dict(Y=X + 16), INVALID, "overlaps"),
    (dict(mean=Y + 64), INVALID, "overlaps"),
    (dict(rstd=M1 + 60), INVALID, "overlaps"),            # mean is 64 bytes
    (dict(Y=W + 4 * 1000, ws=1000), INVALID, "weight"),   # inside the second entry's row
])
def test_layer_norm(L, kw, status, message):
    assert norm(L, **kw) == status
    assert message in dfa.last_error()


def grad(L, dY=RES, X=X, w=W, mean=M1, rstd=M2, dX=Y, dw=BIAS, db=GATE, ws=WS, nws=1 << 20, xt=dfa.F32, B=2, l=600, C=64,
         st=0, off=0.0, groups=1):
    return L.dfa_layer_norm_backward(dY, X, w, mean, rstd, dX, dw, db, ws, nws, xt, B, l, C, st, off, groups, None)


@pytest.mark.parametrize("kw,status,message", [
    (dict(dY=None), INVALID, "dY is NULL"),
    (dict(X=None), INVALID, "X is NULL"),
    (dict(dX=None), INVALID, "dX is NULL"),
    (dict(mean=None), INVALID, "mean is NULL"),
    (dict(rstd=None), INVALID, "rstd is NULL"),
    (dict(dw=BIAS + 1), INVALID, "aligned"),
    (dict(ws=WS + 4), INVALID, "aligned"),
    (dict(ws=None), INVALID, "workspace is NULL"),
    (dict(nws=16), INVALID, "too small"),
    (dict(groups=0), INVALID, "groups"),
    (dict(groups=3), INVALID, "groups"),
    (dict(B=1 << 23, l=1, groups=1 << 23), INVALID, "2^21"),
    (dict(xt=-1), INVALID, "x_type"),
    (dict(C=20000), UNSUPPORTED, "16384"),
    (dict(dX=X), INVALID, "overlaps"),
    (dict(dX=RES), INVALID, "overlaps"),
    (dict(db=BIAS + 128), INVALID, "overlaps"),
    (dict(ws=Y + 1024), INVALID, "overlaps"),
])
def test_layer_norm_backward(L, kw, status, message):
    assert grad(L, **kw) == status
    assert message in dfa.last_error()


def test_layer_norm_backward_workspace():
    assert dfa.layer_norm_backward_workspace_bytes(2, 600, 64, 1) > 0
    assert dfa.layer_norm_backward_workspace_bytes(2, 1, 64, 2) == 0       # a token per group: no partial sums
    for bad in ((0, 5, 64, 1), (2, 5, 64, 3), (2, 5, 1 << 15, 1), (-1, 5, 64, -1)):
        assert dfa.layer_norm_backward_workspace_bytes(*bad) == 0


def linear(L, X=X, W=W, bias=BIAS, gate=GATE, res=RES, Y=Y, act=0, yt=dfa.BF16, B=2, l=8, H=1, K=64, N=32, gs=0):
    return L.dfa_linear(X, W, bias, gate, res, Y, act, yt, B, l, H, K, N, gs, None)


@pytest.mark.parametrize("kw,status,message", [
    (dict(X=None), INVALID, "X is NULL"),
    (dict(W=None), INVALID, "W is NULL"),
    (dict(Y=None), INVALID, "Y is NULL"),
    (dict(W=W + 2), INVALID, "aligned"),
    (dict(bias=BIAS + 2), INVALID, "aligned"),
    (dict(res=RES + 4), INVALID, "aligned"),
    (dict(act=4), INVALID, "activation"),
    (dict(act=-1), INVALID, "activation"),
    (dict(yt=7), INVALID, "y_type"),
    (dict(B=0), INVALID, "positive"),
    (dict(K=0), INVALID, "positive"),
    (dict(N=-4), INVALID, "positive"),
    (dict(K=(1 << 20) + 8), INVALID, "2^20"),
    (dict(N=(1 << 20) + 1), INVALID, "2^20"),
    (dict(B=1 << 16, l=1 << 15), INVALID, "too large"),
    (dict(H=0), INVALID, "heads"),
    (dict(H=3), INVALID, "heads"),
    (dict(H=2), UNSUPPORTED, "head dim"),                 # K / H = 32
    (dict(gs=-2), INVALID, "stride"),
    (dict(Y=X), INVALID, "overlaps"),
    (dict(Y=W), INVALID, "overlaps"),
    (dict(res=Y + 16), INVALID, "overlaps"),              # the residual may be Y, not a part of it
    (dict(gate=Y + 4), INVALID, "overlaps"),
])
def test_linear(L, kw, status, message):
    assert linear(L, **kw) == status
    assert message in dfa.last_error()


def rope(L, Q=X, K=W, Qo=Y, Ko=RES, pos=BIAS, sections=(8, 24), naxes=None, base=1e4, B=2, Hq=4, Hk=2, l=8, d=64, ps=0):
    sec = (ctypes.c_int32 * 8)(*sections) if sections is not None else None
    return L.dfa_rope(Q, K, Qo, Ko, pos, sec, len(sections or ()) if naxes is None else naxes, base, 0, 0, B, Hq, Hk, l, d, ps, None)


@pytest.mark.parametrize("kw,status,message", [
    (dict(Q=None), INVALID, "Q is NULL"),
    (dict(Qo=None), INVALID, "Qout is NULL"),
    (dict(Ko=None), INVALID, "Kout is NULL"),
    (dict(K=None), INVALID, "K is NULL"),
    (dict(Hk=0), INVALID, "Hk"),
    (dict(K=None, Ko=None), INVALID, "Hk"),
    (dict(pos=None), INVALID, "pos is NULL"),
    (dict(pos=BIAS + 2), INVALID, "aligned"),
    (dict(Q=X + 2), INVALID, "aligned"),
    (dict(sections=None, naxes=1), INVALID, "sections is NULL"),
    (dict(naxes=0), INVALID, "naxes"),
    (dict(sections=(2, 2, 2, 2, 2)), INVALID, "naxes"),
    (dict(sections=(8, 7)), INVALID, "even"),
    (dict(sections=(0, 8)), INVALID, "even"),
    (dict(sections=(-2, 8)), INVALID, "even"),
    (dict(sections=(40, 26)), INVALID, "exceed"),
    (dict(base=0.0), INVALID, "base"),
    (dict(base=math.inf), INVALID, "base"),
    (dict(base=math.nan), INVALID, "base"),
    (dict(d=63), UNSUPPORTED, "head dim"),
    (dict(d=258), UNSUPPORTED, "head dim"),
    (dict(l=0), INVALID, "positive"),
    (dict(Hk=-1), INVALID, "positive"),
    (dict(B=1 << 20, l=1 << 11), INVALID, "too large"),
    (dict(ps=-1), INVALID, "stride"),
    (dict(Qo=X + 16), INVALID, "overlaps"),               # in place, but not shifted
    (dict(Qo=W), INVALID, "overlaps"),
    (dict(Ko=X), INVALID, "overlaps"),
    (dict(Ko=Y + 64), INVALID, "overlaps"),
    (dict(Ko=BIAS), INVALID, "overlaps"),
])
def test_rope(L, kw, status, message):
    assert rope(L, **kw) == status
    assert message in dfa.last_error()


def test_binding_refuses_host_tensors():
    """Before any address reaches the library, whatever the other arguments are."""
    t = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    v, s = torch.zeros(64), torch.zeros(1, 4)
    h = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        dfa.dfa_layer_norm(t, v, v, t.clone())
    with pytest.raises(ValueError, match="GPU"):
        dfa.dfa_layer_norm_backward(t, t, v, s, s, t.clone(), v, v)
    with pytest.raises(ValueError, match="GPU"):
        dfa.dfa_linear(t, torch.zeros(64, 64, dtype=torch.bfloat16), v, t.clone())
    with pytest.raises(ValueError, match="GPU"):
        dfa.dfa_rope(h, None, h, None, torch.zeros(4, 2), [8, 8])
    with pytest.raises(TypeError, match="bf16 or fp32"):
        dfa.dfa_layer_norm(t.half(), v, v, t)
    with pytest.raises(ValueError, match="B, L, C"):
        dfa.dfa_layer_norm(t[0], v, v, t)
    with pytest.raises(ValueError, match="neither"):
        dfa.dfa_rope(h, h, h, None, torch.zeros(4, 2), [8, 8])


def test_binding_refuses_sizes_past_32_bits():
    """The C ABI's sizes are int: a larger one must not arrive as its low bits."""
    big = (1 << 32) + 8
    m = lambda *n, dtype=torch.bfloat16: torch.empty(n, dtype=dtype, device="meta")  # noqa: E731
    v = torch.zeros(64)
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_layer_norm(m(1, big, 64), v, v, m(1, big, 64))
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_layer_norm_backward(m(1, big, 64), m(1, big, 64), v, v, v, m(1, big, 64), v, v)
    with pytest.raises(ValueError, match="too large"):
        dfa.layer_norm_backward_workspace_bytes(1, big, 64)
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_linear(m(1, 4, big), m(64, big), v, m(1, 4, 64))
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_linear(m(1, 1 << 28, 4, 64), m(64, 1 << 34), v, m(1, 4, 64))
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_linear(m(1, 4, 64), m(big, 64), None, m(1, 4, big))
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_linear(m(1, 4, 64), m(64, 64), v, m(1, 4, 64), act=1 << 32)
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_rope(m(1, 2, big, 8), None, m(1, 2, big, 8), None, m(big, 1, dtype=torch.float32), [8])
    with pytest.raises(ValueError, match="too large"):
        dfa.dfa_rope(m(1, 2, 4, 8), None, m(1, 2, 4, 8), None, m(4, 1, dtype=torch.float32), [big])
    with pytest.raises(TypeError):
        dfa.dfa_rope(m(1, 2, 4, 8), None, m(1, 2, 4, 8), None, m(4, 1, dtype=torch.float32), [7.5])
