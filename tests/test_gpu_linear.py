"""The linear layer against its definition in float64.

Bar, with u = 2^-23 for an addition whose rounding may be a truncation: the
product sums 16 terms at a time, then those sums, so it is off by at most
(K / 16 + 32) u sum|x w|; an activation's slope is at most 1.13, its own value
off by at most 8 u |z| (the argument of an exponential of up to 2^4 keeps
2^-20); the gate multiplies; each further operation rounds its result once, u;
and the output's rounding, 2^-8 for bf16 and 2^-24 for fp32."""
import math

import pytest
import torch

from paper_2406_08552_amd import dfa
from tests.test_gpu_parity import Guarded, say

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
U = 2.0 ** -23
BF16, F32 = torch.bfloat16, torch.float32
ACTS = {"none": dfa.ACT_NONE, "gelu": dfa.ACT_GELU, "gelu_tanh": dfa.ACT_GELU_TANH, "silu": dfa.ACT_SILU}


def _act64(z, act):
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _inputs(B, L, K, N, ytype, gate, seed, heads=1, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    X = r(B, heads, L, K // heads) if heads > 1 else r(B, L, K)
    gv = {"none": lambda: None, "shared": lambda: r(N), "batch": lambda: r(B, 2 * N + 1)[:, N:2 * N]}[gate]()
    return X.to(BF16), (r(N, K) * scale * K ** -0.5).to(BF16), r(N), gv, r(B, L, N).to(ytype)


def _check(got, X, W, bias, gate, res, act, B, L, K, N):
    x = X.double()
    if x.dim() == 4:
        x = x.transpose(1, 2).contiguous()
    x, w = x.reshape(B * L, K), W.double().t().contiguous()
    z = (x @ w).view(B, L, N)
    off = (K / 16 + 32) * U * (x.abs() @ w.abs()).view(B, L, N)
    if bias is not None:
        z = z + bias.double()
        off = off + U * z.abs()
    y = _act64(z, act)
    off = 1.13 * off + (8 * U * z.abs() if act != "none" else 0)
    if gate is not None:
        gd = gate.double().reshape(-1, 1, N)
        y, off = y * gd, off * gd.abs() + U * (y * gd).abs()
    if res is not None:
        y = y + res.double()
        off = off + U * y.abs()
    off = off + y.abs() * (2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24)
    err = (got.double() - y).abs()
    assert (err <= off).all(), f"{int((err > off).sum())} outputs off, max {float((err - off).max()):.3e}"


# (B, L, K, N): one token; few tokens; K of one element, below, at and past the
# steps of 8, 16, 64 and 128; N of one, odd, past a tile; many tokens
SHAPES = [(1, 1, 1, 1), (1, 1, 1152, 6912), (2, 1, 1152, 1152), (3, 1, 100, 33), (1, 5, 4608, 256), (2, 8, 72, 40), (1, 17, 1000, 130),
          (2, 16, 1152, 32), (1, 33, 7, 65), (3, 21, 64, 64), (1, 64, 136, 128), (5, 13, 128, 200), (2, 65, 192, 1), (1, 130, 1153, 129),
          (3, 101, 200, 192), (2, 301, 1152, 1152), (2, 301, 776, 1001), (1, 1100, 520, 1160), (4, 1024, 1152, 640), (2, 2500, 320, 2050),
          (1, 9001, 24, 390), (7, 700, 1032, 1152), (2, 4100, 576, 1920), (1, 12345, 640, 768)]


@pytest.mark.parametrize("ytype", [BF16, F32])
@pytest.mark.parametrize("B,L,K,N", SHAPES)
def test_shapes(B, L, K, N, ytype):
    X, W, bias, gate, res = _inputs(B, L, K, N, ytype, "batch", K + N + L)
    for act, b, g, r in (("none", None, None, None), ("gelu_tanh", bias, None, None), ("none", bias, gate, res), ("silu", bias, gate, None),
                         ("gelu", None, None, res)):
        say(f"linear {B} {L} {K} {N} {ytype} {act} bias={b is not None} gate={g is not None} res={r is not None}")
        Y = Guarded((B, L, N), DEV, ytype)
        dfa.dfa_linear(X, W, b, Y.t, act=ACTS[act], gate=g, residual=r)
        torch.cuda.synchronize()
        _check(Y.t, X, W, b, g, r, act, B, L, K, N)
        assert Y.guards_intact()


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("B,L,K,N", [(2, 1, 256, 96), (2, 40, 77, 64), (3, 200, 384, 256), (2, 3000, 256, 1152)])
def test_activations_over_their_range(B, L, K, N, act):
    """Arguments of both signs up to about 40, and 0."""
    X, W, bias, gate, res = _inputs(B, L, K, N, F32, "shared", 3 * K, scale=8.0)
    X[0, 0] = 0
    bias[: N // 2] = 0
    for ytype in (BF16, F32):
        Y = torch.zeros((B, L, N), dtype=ytype, device=DEV)
        dfa.dfa_linear(X, W, bias, Y, act=ACTS[act], gate=gate, residual=res.to(ytype))
        torch.cuda.synchronize()
        _check(Y, X, W, bias, gate, res.to(ytype), act, B, L, K, N)


@pytest.mark.parametrize("B,H,L,d,N", [(1, 2, 1, 64, 64), (2, 16, 1, 72, 1152), (2, 3, 5, 72, 100), (3, 16, 37, 72, 1152), (2, 6, 701, 64, 384),
                                      (32, 16, 45, 72, 1152), (2, 16, 2050, 72, 1152), (1, 5, 600, 64, 321), (3, 7, 333, 72, 504)])
def test_merged_heads(B, H, L, d, N):
    K = H * d
    X, W, bias, gate, res = _inputs(B, L, K, N, F32, "batch", 11 * L, heads=H)
    say(f"linear heads {B} {H} {L} {d} {N}")
    Y = Guarded((B, L, N), DEV, F32)
    dfa.dfa_linear(X, W, bias, Y.t, gate=gate, residual=res)
    merged = X.transpose(1, 2).contiguous().view(B, L, K)
    Z = torch.zeros((B, L, N), device=DEV)
    dfa.dfa_linear(merged, W, bias, Z, gate=gate, residual=res)
    torch.cuda.synchronize()
    _check(Y.t, X, W, bias, gate, res, "none", B, L, K, N)
    assert torch.equal(Y.t, Z), "the heads' layout changes no bit"
    assert Y.guards_intact()


@pytest.mark.parametrize("ytype", [BF16, F32])
@pytest.mark.parametrize("B,L,K,N", [(2, 1, 1152, 1152), (3, 21, 100, 33), (2, 301, 1152, 1152), (2, 4100, 576, 1920), (1, 12345, 640, 768)])
def test_residual_in_place(B, L, K, N, ytype):
    X, W, bias, gate, res = _inputs(B, L, K, N, ytype, "batch", 5)
    Y = torch.zeros((B, L, N), dtype=ytype, device=DEV)
    dfa.dfa_linear(X, W, bias, Y, gate=gate, residual=res)
    dfa.dfa_linear(X, W, bias, res, gate=gate, residual=res)
    torch.cuda.synchronize()
    assert torch.equal(res, Y)


@pytest.mark.parametrize("B,L,K,N", [(1, 3, 72, 64), (1, 40, 200, 96), (2, 300, 1096, 200), (1, 6000, 136, 1000), (1, 70, 77, 64)])
def test_non_finite_values_stay_in_their_row(B, L, K, N):
    """A token's NaN reaches that token alone, a weight row's that feature
    alone: nothing is read past the end of a row of K, not even times zero."""
    X, W, bias, _, _ = _inputs(B, L, K, N, BF16, "none", 17)
    want = torch.zeros((B, L, N), dtype=BF16, device=DEV)
    dfa.dfa_linear(X, W, bias, want)
    X[0, 1] = float("nan")
    W[5] = float("inf")
    got = torch.zeros_like(want)
    dfa.dfa_linear(X, W, bias, got)
    torch.cuda.synchronize()
    assert got[0, 1].isnan().all()
    keep = torch.ones((B, L), dtype=torch.bool, device=DEV)
    keep[0, 1] = False
    cols = torch.arange(N, device=DEV) != 5
    assert torch.equal(got[keep][:, cols], want[keep][:, cols])
    assert not got[keep][:, 5].isfinite().any()


def test_refused_shapes_and_types():
    X = torch.zeros((2, 4, 64), dtype=BF16, device=DEV)
    W, Y, v = torch.zeros((32, 64), dtype=BF16, device=DEV), torch.zeros((2, 4, 32), dtype=BF16, device=DEV), torch.zeros(32, device=DEV)
    with pytest.raises(ValueError, match="W"):
        dfa.dfa_linear(X, W.t(), v, Y)
    with pytest.raises(ValueError, match="X"):
        dfa.dfa_linear(X.float(), W, v, Y)
    with pytest.raises(ValueError, match="bias"):
        dfa.dfa_linear(X, W, v[:31], Y)
    with pytest.raises(ValueError, match="residual"):
        dfa.dfa_linear(X, W, v, Y, residual=Y.float())
    with pytest.raises(ValueError, match="gate"):
        dfa.dfa_linear(X, W, v, Y, gate=torch.zeros((4, 32), device=DEV))
    with pytest.raises(ValueError, match="Y"):
        dfa.dfa_linear(X, W, v, Y.view(8, 32))
    with pytest.raises(TypeError, match="Y"):
        dfa.dfa_linear(X, W, v, Y.half())
    with pytest.raises(dfa.DfaError, match="activation"):
        dfa.dfa_linear(X, W, v, Y, act=9)
    with pytest.raises(dfa.DfaError, match="head dim"):
        dfa.dfa_linear(torch.zeros((2, 2, 4, 32), dtype=BF16, device=DEV), W, v, Y)
