"""Layer norm and its gradients against their definitions in float64.

Bars, with u = 2^-24 the rounding of fp32.  A sum over C features is at most 32
additions in a lane, 6 across the wavefront, 8 across wavefronts, so its error
is at most 64 u times the sum of magnitudes, with room for the products:
  mean    64 u mean|x|
  rstd    64 u of itself (a mean that is off by 64 u mean|x| changes the
          variance by that squared, which is added)
  Y       what these do to xh and its factor, and one rounding to bf16 (2^-8)
  dX      64 u of each of its three terms' magnitudes, times rstd, and its rounding
  dw, db  a token's share is summed in at most `rows` + 64 steps (the rows of a
          wavefront, its workgroup, the splits): that many u times the sum of
          magnitudes
"""
import pytest
import torch

from paper_2406_08552_amd import dfa
from tests.test_gpu_parity import Guarded, say

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
U = 2.0 ** -24
EPS = 1e-6

# one token; widths below a wavefront, odd, a vector past a whole number, at the
# ends of what a wavefront and a workgroup hold; few and many tokens
SHAPES = [(1, 1, 1), (1, 1, 64), (2, 3, 7), (2, 5, 512), (3, 2, 513), (3, 57, 777), (1, 3, 1279), (2, 4, 1280), (2, 301, 1152),
          (1, 9, 1281), (1, 2, 2048), (2, 3, 2049), (1, 5, 4096), (1, 5, 4097), (2, 2, 16384), (1, 4500, 130), (9, 1000, 64),
          (1, 9000, 256), (2, 1100, 250), (1, 2100, 257), (2, 8500, 122)]


def _inputs(B, L, C, dtype, affine, seed, offset=0.0, slices=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    X = (r(B, L, C) * (1 + r(C).abs()) + offset).to(dtype)
    if affine == "none":
        w = b = None
    elif affine == "shared":
        w, b = r(C), r(C)
    else:
        m = r(B, 2 * C + 3) if slices else r(B, 2 * C)
        w, b = m[:, 1:C + 1], m[:, C + 2:2 * C + 2] if slices else m[:, C:]
    return g, X, w, b


def _rows64(v, B, C):
    return v.double().reshape(-1, 1, C)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("affine", ["none", "shared", "batch"])
@pytest.mark.parametrize("B,L,C", SHAPES)
def test_forward(B, L, C, dtype, affine):
    g, X, w, b = _inputs(B, L, C, dtype, affine, C + L, offset=3.0)
    say(f"layer_norm {B} {L} {C} {dtype} {affine}")
    Y, mean, rstd = Guarded((B, L, C), DEV), Guarded((B, L), DEV, torch.float32), Guarded((B, L), DEV, torch.float32)
    dfa.dfa_layer_norm(X, w, b, Y.t, mean.t, rstd.t, eps=EPS, weight_offset=1.0)
    bare = torch.zeros_like(Y.t)
    dfa.dfa_layer_norm(X, w, b, bare, eps=EPS, weight_offset=1.0)
    torch.cuda.synchronize()
    assert torch.equal(bare, Y.t)
    x = X.double()
    m = x.mean(-1, keepdim=True)
    rs = (((x - m) ** 2).mean(-1, keepdim=True) + EPS) ** -0.5
    xh = (x - m) * rs
    dm = 64 * U * x.abs().mean(-1, keepdim=True)
    dr = 64 * U + (dm * rs) ** 2
    wd = torch.ones((1, 1, 1), dtype=torch.float64, device=DEV) if w is None else _rows64(w, B, C) + 1.0
    bd = torch.zeros_like(wd) if b is None else _rows64(b, B, C)
    y = xh * wd + bd
    assert ((mean.t.double() - m[..., 0]).abs() <= dm[..., 0]).all()
    assert ((rstd.t.double() - rs[..., 0]).abs() <= dr[..., 0] * rs[..., 0]).all()
    bar = 2.0 ** -8 * y.abs() + wd.abs() * (dm * rs + (dr + 4 * U) * xh.abs()) * 1.01 + 2 * U * (xh.abs() * (wd.abs() + 1) + bd.abs())
    assert ((Y.t.double() - y).abs() <= bar).all(), float(((Y.t.double() - y).abs() - bar).max())
    assert Y.guards_intact() and mean.guards_intact() and rstd.guards_intact()


@pytest.mark.parametrize("groups", ["none", "shared", "batch"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,C", SHAPES)
def test_backward(B, L, C, dtype, groups):
    affine = {"none": "none", "shared": "shared", "batch": "batch"}[groups]
    g, X, w, _ = _inputs(B, L, C, dtype, affine, 7 * C + L)
    say(f"layer_norm_backward {B} {L} {C} {dtype} {groups}")
    dY = torch.randn((B, L, C), generator=g, device=DEV).to(torch.bfloat16)
    x = X.double()
    mean = x.mean(-1)
    rstd = (((x - mean[..., None]) ** 2).mean(-1) + EPS) ** -0.5
    mean, rstd = mean.float(), rstd.float()
    n = (B, C) if groups == "batch" else (C,)
    dX, dw, db = Guarded((B, L, C), DEV, dtype), Guarded(n, DEV, torch.float32), Guarded(n, DEV, torch.float32)
    nbytes = dfa.layer_norm_backward_workspace_bytes(B, L, C, B if groups == "batch" else 1)
    ws = torch.full((nbytes + 256,), 77, dtype=torch.uint8, device=DEV)
    args = (dY, X, w, mean, rstd)
    dfa.dfa_layer_norm_backward(*args, dX.t, dw.t, db.t, ws[:nbytes] if nbytes else None, weight_offset=1.0)
    again = [torch.zeros_like(t.t) for t in (dX, dw, db)]
    ws2 = torch.zeros_like(ws)
    dfa.dfa_layer_norm_backward(*args, *again, ws2[:nbytes] if nbytes else None, weight_offset=1.0)
    one = [torch.zeros_like(t.t) for t in (dX, dX, dw, db)]
    dfa.dfa_layer_norm_backward(*args, one[0], None, one[3], ws2, weight_offset=1.0)
    dfa.dfa_layer_norm_backward(*args, one[1], one[2], None, ws2, weight_offset=1.0)
    only = torch.zeros_like(dX.t)
    dfa.dfa_layer_norm_backward(*args, only, None, None, weight_offset=1.0)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 77).all()), "write behind the workspace"
    for got, want in ((again[0], dX.t), (again[1], dw.t), (again[2], db.t), (one[0], dX.t), (one[1], dX.t), (one[2], dw.t),
                      (one[3], db.t), (only, dX.t)):
        assert torch.equal(got, want)
    dy, md, rd = dY.double(), mean.double()[..., None], rstd.double()[..., None]
    xh = (x - md) * rd
    gd = dy if w is None else dy * (_rows64(w, B, C) + 1.0)
    # weight + offset is rounded once: u (|w| + 1) of the factor
    gu = gd.abs() + (0 if w is None else dy.abs() * (_rows64(w, B, C).abs() + 1))
    sx = (gd * xh).mean(-1, keepdim=True)
    dx = rd * (gd - gd.mean(-1, keepdim=True) - xh * sx)
    bar = rd * 64 * U * (gu + gu.mean(-1, keepdim=True) + xh.abs() * (gu * xh.abs()).mean(-1, keepdim=True))
    bar = bar + dx.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else U)
    assert ((dX.t.double() - dx).abs() <= bar).all(), float(((dX.t.double() - dx).abs() - bar).max())
    rows = max(4, -(-B * L // 512)) + 64
    dims = (1,) if groups == "batch" else (0, 1)
    for name, got, term in (("dweight", dw, dy * xh), ("dbias", db, dy)):
        off = (got.t.double() - term.sum(dims)).abs()
        assert (off <= (rows + 4) * U * term.abs().sum(dims)).all(), name
        assert got.guards_intact(), name
    assert dX.guards_intact()


def test_gradients_against_differences():
    """sum(dY * Y) in float64 moves with X, weight and bias as the gradients say."""
    B, L, C = 2, 3, 24
    g, X, w, b = _inputs(B, L, C, torch.float32, "batch", 5)
    dY = torch.randn((B, L, C), generator=g, device=DEV).to(torch.bfloat16)
    Y, mean, rstd = torch.empty_like(dY), torch.empty((B, L), device=DEV), torch.empty((B, L), device=DEV)
    dfa.dfa_layer_norm(X, w, b, Y, mean, rstd, eps=EPS)
    dX, dw, db = torch.empty_like(X), torch.empty((B, C), device=DEV), torch.empty((B, C), device=DEV)
    n = dfa.layer_norm_backward_workspace_bytes(B, L, C, B)
    dfa.dfa_layer_norm_backward(dY, X, w, mean, rstd, dX, dw, db, torch.empty(max(n, 1), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()

    def f(x, w, b):
        m = x.mean(-1, keepdim=True)
        xh = (x - m) * (((x - m) ** 2).mean(-1, keepdim=True) + EPS) ** -0.5
        return (dY.double() * (xh * w[:, None] + b[:, None])).sum()

    at = [X.double(), w.double(), b.double()]
    h = 1e-6
    for i, got in enumerate((dX, dw, db)):
        for k in range(0, at[i].numel(), 5):
            d = torch.zeros_like(at[i])
            d.view(-1)[k] = h
            hi, lo = ([t + d if j == i else t for j, t in enumerate(at)], [t - d if j == i else t for j, t in enumerate(at)])
            want = float((f(*hi) - f(*lo)) / (2 * h))
            # differences: h^2 times third derivatives and 2^-52 / h of the sum; the kernel: 64 u of terms of size 10
            assert abs(float(got.reshape(-1)[k]) - want) < 2e-4, (i, k)


def test_large_mean_and_constant_rows():
    """A mean a thousand times the spread; a constant row, whose variance is 0 and whose xh is 0."""
    C = 1152
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.randn((1, 3, C), generator=g, device=DEV) + 1000.0
    X[0, 1] = 0.1
    X[0, 2] = 0.0
    Y, mean, rstd = torch.empty((1, 3, C), dtype=torch.bfloat16, device=DEV), torch.empty((1, 3), device=DEV), torch.empty((1, 3), device=DEV)
    dfa.dfa_layer_norm(X, None, None, Y, mean, rstd, eps=EPS)
    torch.cuda.synchronize()
    x = X.double()[0, 0]
    xh = (x - x.mean()) / (x.var(correction=0) + EPS).sqrt()
    dm = 64 * U * 1010                       # mean of |x|, in units of the spread 1
    assert ((Y[0, 0].double() - xh).abs() <= 2.0 ** -8 * xh.abs() + 1.1 * (dm + (64 * U + dm * dm) * xh.abs())).all()
    # x - mean is at most 64 u 0.1, rstd at most eps^-1/2 = 1000
    assert (Y[0, 1].double().abs() <= 64 * U * 0.1 * 1000 * 1.01).all()
    assert not Y[0, 2].any() and float(mean[0, 2]) == 0 and abs(float(rstd[0, 2]) - 1000) < 1000 * 8 * U


def test_non_finite_values_stay_in_their_token():
    B, L, C = 2, 8, 777
    g, X, w, b = _inputs(B, L, C, torch.bfloat16, "shared", 3)
    want = torch.empty_like(X)
    dfa.dfa_layer_norm(X, w, b, want)
    X2 = X.clone()
    X2[0, 3, 700] = float("nan")
    X2[1, 7, 776] = float("inf")
    got = torch.empty_like(X)
    dfa.dfa_layer_norm(X2, w, b, got)
    torch.cuda.synchronize()
    bad = torch.zeros((B, L), dtype=torch.bool, device=DEV)
    bad[0, 3] = bad[1, 7] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], want[~bad])


def test_refused_shapes_and_types():
    X = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=DEV)
    Y, v, s = torch.zeros_like(X), torch.zeros(64, device=DEV), torch.zeros((2, 4), device=DEV)
    for bad in (torch.zeros(63, device=DEV), torch.zeros((3, 64), device=DEV), torch.zeros((2, 128), device=DEV)[:, ::2]):
        with pytest.raises(ValueError, match="weight"):
            dfa.dfa_layer_norm(X, bad, None, Y)
    with pytest.raises(TypeError, match="weight"):
        dfa.dfa_layer_norm(X, v.bfloat16(), None, Y)
    with pytest.raises(ValueError, match="Y"):
        dfa.dfa_layer_norm(X, v, v, Y.float())
    with pytest.raises(ValueError, match="X"):
        dfa.dfa_layer_norm(torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=DEV)[..., ::2], v, v, Y)
    with pytest.raises(dfa.DfaError, match="overlaps"):
        dfa.dfa_layer_norm(X, v, v, X)
    with pytest.raises(ValueError, match="dbias"):
        dfa.dfa_layer_norm_backward(X, X, v, s, s, Y, v, torch.zeros((2, 64), device=DEV))
    big = torch.zeros((2, 600, 64), dtype=torch.bfloat16, device=DEV)
    t = torch.zeros((2, 600), device=DEV)
    with pytest.raises(dfa.DfaError, match="workspace"):
        dfa.dfa_layer_norm_backward(big, big, v, t, t, torch.zeros_like(big), v.clone(), None)
