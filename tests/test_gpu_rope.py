"""Rotary positions against their definition in float64.

Bar: sine and cosine of a fraction of a turn, reduced in fp64 and rounded to
fp32, are off by at most 2^-22, each product and the sum by 2^-24 of
themselves: 2^-21 (|x| + |y|); and one rounding to bf16, 2^-8.  Frequencies are
products of up to 128 factors in fp64: 2^-46 of an angle."""
import math

import pytest
import torch

from paper_2406_08552_amd import dfa
from tests.test_gpu_parity import Guarded, say

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def _ref(x, pos, sections, base, interleaved, inverse):
    """x [B, H, L, d] float64, pos [L, A] or [B, L, A]; the rotated values and the bar."""
    y, mag, o = x.clone(), torch.zeros_like(x), 0
    pos = pos.double()
    pos = pos[None] if pos.dim() == 2 else pos
    ang = 0.0
    for a, n in enumerate(sections):
        i = torch.arange(n // 2, device=x.device)
        f = base ** (-2.0 * i.double() / n)
        t = (pos[..., a:a + 1] * f)[:, None] * (-1 if inverse else 1)
        ang = max(ang, float(t.abs().max()))
        p, q = (o + 2 * i, o + 2 * i + 1) if interleaved else (o + i, o + n // 2 + i)
        u, v = x[..., p], x[..., q]
        y[..., p], y[..., q] = u * torch.cos(t) - v * torch.sin(t), u * torch.sin(t) + v * torch.cos(t)
        mag[..., p] = mag[..., q] = u.abs() + v.abs()
        o += n
    return y, mag * (2.0 ** -21 + ang * 2.0 ** -45) + 2.0 ** -8 * y.abs()


# (B, Hq, Hk, L, d, sections): every width of a lane's access in both orders,
# dims that stay, one to four axes, one token, fewer key heads, odd head counts
SHAPES = [(1, 1, 1, 1, 2, [2]), (2, 3, 1, 5, 18, [6, 12]), (1, 2, 2, 77, 20, [4, 8]), (2, 16, 16, 256, 72, [36, 36]), (1, 6, 3, 100, 64, [64]),
          (2, 4, 4, 405, 72, [24, 24, 24]), (1, 5, 2, 33, 72, [8, 12, 20, 32]), (1, 12, 1, 300, 128, [16, 56, 56]), (3, 7, 7, 50, 96, [32, 32, 32]),
          (1, 2, 1, 19, 256, [256]), (2, 3, 2, 65, 254, [2, 84]), (40, 1, 1, 3, 48, [48]), (1, 16, 16, 4100, 64, [32, 32]), (1, 33, 9, 130, 80, [16, 32])]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,Hq,Hk,L,d,sections", SHAPES)
def test_rotation(B, Hq, Hk, L, d, sections, interleaved):
    g = torch.Generator(device="cuda")
    g.manual_seed(L + d)
    Q, K = (torch.randn((B, h, L, d), generator=g, device=DEV).to(torch.bfloat16) for h in (Hq, Hk))
    A = len(sections)
    whole = torch.randint(0, 20000, (L, A), generator=g, device=DEV).float()
    parts = torch.rand((B, L, A), generator=g, device=DEV) * 100 - 50
    for pos, inverse in ((whole, False), (parts, True)):
        say(f"rope {B} {Hq} {Hk} {L} {d} {sections} interleaved={interleaved} inverse={inverse}")
        Qo, Ko = Guarded(Q.shape, DEV), Guarded(K.shape, DEV)
        dfa.dfa_rope(Q, K, Qo.t, Ko.t, pos, sections, base=10000.0, interleaved=interleaved, inverse=inverse)
        alone, q, k = torch.zeros_like(Q), Q.clone(), K.clone()
        dfa.dfa_rope(Q, None, alone, None, pos, sections, base=10000.0, interleaved=interleaved, inverse=inverse)
        dfa.dfa_rope(q, k, q, k, pos, sections, base=10000.0, interleaved=interleaved, inverse=inverse)
        torch.cuda.synchronize()
        for x, y in ((Q, Qo), (K, Ko)):
            want, bar = _ref(x.double(), pos, sections, 10000.0, interleaved, inverse)
            err = (y.t.double() - want).abs()
            assert (err <= bar).all(), float((err - bar).max())
            n = sum(sections)
            assert torch.equal(y.t[..., n:], x[..., n:]), "the dims behind the sections stay"
            assert y.guards_intact()
        assert torch.equal(alone, Qo.t) and torch.equal(q, Qo.t) and torch.equal(k, Ko.t)


def test_position_zero_is_the_identity():
    Q = torch.randn((2, 3, 10, 72), device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(Q)
    dfa.dfa_rope(Q, None, out, None, torch.zeros((10, 3), device=DEV), [24, 24, 24])
    assert torch.equal(out, Q)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_other_positions(interleaved):
    """Positions up to 2^24 (whole in fp32) and bases from 1 to 1e6."""
    L, d, sections = 64, 64, [16, 48]
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    Q = torch.randn((1, 2, L, d), generator=g, device=DEV).to(torch.bfloat16)
    pos = (2.0 ** torch.linspace(0, 24, L, device=DEV)).floor()[:, None] * torch.tensor([1.0, -1.0], device=DEV)
    for base in (1.0, 2.5, 256.0, 1e6):
        out = torch.zeros_like(Q)
        dfa.dfa_rope(Q, None, out, None, pos, sections, base=base, interleaved=interleaved)
        torch.cuda.synchronize()
        want, bar = _ref(Q.double(), pos, sections, base, interleaved, False)
        assert ((out.double() - want).abs() <= bar).all(), base


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    """<rope(x), g> = <x, inverse(g)>: the inverse is the transpose."""
    L, d, sections = 50, 72, [24, 24, 24]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    x, gr = (torch.randn((1, 2, L, d), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    pos = torch.rand((L, 3), generator=gen, device=DEV) * 30
    y, gx = torch.zeros_like(x), torch.zeros_like(x)
    dfa.dfa_rope(x, None, y, None, pos, sections, interleaved=interleaved)
    dfa.dfa_rope(gr, None, gx, None, pos, sections, interleaved=interleaved, inverse=True)
    torch.cuda.synchronize()
    a, b = y.double() * gr.double(), x.double() * gx.double()
    # each side's values are rounded to bf16 once: 2^-8 of every product, and the fp32 arithmetic
    bar = (2.0 ** -8 + 2.0 ** -20) * (a.abs().sum() + b.abs().sum() + (x.double().abs() * gr.double().abs()).sum() * 2.0 ** -12)
    assert abs(float(a.sum() - b.sum())) <= float(bar)
    h = 1e-6                                     # and by differences of the definition, pair by pair
    for k in (0, 7, 12, 40, 71):
        dx = torch.zeros_like(x.double())
        dx[0, 1, 9, k] = h
        f = lambda v: float((_ref(v, pos, sections, 1e4, interleaved, False)[0] * gr.double()).sum())  # noqa: E731
        want = (f(x.double() + dx) - f(x.double() - dx)) / (2 * h)
        assert abs(float(gx[0, 1, 9, k]) - want) <= 2.0 ** -8 * abs(want) + 1e-5


def test_non_finite_positions_and_values_stay_in_their_pairs():
    L, d = 8, 64
    Q = torch.randn((1, 2, L, d), device=DEV).to(torch.bfloat16)
    pos = torch.arange(2 * L, device=DEV).float().view(L, 2)
    want, got = torch.zeros_like(Q), torch.zeros_like(Q)
    dfa.dfa_rope(Q, None, want, None, pos, [16, 16])
    pos[3, 1] = math.nan
    Q2 = Q.clone()
    Q2[0, 1, 5, 40] = math.inf                   # behind the sections: copied as it is
    Q2[0, 0, 6, 63] = math.nan
    dfa.dfa_rope(Q2, None, got, None, pos, [16, 16])
    torch.cuda.synchronize()
    assert got[0, :, 3, 16:32].isnan().all()
    assert float(got[0, 1, 5, 40]) == math.inf and got[0, 0, 6, 63].isnan()
    same = torch.ones_like(got, dtype=torch.bool)
    same[0, :, 3, 16:32] = False
    same[0, 1, 5, 40] = same[0, 0, 6, 63] = False
    assert torch.equal(got[same], want[same])


def test_refused_shapes_and_types():
    Q = torch.zeros((2, 4, 8, 64), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros((8, 2), device=DEV)
    for bad in (torch.zeros((7, 2), device=DEV), torch.zeros((8, 3), device=DEV), pos.double(), torch.zeros((3, 8, 2), device=DEV),
                torch.zeros((2, 8), device=DEV).t()):
        with pytest.raises(ValueError, match="pos"):
            dfa.dfa_rope(Q, None, Q, None, bad, [8, 8])
    with pytest.raises(ValueError, match="Q"):
        dfa.dfa_rope(Q.transpose(1, 2), None, Q.clone(), None, torch.zeros((4, 2), device=DEV), [8, 8])
    with pytest.raises(ValueError, match="K"):
        dfa.dfa_rope(Q, Q[:1], Q, Q[:1], pos, [8, 8])
    with pytest.raises(dfa.DfaError, match="even"):
        dfa.dfa_rope(Q, None, Q, None, pos, [8, 9])
