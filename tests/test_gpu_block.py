"""Layer norm, rotary positions, linear layers and the attention path run
together, as a transformer block uses them: stage by stage against float64,
replayed from a HIP graph, on other streams, and through both marshalling
paths; tensors of more than 2^31 elements; tile routes of the linear layer."""
import math

import pytest
import torch

from paper_2406_08552_amd import dfa
from tests.test_gpu_linear import _check as check_linear
from tests.test_gpu_linear import _inputs as linear_inputs
from tests.test_gpu_parity import Guarded, say

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


class _Sub(torch.Tensor):
    pass


class Block:
    """One block of a diffusion transformer on a residual stream of `stream`
    type, updated in place: modulated layer norms, gated branches, a grid of
    tokens with rotary positions, full or window attention."""

    def __init__(self, B, H, grid, d, stream, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.B, self.H, self.d, self.L, self.C = B, H, d, math.prod(grid), H * d
        B, L, C = B, self.L, self.C
        self.x0 = r(B, L, C).to(stream)
        self.x = self.x0.clone()
        self.t = r(B, 1, C).to(BF16)                       # the time step's embedding, a token per entry
        self.Wm, self.bm = (r(6 * C, C) * 0.3 * C ** -0.5).to(BF16), r(6 * C) * 0.1
        self.Wqkv, self.bqkv = (r(3 * C, C) * C ** -0.5).to(BF16), r(3 * C) * 0.1
        self.Wo, self.bo = (r(C, C) * C ** -0.5).to(BF16), r(C) * 0.1
        self.W1, self.b1 = (r(4 * C, C) * C ** -0.5).to(BF16), r(4 * C) * 0.1
        self.W2, self.b2 = (r(C, 4 * C) * (4 * C) ** -0.5).to(BF16), r(C) * 0.1
        self.pos = torch.stack(torch.meshgrid(*[torch.arange(n, device=DEV, dtype=F32) for n in grid], indexing="ij"), -1)
        self.pos = self.pos.reshape(L, len(grid)).contiguous()
        self.sections = [2 * (d // (2 * len(grid)))] * len(grid)
        e = lambda *s, dt=BF16: torch.empty(s, dtype=dt, device=DEV)  # noqa: E731
        self.mod = e(B, 1, 6 * C, dt=F32)
        self.n1, self.n2, self.mid = e(B, L, C), e(B, L, C), e(B, L, 4 * C)
        self.Q, self.K, self.V, self.O = (e(B, H, L, d) for _ in range(4))
        self.x1 = torch.empty_like(self.x)

    def run(self, keep=None, stream=None):
        m = self.mod.view(self.B, 6, self.C)
        kw = {} if stream is None else {"stream": stream}
        dfa.dfa_linear(self.t, self.Wm, self.bm, self.mod, **kw)
        dfa.dfa_layer_norm(self.x, m[:, 1], m[:, 0], self.n1, eps=EPS, weight_offset=1.0, **kw)
        dfa.dfa_qkv_proj(self.n1, self.Wqkv, self.bqkv, self.Q, self.K, self.V, **kw)
        if keep is not None:
            keep["q"], keep["k"] = self.Q.clone(), self.K.clone()
        dfa.dfa_rope(self.Q, self.K, self.Q, self.K, self.pos, self.sections, **kw)
        dfa.dfa_attn_full(self.Q, self.K, self.V, self.O, **kw)
        dfa.dfa_linear(self.O, self.Wo, self.bo, self.x1, gate=m[:, 2], residual=self.x, **kw)
        dfa.dfa_layer_norm(self.x1, m[:, 4], m[:, 3], self.n2, eps=EPS, weight_offset=1.0, **kw)
        dfa.dfa_linear(self.n2, self.W1, self.b1, self.mid, act=dfa.ACT_GELU_TANH, **kw)
        if keep is not None:
            keep["x1"] = self.x1.clone()
        dfa.dfa_linear(self.mid, self.W2, self.b2, self.x1, gate=m[:, 5], residual=self.x1, **kw)   # in place


def _norm64(x, scale, shift):
    x = x.double()
    x = x - x.mean(-1, keepdim=True)
    x = x * ((x * x).mean(-1, keepdim=True) + EPS) ** -0.5
    return x * (1 + scale.double()[:, None]) + shift.double()[:, None]


@pytest.mark.parametrize("B,H,grid,d,stream", [(2, 16, (5, 7, 9), 72, F32), (3, 2, (11, 13), 64, BF16), (1, 16, (1, 1), 72, F32),
                                               (2, 16, (32, 32), 72, BF16)])
def test_block_stage_by_stage(B, H, grid, d, stream):
    """Each stage against float64 of the stage's own inputs as the library left
    them, with the stages' own bars (those of their tests)."""
    b = Block(B, H, grid, d, stream)
    L, C = b.L, b.C
    keep = {}
    say(f"block {B} {H} {grid} {d} {stream}")
    b.run(keep)
    torch.cuda.synchronize()
    m = b.mod.view(B, 6, C)
    check_linear(b.mod, b.t, b.Wm, b.bm, None, None, "none", B, 1, C, 6 * C)
    for got, x, scale, shift in ((b.n1, b.x, m[:, 1], m[:, 0]), (b.n2, keep["x1"], m[:, 4], m[:, 3])):
        want = _norm64(x, scale, shift)
        # one rounding, and 2^-16 of factors and offsets of size one to a few, from fp32 statistics
        assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * (want.abs() + 4)).all()
    cos, sin = [], []
    for a, n in enumerate(b.sections):
        t = b.pos[:, a:a + 1].double() * 10000.0 ** (-torch.arange(0, n, 2, device=DEV, dtype=torch.float64) / n)
        cos.append(torch.cos(t))
        sin.append(torch.sin(t))
    for got, x in ((b.Q, keep["q"].double()), (b.K, keep["k"].double())):
        o = 0
        for a, n in enumerate(b.sections):
            u, v = x[..., o:o + n // 2], x[..., o + n // 2:o + n]
            for part, want in ((got[..., o:o + n // 2], u * cos[a] - v * sin[a]), (got[..., o + n // 2:o + n], u * sin[a] + v * cos[a])):
                assert ((part.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * (u.abs() + v.abs())).all()
            o += n
    check_linear(keep["x1"], b.O, b.Wo, b.bo, m[:, 2], b.x, "none", B, L, C, C)
    check_linear(b.mid, b.n2, b.W1, b.b1, None, None, "gelu_tanh", B, L, C, 4 * C)
    check_linear(b.x1, b.mid, b.W2, b.b2, m[:, 5], keep["x1"], "none", B, L, 4 * C, C)
    assert torch.equal(b.x, b.x0), "the stream that the block reads stays"


def test_block_in_a_graph_and_on_another_stream():
    b = Block(2, 16, (6, 8), 72, F32, seed=3)
    b.run()
    torch.cuda.synchronize()
    want = b.x1.clone()
    side = torch.cuda.Stream()
    b.x1.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b.run()
    side.synchronize()
    assert torch.equal(b.x1, want), "the current stream"
    b.x1.zero_()
    torch.cuda.synchronize()
    b.run(stream=side)                      # explicit: the general marshalling path
    side.synchronize()
    assert torch.equal(b.x1, want), "an explicit stream"
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.run()
    for i in range(3):
        b.x1.zero_()
        for t in (b.n1, b.n2, b.mid, b.mod, b.O):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.x1, want), f"replay {i}"
        b.run()                             # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(b.x1, want)
    b.x.copy_(b.x0 * 0.5)                   # a replay reads what its inputs hold now
    graph.replay()
    torch.cuda.synchronize()
    replayed = b.x1.clone()
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(b.x1, replayed) and not torch.equal(replayed, want)


def test_gradients_in_a_graph():
    """A captured backward pass with its own workspace beside an eager one."""
    B, L, C = 2, 700, 1152
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    X, dY = torch.randn((B, L, C), generator=g, device=DEV), torch.randn((B, L, C), generator=g, device=DEV).to(BF16)
    w = torch.randn((B, C), generator=g, device=DEV)
    Y, mean, rstd = torch.empty_like(dY), torch.empty((B, L), device=DEV), torch.empty((B, L), device=DEV)
    out = [(torch.empty_like(X), torch.empty((B, C), device=DEV), torch.empty((B, C), device=DEV)) for _ in range(2)]
    n = dfa.layer_norm_backward_workspace_bytes(B, L, C, B)
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]

    def step(i):
        dfa.dfa_layer_norm(X, w, None, Y, mean, rstd, eps=EPS)
        dfa.dfa_layer_norm_backward(dY, X, w, mean, rstd, *out[i], ws[i])

    step(0)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(1)
    for _ in range(3):
        for t in (*out[1], ws[1].view(torch.int32)):
            t.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*out))
        step(0)
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Calls on two streams share nothing but their inputs."""
    a, b = (Block(1, 16, (30, 20), 72, F32, seed=s) for s in (1, 2))
    for blk in (a, b):
        blk.run()
    torch.cuda.synchronize()
    want = [blk.x1.clone() for blk in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for blk in (a, b):
        blk.x1.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, blk in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                blk.run()
    torch.cuda.synchronize()
    assert torch.equal(a.x1, want[0]) and torch.equal(b.x1, want[1])


def test_native_and_general_marshalling_agree(monkeypatch):
    native, made = dfa._native(), []

    class Spy:
        def __getattr__(self, name):
            return lambda *a: made.append((name, getattr(native, name)(*a))) or made[-1][1]

    monkeypatch.setattr(dfa, "_NATIVE", Spy())
    b = Block(2, 2, (9, 5), 64, BF16)
    names = {"layer_norm", "linear", "rope"}
    outs = []
    for stream in (None, torch.cuda.current_stream()):
        made.clear()
        b.run(stream=stream)
        torch.cuda.synchronize()
        outs.append(b.x1.clone())
        calls = [s for n, s in made if n in names]
        assert calls == ([0] * 7 if stream is None else []), made
    assert torch.equal(*outs)
    # sections in a tuple and a module's parameter are ordinary; a call of another
    # tensor class is declined, and the general path makes it
    made.clear()
    dfa.dfa_rope(b.Q, None, b.Q, None, b.pos, tuple(b.sections))
    dfa.dfa_layer_norm(torch.nn.Parameter(b.x), None, None, b.n1)
    b.n2.zero_()
    dfa.dfa_layer_norm(b.x.as_subclass(_Sub), None, None, b.n2)
    torch.cuda.synchronize()
    assert [s for _, s in made] == [0, 0, -1] and torch.equal(b.n1, b.n2)
    for stream in (None, torch.cuda.current_stream()):   # the same errors on both
        with pytest.raises(dfa.DfaError, match="overlaps"):
            dfa.dfa_layer_norm(b.n1, None, None, b.n1, stream=stream)
        with pytest.raises(dfa.DfaError, match="activation"):
            dfa.dfa_linear(b.n1, b.Wo, b.bo, b.n2, act=7, stream=stream)
        with pytest.raises(dfa.DfaError, match="exceed"):
            dfa.dfa_rope(b.Q, None, b.Q, None, b.pos, [64, 64], stream=stream)


def test_another_device_is_refused(monkeypatch):
    """Tensors on another device than the current one (pretended: the current
    device is made to look like another)."""
    x = torch.zeros((1, 4, 64), dtype=BF16, device=DEV)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="current device is cuda:1"):
        dfa.dfa_layer_norm(x, None, None, torch.zeros_like(x), stream=side)


# the routes of the linear layer: every tile, with a ragged last tile of either kind
def _route(B, L, K, N, heads=1, ytype=F32):
    M = B * L
    t = lambda f, k: -(-N // f) * -(-M // k)  # noqa: E731
    narrow = K % 8 != 0 or N <= 4096
    if M <= 4 or (narrow and M <= 16):
        return "few 16"
    if t(16, 16) <= 256 and (K % 8 or t(16, 16) * K <= 256 * 2304):
        return "few 16"
    if narrow and M <= 32 and (K % 8 or K <= 2304):
        return "few 32"
    if K % 8 and t(16, 32) <= 512:
        return "few 32"
    if K % 8:
        return "any 64" if t(128, 128) <= 128 else "any 128"
    if t(64, 64) <= 512:
        return "64 ring"
    n = t(128, 128)
    if n <= 256:
        return "128 ring"
    c128 = 100 * (n // 512) + (0 if n % 512 == 0 else 65 if n % 512 <= 256 else 100)
    c192, r256 = 138 * -(-t(192, 256) // 256), -(-t(256, 256) // 256)
    if heads == 1 and K % 128 == 0 and 176 * r256 + ((32000 if ytype == F32 else 6000) // K if r256 == 1 else 0) < min(c128, c192):
        return "256"
    return "128" if c128 <= c192 else "192"


@pytest.mark.parametrize("B,L,K,N,heads,route", [
    (1, 4, 1152, 6912, 1, "few 16"), (2, 8, 72, 40, 1, "few 16"), (2, 8, 77, 40, 1, "few 16"), (2, 15, 2304, 100, 1, "few 16"),
    (2, 16, 9, 5000, 1, "few 32"), (1, 32, 5000, 64, 1, "few 16"), (1, 5, 1152, 6912, 1, "64 ring"), (2, 150, 136, 515, 1, "64 ring"),
    (2, 1100, 128, 1030, 1, "128 ring"), (2, 1100, 1000, 1030, 1, "128 ring"), (3, 100, 999, 333, 1, "few 32"), (1, 3000, 129, 901, 1, "any 128"),
    (2, 6000, 128, 1100, 1, "128"), (12, 1000, 328, 1099, 1, "128"), (1, 8200, 128, 1160, 1, "192"), (1, 8200, 136, 1153, 1, "192"),
    (1, 16100, 384, 2041, 1, "256"), (1, 16128, 128, 2048, 1, "256"), (2, 1100, 128, 1030, 2, "128 ring"), (12, 1000, 320, 1100, 5, "128"),
    (3, 2700, 192, 1160, 3, "192"), (1, 8200, 1152, 1153, 16, "192"), (2, 150, 216, 515, 3, "64 ring"),
    (1, 1790, 136, 1150, 1, "64 ring"), (3, 596, 216, 1150, 3, "64 ring"), (1, 1793, 136, 1153, 1, "128 ring"),
    (1, 30, 2304, 4000, 1, "few 32"), (3, 100, 999, 1333, 1, "any 64"), (1, 285, 2017, 17, 1, "few 16"),
    (2, 301, 1152, 32, 1, "few 16"), (1, 64, 1001, 1153, 1, "few 32"), (1, 9000, 2062, 16, 1, "few 32"),
    (1, 130, 1152, 200, 16, "few 16"), (1, 5900, 2432, 2300, 1, "256")])
def test_linear_routes(B, L, K, N, heads, route):
    assert _route(B, L, K, N, heads) == route, "not the route this case is for"
    for ytype in (BF16, F32):
        X, W, bias, gate, res = linear_inputs(B, L, K, N, ytype, "batch", 3 * K + N, heads=heads)
        say(f"linear route {route} {B} {L} {K} {N} heads={heads} {ytype}")
        Y = Guarded((B, L, N), DEV, ytype)
        dfa.dfa_linear(X, W, bias, Y.t, act=dfa.ACT_SILU, gate=gate, residual=res)
        torch.cuda.synchronize()
        check_linear(Y.t, X, W, bias, gate, res, "silu", B, L, K, N)
        assert Y.guards_intact()


def test_more_than_two_to_the_31_elements():
    """Offsets that 32 bits do not hold, checked on the first and last tokens."""
    C, L = 1032, (1 << 21) + 77             # 2.16e9 elements
    ends = torch.tensor([0, 1, L // 2, L - 2, L - 1], device=DEV)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.empty((1, L, C), dtype=BF16, device=DEV)
    row = torch.randn((1 << 12, C), generator=g, device=DEV).to(BF16)
    for i in range(0, L, 1 << 12):
        n = min(1 << 12, L - i)
        X[0, i:i + n] = row[:n] * (1 + (i >> 12) % 5)
    w, b = torch.randn(C, generator=g, device=DEV), torch.randn(C, generator=g, device=DEV)
    Y, mean, rstd = torch.empty_like(X), torch.empty((1, L), device=DEV), torch.empty((1, L), device=DEV)
    say("layer norm of 2^31 elements")
    dfa.dfa_layer_norm(X, w, b, Y, mean, rstd, eps=EPS)
    torch.cuda.synchronize()
    few = X[:, ends].contiguous()
    y = torch.empty_like(few)
    dfa.dfa_layer_norm(few, w, b, y, eps=EPS)
    assert torch.equal(Y[:, ends], y)
    dX, dw = torch.empty_like(X), torch.empty(C, device=DEV)
    n = dfa.layer_norm_backward_workspace_bytes(1, L, C, 1)
    say("gradients of 2^31 elements")
    dfa.dfa_layer_norm_backward(Y, X, w, mean, rstd, dX, dw, None, torch.empty(n, dtype=torch.uint8, device=DEV))
    dx = torch.empty_like(few)
    dfa.dfa_layer_norm_backward(y, few, w, mean[:, ends].contiguous(), rstd[:, ends].contiguous(), dx, None, None)
    torch.cuda.synchronize()
    assert torch.equal(dX[:, ends], dx)
    del dX
    W = (torch.randn((1032, C), generator=g, device=DEV) * C ** -0.5).to(BF16)
    say("linear layer of 2^31 outputs")
    dfa.dfa_linear(X, W, None, Y, residual=Y)
    torch.cuda.synchronize()
    z = few.double()[0] @ W.double().t().contiguous() + y.double()[0]
    off = (C / 16 + 32) * 2.0 ** -23 * (few.double().abs()[0] @ W.double().abs().t().contiguous()) + 2.0 ** -8 * z.abs() + 2.0 ** -20 * z.abs()
    assert ((Y[0, ends].double() - z).abs() <= off).all()
    del Y
    B, H, d = 1, 172, 6                      # the same memory as heads: 172 x 2^21 tokens x 6
    Q = X.view(-1)[: B * H * L * d].view(B, H, L, d)
    pos = torch.arange(2 * L, device=DEV, dtype=F32).view(L, 2) % 1009
    at = [Q[:, h:h + 1, ends].contiguous() for h in (0, H - 1)]
    say("rotation of 2^31 elements")
    dfa.dfa_rope(Q, None, Q, None, pos, [2, 4])
    for h, q in zip((0, H - 1), at):
        dfa.dfa_rope(q, None, q, None, pos[ends].contiguous(), [2, 4])
        torch.cuda.synchronize()
        assert torch.equal(Q[:, h:h + 1, ends], q)
