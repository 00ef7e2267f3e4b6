"""Norm, gate, residual scale, sum and norm in one call, and the gradients, against the 64-bit form and its derivative, within a count of
roundings: one element to the widest rows, odd widths, any alignment, with and without each optional argument; rows that are not finite;
graphs, streams, the same bits on every run."""
import math

import pytest
import torch

import decoder_ref as dr
from util import DT, TDT

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


class Case:
    def __init__(self, B, R, E, dtype, rms, seed=0, block=True, gate=True, bias=True, res=True, ds=True, shift=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.R, self.E, self.dtype, self.rms = B, R, E, dtype, rms

        def act(scale=1.0, mean=0.0):
            t = torch.empty(B * R * E + shift, dtype=TDT[dtype], device="cuda")[shift:].view(B, R, E)
            return t.copy_(torch.randn(B, R, E, generator=g) * scale + mean)
        n = lambda s, m=0.0: (torch.randn(B, E, generator=g) * s + m).cuda()
        self.x, self.dy = act(2.0, 0.5), act()
        self.f = act(1.0, 0.3) if block else None
        self.gate = act(2.0) if block and gate else None
        self.ds = act() if ds else None
        self.w1 = n(0.3, 1.0) if block else None
        self.b1 = n(0.3) if block and bias else None
        self.w2, self.b2 = n(0.3, 1.0), n(0.3) if bias else None
        self.res = (torch.rand(B, generator=g) + 0.3).cuda() if block and res else None
        like = lambda: torch.full_like(act(), 7.0)
        self.s, self.df = (like() if block else None for _ in range(2))
        self.dg = like() if self.gate is not None else None
        self.y, self.dx = like(), like()
        stat = lambda on=True: torch.empty(B * R, device="cuda") if on else None
        self.m1, self.i1, self.m2, self.i2 = stat(block and not rms), stat(block), stat(not rms), stat()
        vec = lambda on: torch.full((B, E), 7.0, device="cuda") if on else None
        self.dw1, self.db1, self.dw2, self.db2 = vec(block), vec(self.b1 is not None), vec(True), vec(bias)
        self.dres = torch.empty(B, device="cuda") if self.res is not None else None

    def fwd(self, hb, stream=None):
        hb.gated_residual_norm_fwd(self.B, self.R, self.E, DT[self.dtype], int(self.rms), self.x, self.f, self.gate, self.w1, self.b1, self.res,
                                   self.w2, self.b2, EPS, self.s, self.y, self.m1, self.i1, self.m2, self.i2, stream)

    def bwd(self, hb, ws=None, stream=None):
        if ws is None:
            ws = torch.empty(hb.gated_residual_norm_bwd_workspace_bytes(self.B, self.R, self.E), dtype=torch.uint8, device="cuda").fill_(255)
        hb.gated_residual_norm_bwd(self.B, self.R, self.E, DT[self.dtype], int(self.rms), self.x, self.f, self.gate, self.w1, self.b1, self.res,
                                   self.w2, self.m1, self.i1, self.m2, self.i2, self.ds, self.dy, self.dx, self.df, self.dg, self.dw1, self.db1,
                                   self.dw2, self.db2, self.dres, ws, stream)

    OUT = ("s", "y", "dx", "df", "dg", "dw1", "db1", "dw2", "db2", "dres")

    def check(self):
        h = lambda t: None if t is None else t.double().cpu()
        names = ("x", "f", "gate", "w1", "b1", "res", "w2", "b2")
        p = {n: h(getattr(self, n)) for n in names}
        q = {n: None if v is None else v.clone().requires_grad_() for n, v in p.items()}
        s, y = dr.gated_norm(self.rms, *[q[n] for n in names], EPS)
        ds, dy = h(self.ds), h(self.dy)
        loss = (y * dy).sum() + (0.0 if ds is None else (s * ds).sum())
        loss.backward()
        want = dict(s=s.detach(), y=y.detach(), **{"d" + {"gate": "g"}.get(n, n): v.grad for n, v in q.items() if v is not None})
        bound = dr.gated_norm_bounds(self.rms, *[p[n] for n in names], EPS, ds, dy)
        for n in self.OUT:
            t = getattr(self, n)
            if t is None:
                continue
            b = dr.stored(want[n], bound[n], self.dtype if t.dtype == torch.bfloat16 else "f32")
            bad = (t.double().cpu().view(want[n].shape) - want[n]).abs() - b
            assert float(bad.max()) <= 0, (n, float(bad.max()), float(want[n].abs().max()))


SIZES = [(1, 1, 8), (2, 3, 5), (3, 201, 330), (2, 70, 512), (1, 33, 520), (2, 17, 1024), (1, 9, 1500), (2, 5, 2048), (1, 6, 3001), (1, 4, 4096),
         (1, 3, 7777), (1, 2, 16384), (1, 3, 9001), (1, 3000, 24), (2, 203, 64), (1, 77, 65), (3, 45, 256), (2, 1000, 130), (1, 9, 257), (1, 30001, 16), (3, 5, 1), (1, 70, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_values_and_gradients(hb, dtype, rms, size):
    c = Case(*size, dtype, rms, seed=size[2], shift=size[2] % 3)
    c.fwd(hb)
    c.bwd(hb)
    c.check()


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("without", [("gate",), ("bias",), ("res",), ("ds",), ("block",), ("block", "ds", "bias"), ("gate", "bias", "res", "ds")])
def test_without(hb, rms, without):
    for dtype in ("f32", "bf16"):
        c = Case(2, 37, 260, dtype, rms, seed=5, **{w: False for w in without})
        c.fwd(hb)
        c.bwd(hb)
        c.check()


def test_constant_rows_and_eps(hb):
    """Rows of one value: the deviation is nothing and eps alone stands under the root."""
    c = Case(1, 4, 64, "f32", False, seed=1)
    c.f.fill_(3.0)
    c.fwd(hb)
    c.bwd(hb)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("R,E", [(40, 96), (9, 1500), (5, 5000), (3, 9001)])
def test_gates_far_open_and_far_closed(hb, dtype, rms, bias, R, E):
    """The gate's gradient keeps its digits on both sides: sigma' = h (1 - h) is e^-|g| / (1 + e^-|g|)^2, even."""
    c = Case(2, R, E, dtype, rms, seed=9, bias=bias)
    sides = torch.tensor([-60.0, -20, -17.5, -16, -12, -10, -8, -4, 4, 8, 10, 12, 16, 17.5, 20, 60], device="cuda")
    c.gate.copy_(sides[torch.randint(16, (2, R, E), generator=torch.Generator().manual_seed(1)).cuda()])
    c.fwd(hb)
    c.bwd(hb)
    c.check()
    h = lambda t: None if t is None else t.double().cpu()
    names = ("x", "f", "gate", "w1", "b1", "res", "w2", "b2")
    p = [h(getattr(c, n)) for n in names]
    x, f, g, w1, b1, res, w2, b2 = p
    b1 = torch.zeros_like(w1) if b1 is None else b1
    bound = dr.gated_norm_bounds(rms, *p, EPS, h(c.ds), h(c.dy))
    q = [None if t is None else t.clone().requires_grad_() for t in p]
    s, y = dr.gated_norm(rms, *q, EPS)
    ((y * h(c.dy)).sum() + (s * h(c.ds)).sum()).backward()
    e = torch.exp(-g.abs())
    slope = res[:, None, None] * e / (1 + e) ** 2
    # dG = slope ds u.  ds and u as counted for the other gradients; an exponential of 2 roundings, two quotients and four products: 16
    fc = f if rms else f - f.mean(-1, keepdim=True)
    i1 = 1 / torch.sqrt((fc * fc).mean(-1, keepdim=True) + EPS)
    fh = fc * i1
    u = fh * w1[:, None] + b1[:, None]
    eu = w1.abs()[:, None] * 60 * dr.U * (i1 * f.abs().amax(-1, keepdim=True) + 1) * (1 + fh.abs()) + 4 * dr.U * ((fh * w1[:, None]).abs() + b1.abs()[:, None])
    dsm = q[0].grad
    want = slope * dsm * u
    b = slope * (bound["dx"] * u.abs() + dsm.abs() * eu + 16 * dr.U * (dsm * u).abs())
    bad = (h(c.dg) - want).abs() - dr.stored(want, b, dtype)
    assert float(bad.max()) <= 0, (float(bad.max()), c.gate.flatten()[int(bad.argmax())])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [96, 1500, 5000, 9001])
def test_gates_without_end(hb, dtype, E):
    """Gates of plus and minus infinity are those of 200: open or shut, with a slope of nothing."""
    c, d = (Case(2, 5, E, dtype, False, seed=3) for _ in range(2))
    sign = torch.where(torch.rand(2, 5, E, generator=torch.Generator().manual_seed(2)) < 0.5, -1.0, 1.0).cuda()
    c.gate.copy_(sign * math.inf)
    d.gate.copy_(sign * 200.0)
    for x in (c, d):
        x.fwd(hb)
        x.bwd(hb)
    for n in c.OUT:
        assert torch.equal(getattr(c, n), getattr(d, n)) and bool(torch.isfinite(getattr(c, n)).all()), n
    assert not bool(c.dg.any())


def test_rows_that_are_not_finite(hb):
    for rms in (False, True):
        c = Case(2, 21, 100, "bf16", rms, seed=2)
        c.fwd(hb)
        c.bwd(hb)
        good = {n: getattr(c, n).clone() for n in ("s", "y", "dx", "df", "dg")}
        c.f[0, 3, 5], c.x[1, 7, 0], c.gate[0, 9, 2] = math.nan, math.inf, math.nan
        c.gate[1, 2, :] = -math.inf                               # a closed gate is no fault
        c.fwd(hb)
        c.bwd(hb)
        bad = torch.zeros(2, 21, dtype=torch.bool)
        bad[0, 3] = bad[1, 7] = bad[0, 9] = True
        keep = ~bad
        keep[1, 2] = False
        for n, v in good.items():
            assert torch.equal(getattr(c, n)[keep.cuda()], v[keep.cuda()]), n
        for n in ("y", "dx", "df"):
            assert bool((~torch.isfinite(getattr(c, n).float())).any(2)[bad.cuda()].all()), n
        assert torch.equal(c.s[1, 2], c.x[1, 2]) and bool(torch.isfinite(c.y[1, 2].float()).all()) and not bool(c.df[1, 2].any())


def test_in_place_gradient_and_graph(hb):
    c = Case(2, 150, 256, "bf16", True, seed=3)
    ws = torch.empty(hb.gated_residual_norm_bwd_workspace_bytes(2, 150, 256), dtype=torch.uint8, device="cuda")
    c.fwd(hb)
    c.bwd(hb, ws)
    want = {n: getattr(c, n).clone() for n in c.OUT if getattr(c, n) is not None}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.fwd(hb)
        c.bwd(hb, ws)
    for _ in range(3):
        for n in want:
            getattr(c, n).fill_(3.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for n, v in want.items():
            assert torch.equal(getattr(c, n), v), n
    c.dx = c.ds                                                   # the gradient in place of the one that came
    c.bwd(hb, ws)
    assert torch.equal(c.dx, want["dx"]) and torch.equal(c.df, want["df"])


def test_models_alone_and_together(hb):
    """A model's results are the same bits beside others, on another stream, and in two calls at once."""
    c = Case(3, 64, 96, "f32", False, seed=4)
    c.fwd(hb)
    other = torch.cuda.Stream()
    d = Case(3, 64, 96, "f32", False, seed=4)
    torch.cuda.synchronize()
    d.fwd(hb, other)
    c.bwd(hb)
    torch.cuda.synchronize()
    ws = torch.empty(hb.gated_residual_norm_bwd_workspace_bytes(3, 64, 96), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    d.bwd(hb, ws, other)
    torch.cuda.synchronize()
    for n in c.OUT:
        assert torch.equal(getattr(c, n), getattr(d, n)), n


def test_past_2_31_elements(hb):
    B, R, E = 1, 140000, 16384
    x = torch.zeros(B, R, E, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros_like(x)
    x[0, -2:] = torch.randn(2, E, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    w = torch.ones(1, E, device="cuda")
    inv = torch.empty(R, device="cuda")
    hb.gated_residual_norm_fwd(B, R, E, 1, 1, x, None, None, None, None, None, w, None, EPS, None, y, None, None, None, inv)
    want = dr.gated_norm(True, x[:, -2:].double().cpu(), None, None, None, None, None, w.double().cpu(), None, EPS)[1]
    # 60 roundings of fp32 and one of bf16
    assert float(((y[:, -2:].double().cpu() - want).abs() - (2.0 ** -8 + 120 * dr.U) * want.abs()).max()) <= 0
    assert not bool(y[0, -4:-2].any())


def test_millions_of_rows(hb):
    """Rows of 128 threads, more than 2^22 of them; the last ones, behind a long stretch of zeros."""
    R, E, n = 5000000, 600, 3
    g = torch.Generator().manual_seed(4)
    x, dy = (torch.zeros(1, R, E, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        t[0, -n:] = torch.randn(n, E, generator=g).bfloat16().cuda()
    y, dx = (torch.full_like(x, 7.0) for _ in range(2))
    w = (torch.randn(1, E, generator=g) * 0.3 + 1).cuda()
    inv, dw = torch.empty(R, device="cuda"), torch.empty(1, E, device="cuda")
    ws = torch.empty(hb.gated_residual_norm_bwd_workspace_bytes(1, R, E), dtype=torch.uint8, device="cuda")
    hb.gated_residual_norm_fwd(1, R, E, 1, 1, x, None, None, None, None, None, w, None, EPS, None, y, None, None, None, inv)
    hb.gated_residual_norm_bwd(1, R, E, 1, 1, x, None, None, None, None, None, w, None, None, None, inv, None, dy, dx, None, None, None, None, dw,
                               None, None, ws)
    h = lambda t: t[:, -n:].double().cpu()
    p = [h(x), None, None, None, None, None, w.double().cpu(), None]
    q = [None if t is None else t.clone().requires_grad_() for t in p]
    (dr.gated_norm(True, *q, EPS)[1] * h(dy)).sum().backward()
    bound = dr.gated_norm_bounds(True, *p, EPS, None, h(dy))
    want = dr.gated_norm(True, *p, EPS)[1]
    for got, v, b, t in ((h(y), want, bound["y"], "bf16"), (h(dx), q[0].grad, bound["dx"], "bf16"), (dw.double().cpu(), q[6].grad, bound["dw2"], "f32")):
        assert float(((got - v).abs() - dr.stored(v, b, t)).max()) <= 0
    assert not bool(y[0, :-n].any()) and not bool(dx[0, :-n].any())
