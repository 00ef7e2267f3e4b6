"""The operators of a decoder layer with a recurrent memory as they are used: a norm in front, projections, rotary positions on queries and keys,
linear attention with grouped heads, dropout by counter, and the gate, residual sum and norm behind -- forward and backward, eager and as a replayed
graph, against autograd in 64 bits; and a prompt followed by single tokens against the same layer over whole sequences.

Tolerance: every operator of the chain holds 1e-5 (fp32) and 2e-2 (bf16, which rounds each stored tensor by 2^-8) of its output's largest entry on
its own; a gradient at the bottom has passed the nine forward and the ten backward calls, whose errors add: 19e-5 of the largest entry in fp32.  In
bf16 19 roundings of 2^-8 in a random walk and the three products' inner ones give 2^-8 sqrt(19 + 6) = 2.0e-2 in the 2-norm; it is held to three times
that.  The residual scale's gradient is one sum of terms of both signs, held to its terms' 2-norm."""
import math

import numpy as np
import pytest
import torch

import decoder_ref as dr
from util import DT, TDT

pytestmark = pytest.mark.gpu

B, E, Hq, Hkv, d, PAIRS, EPS = 2, 48, 4, 2, 12, 5, 1e-5
W = (Hq + 2 * Hkv) * d
LENGTHS = [[17, 70, 0, 9, 133, 1], [5, 24, 120, 20, 2, 8]]
BEHIND, SITE, DROP = 6, 3, (0.1, 0.4)
SEED = (0x0123456789abcdef, 77)
TOL = {"f32": 19e-5, "bf16": 6.0e-2}


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def parameters(dtype):
    g = torch.Generator().manual_seed(11)
    n = lambda *s: torch.randn(*s, generator=g)
    p = dict(inw=n(B, E, W) / math.sqrt(E), inb=n(B, W) * 0.1, gw=n(B, E, E) / math.sqrt(E), gb=n(B, E) * 0.1, outw=n(B, Hq * d, E) / math.sqrt(Hq * d),
             outb=n(B, E) * 0.1)
    p = {k: v.to(TDT[dtype]) for k, v in p.items()}
    for k in ("n0w", "n1w", "n2w"):
        p[k] = 1 + 0.1 * n(B, E)
    p["n1b"], p["n2b"] = 0.1 * n(B, E), 0.1 * n(B, E)
    p["res"] = torch.rand(B, generator=g) + 0.5
    return p


def common():
    freq = (100.0 ** (-torch.arange(PAIRS).double() / PAIRS)).float().expand(B, -1).contiguous()
    return freq, torch.zeros(PAIRS, dtype=torch.int32), torch.tensor([[-0.02, -0.3], [0.0, -1.5]])


def oracle(rms, p, x, off, keep):
    """The layer over packed rows; keep: the factor of dropout for each entry, or None.  (x, parameters, S, Y)"""
    p = {k: v.double().requires_grad_() for k, v in p.items()}
    x = x.double().requires_grad_()
    R = x.shape[1]
    freq, axis, ld = common()
    rows, place = dr.inside(off, R)
    bias = lambda k: None if rms else p[k]
    _, y0 = dr.gated_norm(rms, x, None, None, None, None, None, p["n0w"], None, EPS)
    qkv = (y0 @ p["inw"] + p["inb"][:, None]).view(B, R, Hq + 2 * Hkv, d)
    turned, _ = dr.rotary(qkv[:, :, :Hq + Hkv], place[..., None], axis, freq, False, rows)
    ctx = dr.linear_attention(turned[:, :, :Hq], turned[:, :, Hq:], qkv[:, :, Hq + Hkv:], off, ld, 1 / math.sqrt(d))["ctx"].reshape(B, R, Hq * d)
    t = ctx @ p["outw"] + p["outb"][:, None]
    if keep is not None:
        t = t * keep
    gate = y0 @ p["gw"] + p["gb"][:, None]
    s, y = dr.gated_norm(rms, x, t, gate, p["n1w"], bias("n1b"), p["res"], p["n2w"], bias("n2b"), EPS)
    return x, p, t, gate, s, y


class Layer:
    def __init__(self, hb, dtype, rms, off, R):
        self.hb, self.dtype, self.dt, self.rms, self.off, self.R, self.n = hb, dtype, DT[dtype], rms, off.cuda(), R, off.shape[1] - 1
        self.p = {k: v.cuda() for k, v in parameters(dtype).items()}
        if rms:
            del self.p["n1b"], self.p["n2b"]
        self.g = {k: torch.full(v.shape, 7.0, device="cuda") for k, v in self.p.items()}
        self.freq, self.axis, self.ld = (t.cuda() for t in common())
        act = lambda k: torch.zeros(B, R, k, dtype=TDT[dtype], device="cuda")
        for k, w in dict(x=E, y0=E, qkv=W, ctx=Hq * d, t=E, gate=E, s=E, y=E, ds=E, dy=E, dx=E, dt=E, dgate=E, ds1=E, dctx=Hq * d, dqkv=W, da=E, db=E,
                         dy0=E).items():
            setattr(self, "d_t" if k == "dt" else k, act(w))
        self.st = [torch.zeros(B * R, device="cuda") for _ in range(6)]
        self.drop = torch.tensor(DROP, device="cuda")
        self.seed = torch.from_numpy(np.array(SEED, dtype=np.uint64).view(np.int64)).cuda()
        self.step = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.size, self.cs = (B, R, self.n, Hq, Hkv, d, self.dt), (R * Hq * d, Hq * d, d)
        need = [hb.linear_attention_bwd_workspace_bytes(*self.size), hb.linear_attention_fwd_workspace_bytes(*self.size),
                hb.gated_residual_norm_bwd_workspace_bytes(B, R, E)]
        need += [hb.linear_bwd_workspace_bytes(B, R, a, z, self.dt) for a, z in ((E, W), (Hq * d, E), (E, E))]
        self.ws = torch.empty(max(16, *need), dtype=torch.uint8, device="cuda")

    def heads(self, t):
        return t.split([Hq * d, Hkv * d, Hkv * d], 2)

    def front(self, pos=None):
        hb, p, R = self.hb, self.p, self.R
        hb.gated_residual_norm_fwd(B, R, E, self.dt, self.rms, self.x, None, None, None, None, None, p["n0w"], None, EPS, None, self.y0, None, None,
                                   self.st[4], self.st[0])
        hb.linear_fwd(B, R, E, W, self.dt, self.y0, p["inw"], p["inb"], self.qkv)
        self.turn(self.qkv, 0, pos)
        hb.linear_fwd(B, R, E, E, self.dt, self.y0, p["gw"], p["gb"], self.gate)

    def turn(self, qkv, inverse, pos=None):                # queries and keys are neighbours in a row
        s = (self.R * W, W, d)
        self.hb.rotary_packed(B, self.R, self.n, Hq + Hkv, d, self.dt, qkv, s, pos, 1, self.axis, PAIRS, self.freq, 0, None if pos is not None else self.off,
                              inverse, qkv, s)

    def back(self, dropout):
        hb, p, R = self.hb, self.p, self.R
        hb.linear_fwd(B, R, Hq * d, E, self.dt, self.ctx, p["outw"], p["outb"], self.t)
        if dropout:
            hb.dropout_counter(B, R * E, self.dt, self.t, self.drop, self.seed, self.step, SITE, self.t)
        hb.gated_residual_norm_fwd(B, R, E, self.dt, self.rms, self.x, self.t, self.gate, p["n1w"], p.get("n1b"), p["res"], p["n2w"], p.get("n2b"), EPS,
                                   self.s, self.y, self.st[3], self.st[1], self.st[5], self.st[2])

    def fwd(self, dropout=True, state=None):
        self.front()
        q, k, v = self.heads(self.qkv)
        s = (self.R * W, W, d)
        self.hb.linear_attention_fwd(*self.size, q, s, k, v, s, self.off, self.ld, 1 / math.sqrt(d), None, self.ctx, self.cs, state, self.ws)
        self.back(dropout)

    def bwd(self):
        hb, p, g, R, s = self.hb, self.p, self.g, self.R, (self.R * W, W, d)
        hb.gated_residual_norm_bwd(B, R, E, self.dt, self.rms, self.x, self.t, self.gate, p["n1w"], p.get("n1b"), p["res"], p["n2w"], self.st[3], self.st[1],
                                   self.st[5], self.st[2], self.ds, self.dy, self.ds1, self.d_t, self.dgate, g["n1w"], g.get("n1b"), g["n2w"],
                                   g.get("n2b"), g["res"], self.ws)
        hb.dropout_counter(B, R * E, self.dt, self.d_t, self.drop, self.seed, self.step, SITE, self.d_t)
        hb.linear_bwd(B, R, Hq * d, E, self.dt, self.ctx, p["outw"], self.d_t, self.dctx, g["outw"], g["outb"], self.ws)
        q, k, v = self.heads(self.qkv)
        dq, dk, dv = self.heads(self.dqkv)
        hb.linear_attention_bwd(*self.size, q, s, k, v, s, self.off, self.ld, 1 / math.sqrt(d), None, self.dctx, self.cs, None, dq, s, dk, dv, s, None, self.ws)
        self.turn(self.dqkv, 1)
        hb.linear_bwd(B, R, E, W, self.dt, self.y0, p["inw"], self.dqkv, self.da, g["inw"], g["inb"], self.ws)
        hb.linear_bwd(B, R, E, E, self.dt, self.y0, p["gw"], self.dgate, self.db, g["gw"], g["gb"], self.ws)
        hb.add(B * R * E, self.dt, self.da, self.db, self.dy0)
        hb.gated_residual_norm_bwd(B, R, E, self.dt, self.rms, self.x, None, None, None, None, None, p["n0w"], None, None, self.st[4], self.st[0], self.ds1,
                                   self.dy0, self.dx, None, None, None, None, g["n0w"], None, None, self.ws)


def rel(got, want, dtype):
    e = got.double().cpu() - want
    return float(e.norm() / want.norm()) if dtype == "bf16" else float(e.abs().max() / want.abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [0, 1])
def test_training_step(hb, dtype, rms):
    off = dr.offsets(LENGTHS)
    R = int(off.max()) + BEHIND
    g = torch.Generator().manual_seed(5)
    rows = dr.inside(off, R)[0][..., None]
    some = lambda: (torch.randn(B, R, E, generator=g) * rows).to(TDT[dtype])
    layer = Layer(hb, dtype, rms, off, R)
    x, ds, dy = some(), some(), some()
    layer.x.copy_(x), layer.ds.copy_(ds), layer.dy.copy_(dy)
    outs = dict(s=layer.s, y=layer.y, dx=layer.dx, **{"d" + k: v for k, v in layer.g.items()})

    def check(step):
        keep = torch.stack([dr.keep(R * E, DROP[b], SEED[b], SITE, step).view(R, E) / (1 - np.float64(np.float32(DROP[b]))) for b in range(B)])
        p = parameters(dtype)
        if rms:
            del p["n1b"], p["n2b"]
        xr, pr, t, gate, s, y = oracle(rms, p, x, off, keep)
        s.retain_grad()
        ((s * ds.double()).sum() + (y * dy.double()).sum()).backward()
        want = dict(s=s.detach(), y=y.detach(), dx=xr.grad, **{"d" + k: v.grad for k, v in pr.items()})
        for name, w in want.items():
            got = outs[name]
            if name in ("s", "y", "dx"):
                got, w = got.cpu() * rows, w * rows
            if name == "dres":
                u = (s.detach() - xr.detach()) / pr["res"].detach()[:, None, None]
                terms = (u * s.grad).flatten(1).norm(dim=1)
                e = float(((got.double().cpu() - w).abs() / terms).max())
            else:
                e = rel(got, w, dtype)
            print(f"{dtype} {rms} {step} {name}: {e:.2e}", flush=True)
            assert e <= TOL[dtype], (name, e)

    layer.fwd()
    layer.bwd()
    torch.cuda.synchronize()
    check(0)
    eager = {k: v.clone() for k, v in outs.items()}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layer.fwd()
        layer.bwd()
    for step in (0, 1, 2):                                 # the graph draws anew when the counter moves on
        for v in outs.values():
            v.fill_(7.0)
        layer.step.fill_(step)
        layer.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        replayed = {k: v.clone() for k, v in outs.items()}
        for v in outs.values():
            v.fill_(3.0)
        layer.fwd()
        layer.bwd()
        torch.cuda.synchronize()
        for k, v in outs.items():
            assert torch.equal(v, replayed[k]), (step, k)
            if step == 0:
                assert torch.equal(v, eager[k]), k
    check(2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [0, 1])
def test_prompts_then_tokens(hb, dtype, rms):
    """Prompts in one call, their states into a larger pool, then three tokens of some of the sequences, a call for each."""
    prompts, more = [[17, 70, 0, 9], [5, 24, 90, 1]], [[1, 3, 2, 3], [3, 0, 3, 1]]
    whole = [[a + z for a, z in zip(p, m)] for p, m in zip(prompts, more)]
    woff, poff = dr.offsets(whole), dr.offsets(prompts)
    g = torch.Generator().manual_seed(6)
    x = torch.randn(B, int(woff.max()), E, generator=g).to(TDT[dtype])
    p = parameters(dtype)
    if rms:
        del p["n1b"], p["n2b"]
    with torch.no_grad():
        *_, s, y = oracle(rms, p, x, woff, None)
    n, slots = 4, 9
    R = int(poff.max())
    layer = Layer(hb, dtype, rms, poff, R)
    for b in range(B):
        for i in range(n):
            layer.x[b, poff[b, i]:poff[b, i + 1]] = x[b, woff[b, i]:woff[b, i] + prompts[b][i]].cuda()
    ends = torch.full((B, n, Hkv, d, d), 7.0, device="cuda")
    layer.fwd(dropout=False, state=ends)
    place = torch.stack([torch.randperm(slots, generator=g)[:n] for _ in range(B)])
    pool = torch.full((B, slots, Hkv, d, d), 7.0, device="cuda")
    for b in range(B):
        pool[b, place[b].cuda()] = ends[b]
    got_s, got_y, want_s, want_y = [], [], [], []

    def add(gs, gy, b, row, at):
        got_s.append(gs[b, row].double().cpu()), got_y.append(gy[b, row].double().cpu())
        want_s.append(s[b, at]), want_y.append(y[b, at])
    for b in range(B):
        for i in range(n):
            for t in range(prompts[b][i]):
                add(layer.s, layer.y, b, int(poff[b, i]) + t, int(woff[b, i]) + t)
    one = Layer(hb, dtype, rms, dr.offsets([[1] * n] * B), n)
    sq = (n * W, W, d)
    for t in range(3):
        slot = torch.tensor([[int(place[b, i]) if t < more[b][i] else -1 for i in range(n)] for b in range(B)], dtype=torch.int32)
        pos = torch.tensor([[prompts[b][i] + t for i in range(n)] for b in range(B)], dtype=torch.int32)[..., None]
        for b in range(B):
            for i in range(n):
                if t < more[b][i]:
                    one.x[b, i] = x[b, woff[b, i] + prompts[b][i] + t].cuda()
        one.front(pos.cuda())
        q, k, v = one.heads(one.qkv)
        hb.linear_attention_step(B, n, slots, Hq, Hkv, d, DT[dtype], q, sq, k, v, sq, slot.cuda(), one.ld, 1 / math.sqrt(d), pool, one.ctx, one.cs, pool)
        one.back(False)
        torch.cuda.synchronize()
        for b in range(B):
            for i in range(n):
                if t < more[b][i]:
                    add(one.s, one.y, b, i, int(woff[b, i]) + prompts[b][i] + t)
    for name, got, want in (("s", got_s, want_s), ("y", got_y, want_y)):
        assert rel(torch.stack(got), torch.stack(want), dtype) <= TOL[dtype], name
    free = torch.ones(B, slots, dtype=torch.bool)
    for b in range(B):
        free[b, place[b]] = False
    assert bool((pool[free.cuda()] == 7.0).all())
