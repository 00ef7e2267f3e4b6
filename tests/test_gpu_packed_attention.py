"""Attention over packed sequences with grouped heads against the 64-bit form, within its count of roundings
(packed_ref.attention): lengths from none to past every tile, rows in front of and behind the sequences, head widths that
fill a tile and that do not, layouts with heads inside and outside the rows, rows at any alignment; values that are not
finite; calls captured into a graph, on another stream, twice at once; tensors past 2^31 elements."""
import math

import pytest
import torch

import packed_ref as pr
from util import DT, TDT

pytestmark = pytest.mark.gpu
MARK = 7.0                      # what rows outside the sequences hold before and after


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def buffers(B, R, heads, d, dtype, layout, fill=MARK):
    """An empty tensor [B, R, heads, d] as a view of its storage, and its strides (model, row, head)."""
    if layout == "heads":                       # [B][heads][R][d]
        t = torch.full((B, heads, R, d), fill, dtype=TDT[dtype], device="cuda").permute(0, 2, 1, 3)
    elif layout == "odd":                       # rows and heads a step apart that is no multiple of anything, an odd first element
        hs, rs = d + 3, heads * (d + 3) + 5
        flat = torch.full((B * R * rs + 1,), fill, dtype=TDT[dtype], device="cuda")
        t = flat[1:].as_strided((B, R, heads, d), (R * rs, rs, hs, 1), flat.storage_offset() + 1)
    else:
        t = torch.full((B, R, heads, d), fill, dtype=TDT[dtype], device="cuda")
    s = t.stride()
    return t, (s[0], s[1], s[2])


class Case:
    def __init__(self, dtype, B, lengths, Hq, Hkv, d, layout="rows", first=0, behind=0, seed=0, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.B, self.Hq, self.Hkv, self.d = dtype, B, Hq, Hkv, d
        self.R = max(sum(n) for n in lengths) + first + behind
        self.off = pr.offsets(lengths, first)
        self.nseq = len(lengths[0])
        self.scale = scale or 1.0 / math.sqrt(d)
        for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv), ("dctx", Hq)):
            t, s = buffers(B, self.R, h, d, dtype, layout)
            t.copy_(torch.randn(B, self.R, h, d, generator=g))
            setattr(self, n, t)
            setattr(self, n + "s", s)
        for n, h in (("ctx", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv)):
            t, s = buffers(B, self.R, h, d, dtype, layout)
            setattr(self, n, t)
            setattr(self, n + "s", s)
        self.lse = torch.full((B, Hq, self.R), MARK, device="cuda")
        self.offd = self.off.cuda()
        self.size = (B, self.R, self.nseq, Hq, Hkv, d, DT[dtype])

    def fwd(self, hb, causal, stream=None):
        hb.attention_packed_fwd(*self.size, self.q, self.qs, self.k, self.v, self.ks, self.offd, self.scale, causal, self.ctx, self.ctxs,
                                self.lse, stream)

    def bwd(self, hb, causal, stream=None):
        if not hasattr(self, "ws"):
            self.ws = torch.empty(hb.attention_packed_bwd_workspace_bytes(*self.size), dtype=torch.uint8, device="cuda")
        hb.attention_packed_bwd(*self.size, self.q, self.qs, self.k, self.v, self.ks, self.offd, self.scale, causal, self.ctx, self.dctx,
                                self.ctxs, self.lse, self.dq, self.dqs, self.dk, self.dv, self.dks, self.ws, stream)

    def outputs(self):
        return {"ctx": self.ctx, "lse": self.lse, "dq": self.dq, "dk": self.dk, "dv": self.dv}

    def ref(self, causal):
        h = lambda t: t.detach().double().cpu().contiguous()
        return pr.attention(h(self.q), h(self.k), h(self.v), self.off, self.scale, causal, h(self.dctx), self.dtype)

    def check(self, causal):
        ref = self.ref(causal)
        is_in, _ = pr.inside(self.off, self.R)
        for n, t in self.outputs().items():
            got = t.detach().double().cpu()
            rows = is_in[:, None].expand_as(got) if n == "lse" else is_in[..., None, None].expand_as(got)
            assert bool((got[~rows] == MARK).all()), f"{n}: rows of no sequence were written"
            assert bool(torch.isfinite(got[rows]).all()), n
            over = (got - ref[n]).abs() / ref[n + "_b"].clamp(min=1e-30)
            worst = float(over[rows].max()) if bool(rows.any()) else 0.0
            print(f"  {n}: worst error {worst:.3f} of its bound", flush=True)
            assert worst <= 1.0, (n, worst)


LENGTHS = [
    [[1]], [[0, 2]], [[33]], [[64, 0, 1]], [[128]], [[129, 127]], [[1] * 150], [[0, 1, 127, 0, 130, 3]], [[300]],
    [[31, 32, 33, 5, 64, 65, 2]],
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "-".join(map(str, x[0][:8])))
def test_lengths(hb, dtype, causal, lengths):
    print(dtype, causal, lengths, flush=True)
    c = Case(dtype, 1, lengths, 2, 1, 64, first=3 if len(lengths[0]) > 1 else 0, behind=5, seed=len(lengths[0]))
    c.fwd(hb, causal)
    c.bwd(hb, causal)
    torch.cuda.synchronize()
    c.check(causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["rows", "heads", "odd"])
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 1), (4, 4, 16), (4, 2, 24), (6, 2, 32), (3, 3, 40), (8, 1, 64), (2, 2, 72), (4, 2, 100), (4, 1, 128), (3, 1, 127)])
def test_heads_and_layouts(hb, dtype, layout, Hq, Hkv, d):
    causal = (Hq + d) % 2
    print(dtype, layout, Hq, Hkv, d, causal, flush=True)
    c = Case(dtype, 2, [[70, 0, 61, 9], [3, 99, 20, 1]], Hq, Hkv, d, layout, first=2, behind=4, seed=d)
    c.fwd(hb, causal)
    c.bwd(hb, causal)
    torch.cuda.synchronize()
    c.check(causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [24, 64, 120])
@pytest.mark.parametrize("causal", [1, 0])
def test_many_heads(hb, dtype, d, causal):
    """Enough tiles of 128 rows to fill the chip: a wavefront has 32 rows of its own and all keys."""
    c = Case(dtype, 2, [[150, 0, 61, 90], [3, 299, 1, 0]], 96, 48, d, first=1, behind=4, seed=d)
    c.fwd(hb, causal)
    c.bwd(hb, causal)
    torch.cuda.synchronize()
    c.check(causal)


@pytest.mark.parametrize("Hq", [2, 300])
def test_more_sequences_than_threads(hb, Hq):
    g = torch.Generator().manual_seed(6)
    c = Case("bf16", 1, [torch.randint(0, 4, (700,), generator=g).tolist()], Hq, 2, 16, first=2, behind=3, seed=6)
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()
    c.check(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [4, 256])
def test_inputs_of_stride_zero(hb, dtype, Hq):
    """Keys and values shared by all heads, queries by all rows (expanded tensors): gradients come per head and row."""
    c = Case(dtype, 2, [[90, 120], [200, 10]], Hq, Hq, 64, seed=8)
    for n in ("k", "v"):
        t = getattr(c, n)[:, :, :1].contiguous().expand(-1, -1, Hq, -1)
        setattr(c, n, t)
        setattr(c, n + "s", t.stride()[:3])
    c.q = c.q[:, :1].contiguous().expand(-1, c.R, -1, -1)
    c.qs = c.q.stride()[:3]
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()
    c.check(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_in_reverse(hb, dtype):
    """Negative row strides."""
    c = Case(dtype, 1, [[60, 75]], 2, 2, 32, seed=10)
    for n in ("q", "k", "v", "dctx", "ctx", "dq", "dk", "dv"):
        t = getattr(c, n)
        flat = t.flip(1).contiguous()
        s = flat.stride()

        class Last:                                      # the last row in memory is the first
            def __init__(self, x):
                self.x = x

            def data_ptr(self):
                return self.x[:, -1].data_ptr()
        setattr(c, n, Last(flat))
        setattr(c, n + "s", (s[0], -s[1], s[2]))
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()
    for n in ("q", "k", "v", "dctx", "ctx", "dq", "dk", "dv"):
        setattr(c, n, getattr(c, n).x.flip(1))
    c.check(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_projection_and_long_rows(hb, dtype):
    """Q, K, V and their gradients as blocks of one [R][q | k | v] tensor, sequences past several tiles of keys."""
    B, Hq, Hkv, d = 2, 4, 2, 64
    c = Case(dtype, B, [[700, 77, 5], [10, 400, 389]], Hq, Hkv, d, behind=3, seed=9)
    w = (Hq + 2 * Hkv) * d
    for names in (("q", "k", "v"), ("dq", "dk", "dv")):
        t = torch.full((B, c.R, w), MARK, dtype=TDT[dtype], device="cuda")
        for n, x in zip(names, t.split([Hq * d, Hkv * d, Hkv * d], 2)):
            x = x.unflatten(2, (-1, d))
            x.copy_(getattr(c, n))
            setattr(c, n, x)
            setattr(c, n + "s", (c.R * w, w, d))
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()
    c.check(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_equal_scores(hb, dtype):
    """Scores far from zero on both sides, and rows whose scores are all the same: the running maximum moves by much, and not at all."""
    c = Case(dtype, 1, [[200, 90]], 2, 2, 64, seed=4, scale=0.5)
    c.q.mul_(3)
    c.k[:, ::7].mul_(4)
    c.q[:, 200:] = 0
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()
    c.check(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["v", "k", "dctx", "q"])
@pytest.mark.parametrize("many", [0, 1])
def test_values_that_are_not_finite(hb, many, dtype, causal, value, what):
    """One such value in one row: rows that do not see it keep their bits, outputs it takes part in are not finite."""
    lengths, at = [[20, 150, 40]], 20 + 101
    a, b = (Case(dtype, 1, lengths, *((300, 150) if many else (2, 1)), 64, first=4, behind=6, seed=21) for _ in range(2))
    at += 4
    getattr(b, what)[0, at, 0, 9] = value
    for c in (a, b):
        c.fwd(hb, causal)
        if what == "dctx":
            c.bwd(hb, causal)
    torch.cuda.synchronize()
    seq = torch.zeros(a.R, dtype=torch.bool)
    seq[24:174] = True
    row = torch.arange(a.R)
    sees = seq & ((row >= at) if causal else seq)              # queries that see row `at`
    if what in ("v", "k"):
        clean = ~sees
    elif what == "q":
        clean = row != at
    else:
        clean = row != at
    ca, cb = a.ctx[0].float().cpu(), b.ctx[0].float().cpu()
    if what != "dctx":
        heads = slice(0, 2) if what in ("v", "k") else slice(0, 1)
        assert torch.equal(ca[clean], cb[clean]) and torch.equal(ca[:, 2:], cb[:, 2:])
        if what == "v":
            assert not bool(torch.isfinite(cb[sees][:, :2, 9]).any())
            other = [i for i in range(64) if i != 9]
            assert torch.equal(ca[:, :, other], cb[:, :, other])
        elif what == "q" or math.isnan(value):
            hit = (row == at) if what == "q" else sees
            assert not bool(torch.isfinite(cb[hit][:, heads]).any())
        return
    assert torch.equal(ca, cb)
    seen = seq & ((row <= at) if causal else seq)              # keys that row `at` sees
    for n in ("dk", "dv"):
        x, y = getattr(a, n)[0].float().cpu(), getattr(b, n)[0].float().cpu()
        assert torch.equal(x[~seen], y[~seen]) and torch.equal(x[:, 1:], y[:, 1:]), n
        assert not bool(torch.isfinite(y[seen][:, 0]).all(dim=1).any()), n
    x, y = a.dq[0].float().cpu(), b.dq[0].float().cpu()
    assert torch.equal(x[clean], y[clean]) and torch.equal(x[:, 1:], y[:, 1:])
    assert not bool(torch.isfinite(y[at, 0]).any())


@pytest.mark.parametrize("what", ["q", "k"])
@pytest.mark.parametrize("Hq", [2, 600])
def test_gradients_of_rows_that_do_not_see_it(hb, what, Hq):
    """A NaN in a query or key: gradients of the sequences beside it, in the same tiles, keep their bits."""
    a, b = (Case("bf16", 1, [[30, 50, 40]], Hq, Hq, 64, seed=23) for _ in range(2))
    getattr(b, what)[0, 55, 1, 3] = math.nan
    for c in (a, b):
        c.fwd(hb, 1)
        c.bwd(hb, 1)
    torch.cuda.synchronize()
    for n in ("ctx", "dq", "dk", "dv"):
        x, y = getattr(a, n)[0].float().cpu(), getattr(b, n)[0].float().cpu()
        for rows in (slice(0, 30), slice(80, 120)):
            assert torch.equal(x[rows], y[rows]), n
        assert torch.equal(x[:, 0], y[:, 0]), n                # the other head
        assert bool(torch.isnan(y[30:80, 1]).any()), n


def test_garbage_outside_the_sequences_is_not_read(hb):
    a, b = (Case("bf16", 1, [[50, 30]], 2, 1, 64, first=7, behind=60, seed=31) for _ in range(2))
    for n in ("q", "k", "v", "dctx"):
        getattr(b, n)[:, :7] = math.nan
        getattr(b, n)[:, 87:] = math.inf
    b.lse[:] = math.nan
    for c in (a, b):
        c.fwd(hb, 0)
        c.bwd(hb, 0)
    torch.cuda.synchronize()
    for n in ("ctx", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n


def test_offsets_out_of_range_stay_inside(hb):
    """Offsets past the rows, below zero and out of order: taken into range, every row finite, none twice."""
    c = Case("bf16", 1, [[40, 40]], 2, 1, 64, seed=33)
    for off in ([-5, 40, 10 ** 6], [80, 0, 40], [2 ** 31 - 1, -2 ** 31, 3]):
        c.offd = torch.tensor([off], dtype=torch.int32, device="cuda")
        c.fwd(hb, 1)
        c.bwd(hb, 1)
        torch.cuda.synchronize()
        assert all(bool(torch.isfinite(t.float()).all()) for t in c.outputs().values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_streams_and_replays(hb, dtype):
    """Two calls at once on two streams with workspaces of their own, and a captured call replayed between eager ones with
    other inputs, give the bits of single eager calls."""
    cases = [Case(dtype, 2, [[200, 9, 60], [90, 100, 79]], 4, 2, 64, seed=s) for s in (41, 42)]
    want = []
    for c in cases:
        c.fwd(hb, 1)
        c.bwd(hb, 1)
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in c.outputs().items()})
        for t in c.outputs().values():
            t.fill_(MARK)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for c, s in zip(cases, streams):
        c.fwd(hb, 1, s)
        c.bwd(hb, 1, s)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert all(torch.equal(t, w[n]) for n, t in c.outputs().items())
    a, b = cases
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.fwd(hb, 1)
        a.bwd(hb, 1)
    keep = {n: getattr(a, n).clone() for n in ("q", "k", "v", "dctx")}
    for k in range(4):
        src = b if k % 2 else a
        for n in keep:
            getattr(a, n).copy_(getattr(b, n) if k % 2 else keep[n])
        a.offd.copy_(src.off)
        graph.replay()
        b.fwd(hb, 1)                                     # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[k % 2][n]) for n, t in a.outputs().items()), k


def test_past_two_to_the_31_elements(hb):
    """Rows 150000 elements apart: the last ones lie past 2^31 elements, and past 2^32 bytes."""
    R, d, rs = 16000, 64, 150000
    q = torch.empty(R * rs, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(51)
    data = torch.randn(R, 4, d, generator=g).to(torch.bfloat16)
    rows = q.as_strided((1, R, 4, d), (R * rs, rs, d, 1))       # heads: q, k, v, dctx
    rows.copy_(data[None])
    off = torch.tensor([[0, R - 90, R]], dtype=torch.int32)
    offd, s = off.cuda(), (R * rs, rs, d)
    lse = torch.empty(1, 1, R, device="cuda")
    out = torch.empty(1, R, 4, d, dtype=torch.bfloat16, device="cuda")
    os_ = (R * 4 * d, 4 * d, d)
    ctx, dq, dk, dv = (out[:, :, i] for i in range(4))
    size = (1, R, 2, 1, 1, d, 1)
    # dctx and ctx share their strides, so ctx goes beside dctx
    ctx = rows[:, :, 3].as_strided((1, R, d), (R * rs, rs, 1), rows[:, :, 3].storage_offset() + d)
    hb.attention_packed_fwd(*size, rows[:, :, 0], s, rows[:, :, 1], rows[:, :, 2], s, offd, 0.125, 1, ctx, s, lse)
    ws = torch.empty(hb.attention_packed_bwd_workspace_bytes(*size), dtype=torch.uint8, device="cuda")
    hb.attention_packed_bwd(*size, rows[:, :, 0], s, rows[:, :, 1], rows[:, :, 2], s, offd, 0.125, 1, ctx, rows[:, :, 3], s, lse, dq, os_,
                            dk, dv, os_, ws)
    torch.cuda.synchronize()
    t = data[R - 90:].double()[None]
    ref = pr.attention(*(t[:, :, i:i + 1] for i in range(3)), torch.tensor([[0, 90]]), 0.125, 1, t[:, :, 3:4], "bf16")
    for n, x in (("ctx", ctx), ("dq", dq), ("dk", dk), ("dv", dv)):
        got = x[:, R - 90:].double().cpu()[:, :, None]
        assert bool(((got - ref[n]).abs() <= ref[n + "_b"]).all()), n


@pytest.mark.parametrize("Hq", [2, 20])
def test_thousands_of_sequences(hb, Hq):
    """So many that their offsets are searched: short ones, long runs of empty ones around longer ones, and none at all."""
    g = torch.Generator().manual_seed(40)
    short = torch.randint(0, 2, (2400,), generator=g).tolist()
    around = [0] * 1100 + [70] + [0] * 1298 + [200]
    c = Case("bf16", 3, [short, around, [0] * 2400], Hq, 2, 16, first=1, behind=5, seed=40)
    for causal in (1, 0):
        c.fwd(hb, causal)
        c.bwd(hb, causal)
        torch.cuda.synchronize()
        c.check(causal)
    order = torch.randperm(2401, generator=g)                  # in any order: finite and inside
    c.offd = c.off[:, order].contiguous().cuda()
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d", [40, 128])
@pytest.mark.parametrize("lengths", [[[12] * 60], [[20] * 40], [[130, 150]], [[700]]], ids=["12", "20", "140", "700"])
def test_bf16_errors_are_those_of_two_roundings(hb, lengths, d):
    """An output in bf16 has one rounding; p or ds have one before the product, of the same size and independent, so that the mean error is
    sqrt(2) of the rounded result's.  6 % more are for the rest: D, whose error stays in dq where sequences are long, and the sums."""
    c = Case("bf16", 1, lengths, 4, 2, d, seed=d)
    c.fwd(hb, 1)
    c.bwd(hb, 1)
    torch.cuda.synchronize()
    ref, got = c.ref(1), c.outputs()
    far, near = 0.0, 0.0
    for n in ("dq", "dk", "dv"):
        far += float((got[n].double().cpu() - ref[n]).square().sum())
        near += float((ref[n].bfloat16().double() - ref[n]).square().sum())
    print(f"  {math.sqrt(far / near):.3f} roundings", flush=True)
    assert far <= 1.5 ** 2 * near
