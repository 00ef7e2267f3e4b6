"""Linear attention with decays over packed sequences, forward and backward, and its form for single tokens, against the 64-bit form within
its count of roundings: lengths from none to past every tile and block, rows in front of and behind the sequences, head widths of all
kinds, grouped heads, layouts at any alignment; states in and out and their gradients; no memory and memories that never fade; values that
are not finite; slots named twice and not at all; graphs, streams, workspaces, tensors past 2^31 elements."""
import math

import pytest
import torch

import decoder_ref as dr
from util import DT, TDT

pytestmark = pytest.mark.gpu
MARK = 7.0


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def buffers(B, R, heads, d, dtype, layout, fill=MARK):
    if layout == "heads":
        t = torch.full((B, heads, R, d), fill, dtype=TDT[dtype], device="cuda").permute(0, 2, 1, 3)
    elif layout == "odd":
        hs, rs = d + 3, heads * (d + 3) + 5
        flat = torch.full((B * R * rs + 1,), fill, dtype=TDT[dtype], device="cuda")
        t = flat[1:].as_strided((B, R, heads, d), (R * rs, rs, hs, 1), flat.storage_offset() + 1)
    else:
        t = torch.full((B, R, heads, d), fill, dtype=TDT[dtype], device="cuda")
    s = t.stride()
    return t, (s[0], s[1], s[2])


def same(a, b):
    return torch.equal(a.nan_to_num(123.0), b.nan_to_num(123.0))


class Case:
    def __init__(self, dtype, B, lengths, Hq, Hkv, d, layout="rows", first=0, behind=0, seed=0, decay=None, states=False):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.B, self.Hq, self.Hkv, self.d = dtype, B, Hq, Hkv, d
        self.R = max(sum(n) for n in lengths) + first + behind
        self.off = dr.offsets(lengths, first)
        self.nseq = len(lengths[0])
        self.scale = 1.0 / math.sqrt(d)
        for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv), ("dctx", Hq)):
            t, s = buffers(B, self.R, h, d, dtype, layout)
            t.copy_(torch.randn(B, self.R, h, d, generator=g))
            setattr(self, n, t)
            setattr(self, n + "s", s)
        for n, h in (("ctx", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv)):
            t, s = buffers(B, self.R, h, d, dtype, layout)
            setattr(self, n, t)
            setattr(self, n + "s", s)
        if decay is None:
            decay = -(torch.rand(B, Hkv, generator=g) * 6 - 5).exp()
        self.ld = torch.as_tensor(decay, dtype=torch.float32).expand(B, Hkv).contiguous().cuda()
        state = lambda: torch.randn(B, self.nseq, Hkv, d, d, generator=g).cuda() if states else None
        self.s0, self.dsf = state(), state()
        self.s1, self.ds0 = (torch.full_like(self.s0, MARK) if states else None for _ in range(2))
        self.offd = self.off.cuda()
        self.size = (B, self.R, self.nseq, Hq, Hkv, d, DT[dtype])

    def ws(self, hb):
        n = max(16, hb.linear_attention_fwd_workspace_bytes(*self.size), hb.linear_attention_bwd_workspace_bytes(*self.size))
        return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)

    def fwd(self, hb, ws=None, stream=None):
        hb.linear_attention_fwd(*self.size, self.q, self.qs, self.k, self.v, self.ks, self.offd, self.ld, self.scale, self.s0, self.ctx, self.ctxs,
                                self.s1, self.ws(hb) if ws is None else ws, stream)

    def bwd(self, hb, ws=None, stream=None):
        hb.linear_attention_bwd(*self.size, self.q, self.qs, self.k, self.v, self.ks, self.offd, self.ld, self.scale, self.s0, self.dctx, self.ctxs,
                                self.dsf, self.dq, self.dqs, self.dk, self.dv, self.dks, self.ds0, self.ws(hb) if ws is None else ws, stream)

    OUT = (("ctx", "ctx"), ("dq", "dq"), ("dk", "dk"), ("dv", "dv"), ("s1", "state"), ("ds0", "ds0"))

    def check(self, only=None):
        h = lambda t: None if t is None else t.double().cpu()
        args = (h(self.q), h(self.k), h(self.v), self.off, h(self.ld), self.scale, h(self.s0), h(self.dctx), h(self.dsf))
        ref, bound = dr.linear_attention(*args), dr.linear_attention_bounds(*args, dtype=self.dtype)
        rows, _ = dr.inside(self.off, self.R)
        for mine, name in self.OUT:
            t = getattr(self, mine)
            if t is None or (only and mine not in only):
                continue
            want, b = ref[name], dr.stored(ref[name], bound[name], self.dtype if t.dtype == torch.bfloat16 else "f32")
            if name not in ("state", "ds0"):
                want = torch.where(rows[..., None, None], want, torch.full_like(want, MARK))
                b = torch.where(rows[..., None, None], b, torch.zeros_like(b))
            got = t.double().cpu()
            bad = (got - want).abs() - b
            assert bool((bad <= 0).all()), (mine, float(bad.nan_to_num(9e9).max()), (~(bad <= 0)).nonzero()[:3].tolist())


LENGTHS = {
    "tiny": [[1], [0]],
    "small": [[5, 0, 1, 3, 9], [2, 2, 0, 13, 1]],
    "tiles": [[63, 64, 65, 1, 128], [130, 0, 190, 1, 0]],
    "long": [[700, 1, 333], [1030, 0, 4]],
    "one": [[2000], [1537]],
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("heads", [(1, 1), (4, 2)])
@pytest.mark.parametrize("d", [1, 16, 40, 64, 96, 128])
def test_values_and_gradients(hb, dtype, lengths, heads, d):
    for states in (False, True):
        c = Case(dtype, 2, LENGTHS[lengths], *heads, d, first=3 * states, behind=5, seed=d, states=states)
        c.fwd(hb)
        c.bwd(hb)
        c.check()


BLOCKS = {  # B, lengths, Hq, Hkv: how rows are cut into blocks of tiles, and blocks of more than eight tiles
    "one block": (4, [[1100, 0, 80], [3, 1200, 1], [640, 500, 5], [64, 64, 1000]], 65, 65),
    "one block, groups": (4, [[900, 0, 80], [3, 700, 1], [640, 300, 5], [64, 64, 800]], 130, 65),
    "sums of few rows": (1, [[500, 3]], 4, 2),
    "sums of long blocks": (2, [[2600, 0, 1, 2300], [4990, 2, 3, 4]], 40, 40),
    "sums of long blocks, groups": (2, [[2600, 0, 1, 1300], [3500, 2, 3, 4]], 80, 40),
    "sums of many blocks": (1, [[1000, 40, 4000, 0, 3600]], 64, 32),
    "sums along the sequences": (1, [[2500, 40, 30, 3000, 0, 3100]], 4, 2),
    "sums along the sequences, one head": (1, [[4200, 4130]], 2, 1),
    "short ones": (2, [[70, 20, 0, 1, 64, 12, 400, 30, 7, 9, 50, 2, 80, 33, 90, 5, 61, 140, 3, 64], [25] * 19 + [600]], 50, 50),
    "short ones, groups": (2, [[70, 200, 0, 1, 64, 128, 500, 30, 7, 99, 100, 2], [50] * 11 + [700]], 80, 40),
    "short ones, long blocks": (2, [[70, 200, 0, 1, 64, 128, 900, 30, 7, 99, 500, 2], [50] * 11 + [1500]], 100, 100),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("d", [24, 64, 128])
@pytest.mark.parametrize("blocks", list(BLOCKS))
def test_blocks_of_tiles(hb, dtype, states, d, blocks):
    """Some heads of calls with so many that rows fall into few blocks.  Memories that last, so that every block's sum matters."""
    B, lengths, Hq, Hkv = BLOCKS[blocks]
    g = torch.Generator().manual_seed(d)
    c = Case(dtype, B, lengths, Hq, Hkv, d, first=3, behind=5, seed=d, decay=-(torch.rand(B, Hkv, generator=g) * 4 - 10).exp(), states=states)
    c.fwd(hb)
    c.bwd(hb)
    torch.cuda.synchronize()
    G = Hq // Hkv
    for b, h in {(0, 0), (B - 1, Hkv - 1), (B // 2, Hkv // 3)}:
        part = object.__new__(Case)
        part.dtype, part.R, part.off, part.scale, part.ld = dtype, c.R, c.off[b:b + 1], c.scale, c.ld[b:b + 1, h:h + 1]
        for names, lo, n in ((("q", "dctx", "ctx", "dq"), h * G, G), (("k", "v", "dk", "dv"), h, 1)):
            for m in names:
                setattr(part, m, getattr(c, m)[b:b + 1, :, lo:lo + n])
        for m in ("s0", "dsf", "s1", "ds0"):
            t = getattr(c, m)
            setattr(part, m, t[b:b + 1, :, h:h + 1] if states else None)
        part.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["heads", "odd"])
@pytest.mark.parametrize("d", [13, 48, 64, 128])
def test_layouts(hb, dtype, layout, d):
    for states in (False, True):
        c = Case(dtype, 2, [[40, 0, 77], [5, 90, 21]], 3, 1, d, layout, first=2, behind=1, seed=1, states=states)
        c.fwd(hb)
        c.bwd(hb)
        c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays(hb, dtype):
    """No memory at all, memories that never fade (0, and what counts as 0), quick and slow ones, side by side."""
    for states in (False, True):
        decay = torch.tensor([[-math.inf, 0.0, 3.0, -200.0, -5.0, -1e-6]])
        c = Case(dtype, 2, [[300, 1, 64], [129, 0, 1]], 6, 6, 32, behind=2, decay=decay, states=states)
        c.fwd(hb)
        c.bwd(hb)
        c.check()


FADES = {  # B, lengths, d: one block of tiles, few long ones, sums added up by each block and along the sequences, short sequences walked again
    "one block": (90, [[200, 0, 61]], 16),
    "few blocks": (40, [[330, 1, 50]], 32),
    "sums": (1, [[1100, 20]], 32),
    "sums along the sequences": (1, [[2300, 30]], 128),
    "walked": (2, [[100, 90, 150, 7, 64], [64, 128, 30, 1, 70]], 64),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("case", list(FADES))
def test_what_is_left_of_a_state(hb, dtype, states, case):
    """Rows that add nothing: a state, and the gradient of one, has faded by many times its own size and keeps its digits.  Without states in and out
    only a sequence's first keys and last context gradients are not zero."""
    B, lengths, d = FADES[case]
    decay = torch.tensor([[-0.05, -0.1, -0.15, -0.2, -0.27, -0.5]])
    c = Case(dtype, B, lengths * (B // len(lengths)), 6, 6, d, first=3, behind=5, seed=d, decay=decay, states=states)
    for b in range(B):
        for lo, hi in zip(c.off[b, :-1].tolist(), c.off[b, 1:].tolist()):
            n = 0 if states else 5
            c.k[b, lo + n:hi] = 0.0
            c.dctx[b, lo:max(hi - n, lo)] = 0.0
    c.fwd(hb)
    c.bwd(hb)
    c.check()


def test_a_decay_that_is_no_number(hb):
    decay = torch.tensor([[-0.1, math.nan]])
    c = Case("f32", 2, [[30, 9], [20, 1]], 2, 2, 16, decay=decay)
    c.fwd(hb)
    rows, _ = dr.inside(c.off, c.R)
    assert bool(torch.isfinite(c.ctx[:, :, 0].cpu()).all()) and bool(torch.isnan(c.ctx[0, 2:30, 1]).all())


def test_many_sequences(hb):
    g = torch.Generator().manual_seed(0)
    lengths = [torch.randint(0, 4, (3000,), generator=g).tolist() for _ in range(2)]
    for states in (False, True):
        c = Case("bf16", 2, lengths, 2, 1, 32, behind=9, states=states)
        c.fwd(hb)
        c.bwd(hb)
        c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pieces_of_a_prompt(hb, dtype):
    """A sequence in three calls, each from the state that the one before left, gives what one call gives."""
    c = Case(dtype, 1, [[500]], 2, 2, 64, seed=3, states=True)
    c.fwd(hb)
    whole, last = c.ctx.clone(), c.s1.clone()
    at, after = c.s0.clone(), torch.empty_like(c.s0)
    got = torch.zeros_like(whole)
    off = torch.tensor([[0, 0]], dtype=torch.int32, device="cuda")
    for lo, hi in ((0, 131), (131, 132), (132, 500)):
        off[0, 0], off[0, 1] = lo, hi
        hb.linear_attention_fwd(*c.size, c.q, c.qs, c.k, c.v, c.ks, off, c.ld, c.scale, at, got, c.ctxs, after, c.ws(hb))
        at, after = after, at
    c.ctx, c.s1 = got, at
    c.check(("ctx", "s1"))
    # token by token from the same state
    state, one = c.s0[:, 0].reshape(1, 1, 2, 64, 64).clone(), torch.zeros_like(whole)
    for t in range(500):
        hb.linear_attention_step(1, 1, 1, 2, 2, 64, DT[dtype], c.q[:, t], c.qs, c.k[:, t], c.v[:, t], c.ks, None, c.ld, c.scale, state, one[:, t],
                                 c.ctxs, state)
    c.ctx, c.s1 = one, state
    c.check(("ctx", "s1"))
    assert float((last - at).abs().max()) < 1e-3 * float(last.abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_values_that_are_not_finite(hb, dtype, d):
    """They reach the rows that see them and no others, whatever tile they share; gradients go the other way."""
    for states in (False, True):
        for what, row, fwd_from in (("k", 70, True), ("v", 100, True), ("q", 33, False)):
            for bad in (math.nan, math.inf):
                c = Case(dtype, 1, [[20, 130, 30]], 2, 1, d, behind=3, seed=2, states=states)
                good = Case(dtype, 1, [[20, 130, 30]], 2, 1, d, behind=3, seed=2, states=states)
                getattr(c, what)[0, row, 0, 0] = bad
                for x in (c, good):
                    x.fwd(hb)
                    x.bwd(hb)
                t = torch.arange(c.R)
                seq = (t >= 20) & (t < 150)
                fwd_hit = seq & (t >= row) if fwd_from else t == row
                # gradients: dq of later rows, dk and dv of rows up to it where it is a query; of its own row's partner everywhere
                hit = dict(ctx=fwd_hit, dq=seq & (t >= row) if fwd_from else torch.zeros_like(seq),
                           dk={"k": torch.zeros_like(seq), "v": t == row, "q": seq & (t <= row)}[what],
                           dv={"k": t == row, "v": torch.zeros_like(seq), "q": seq & (t <= row)}[what])
                for n, h in hit.items():
                    keep = (~h).cuda()
                    a, b = getattr(c, n)[0, keep], getattr(good, n)[0, keep]
                    assert torch.equal(a, b), (what, row, n, bad, states)
                head = 0
                assert bool((~torch.isfinite(c.ctx[0, fwd_hit.cuda()][:, head].float())).any(1).all()), (what, row, bad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_gradients_and_states_that_are_not_finite(hb, dtype, d):
    """A context gradient reaches its own query and the keys and values up to its row; a state its own sequence."""
    for states in (False, True):
        for bad in (math.nan, -math.inf):
            for row in (33, 148):
                c, good = (Case(dtype, 1, [[20, 130, 30]], 2, 1, d, behind=3, seed=2, states=states) for _ in range(2))
                c.dctx[0, row, 0, 0] = bad
                for x in (c, good):
                    x.bwd(hb)
                t = torch.arange(c.R)
                seq = (t >= 20) & (t < 150)
                for n, h in (("dq", t == row), ("dk", seq & (t <= row)), ("dv", seq & (t <= row))):
                    assert same(getattr(c, n)[0, (~h).cuda()], getattr(good, n)[0, (~h).cuda()]), (n, row, bad, states)
                    assert not bool(torch.isfinite(getattr(c, n)[0, h.cuda()][:, 0].float()).all(-1).any()), (n, row, bad, states)
    for bad in (math.nan, math.inf):
        c, good = (Case(dtype, 1, [[20, 130, 30]], 2, 1, d, behind=3, seed=2, states=True) for _ in range(2))
        c.s0[0, 1, 0, 0, 0] = bad
        c.dsf[0, 1, 0, 0, 0] = bad
        for x in (c, good):
            x.fwd(hb)
            x.bwd(hb)
        other = (torch.arange(c.R) < 20) | (torch.arange(c.R) >= 150)
        for n in ("ctx", "dq", "dk", "dv"):
            assert same(getattr(c, n)[0, other.cuda()], getattr(good, n)[0, other.cuda()]), (n, bad)
        for n in ("s1", "ds0"):
            a, b = getattr(c, n), getattr(good, n)
            assert torch.equal(a[:, ::2], b[:, ::2]) and not bool(torch.isfinite(a[0, 1, 0, 0, 0])), (n, bad)
        assert not bool(torch.isfinite(c.ctx[0, 20:150, 0].float()).all(-1).any()) and not bool(torch.isfinite(c.dk[0, 20:150, 0].float()).all(-1).any()), bad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_thousands_of_query_heads_on_one_key_head(hb, dtype):
    for states in (False, True):
        c = Case(dtype, 1, [[140, 9]], 4096, 1, 16, first=1, behind=2, seed=8, decay=-0.03, states=states)
        c.fwd(hb)
        c.bwd(hb)
        torch.cuda.synchronize()
        rows = slice(0, 4096, 4095 // 12)                         # some of the query heads; keys, values and states of all of them
        part = object.__new__(Case)
        part.__dict__.update(c.__dict__)
        for m in ("q", "dctx", "ctx", "dq"):
            setattr(part, m, getattr(c, m)[:, :, rows])
        part.check(("ctx", "dq", "s1"))
    h = lambda t: t.double().cpu()
    # dk = sum over heads of lambda^(t - s) (v_s . dctx_t) q_t scale: the heads' sum is one product of matrices
    lo, hi = c.off[0, 0].item(), c.off[0, 1].item()
    t = torch.arange(hi - lo, dtype=torch.float64)
    D = torch.exp(h(c.ld)[0, 0] * (t[:, None] - t).clamp(min=0)).tril()
    q, dctx, k, v, dsf = (h(x) for x in (c.q[0, lo:hi], c.dctx[0, lo:hi], c.k[0, lo:hi, 0], c.v[0, lo:hi, 0], c.dsf[0, 0, 0]))
    down = torch.exp(h(c.ld)[0, 0] * (t.numel() - 1 - t))[:, None]
    base = (2 * 16 + (2 + 4096) * (hi - lo) + 40) * dr.U + (3 * 2.0 ** -16 if dtype == "bf16" else 0.0)
    for got, a, b, x, st in ((c.dk, v, dctx, q, dsf.T), (c.dv, k, q, dctx, dsf)):
        f = lambda a, b, x, st: sum(c.scale * (D.T * (a @ b[:, i].T)) @ x[:, i] for i in range(b.shape[1])) + down * (a @ st)
        want, bound = f(a, b, x, st), base * f(a.abs(), b.abs(), x.abs(), st.abs())
        assert float(((h(got[0, lo:hi, 0]) - want).abs() - dr.stored(want, bound, dtype)).max()) <= 0


def test_as_many_heads_and_blocks_as_a_launch_takes(hb):
    """Query heads that leave room for fewer blocks than there are tiles."""
    H, d, lengths = 40000, 8, [[2000, 5, 1800]]
    g = torch.Generator(device="cuda").manual_seed(2)
    off = dr.offsets(lengths)
    R = int(off.max())
    q = torch.randn(1, R, H, d, generator=g, device="cuda").bfloat16()
    k, v = (torch.randn(1, R, 1, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    ctx, ld = torch.full_like(q, MARK), torch.full((1, 1), -0.01, device="cuda")
    size = (1, R, 3, H, 1, d, 1)
    ws = torch.empty(hb.linear_attention_fwd_workspace_bytes(*size), dtype=torch.uint8, device="cuda")
    hb.linear_attention_fwd(*size, q, (R * H * d, H * d, d), k, v, (R * d, d, d), off.cuda(), ld, 0.3, None, ctx, (R * H * d, H * d, d), None, ws)
    some = [0, 1, 777, 20000, H - 1]
    args = (q[:, :, some].double().cpu(), k.double().cpu(), v.double().cpu(), off, ld.cpu(), 0.3)
    want, bound = dr.linear_attention(*args)["ctx"], dr.linear_attention_bounds(*args, dtype="bf16")["ctx"]
    assert float(((ctx[:, :, some].double().cpu() - want).abs() - dr.stored(want, bound, "bf16")).max()) <= 0


def test_rows_outside_do_not_matter(hb):
    for dtype in ("f32", "bf16"):
        c = Case(dtype, 2, [[60, 0, 9], [3, 40, 1]], 2, 2, 32, first=7, behind=80, seed=4)
        rows = dr.inside(c.off, c.R)[0].cuda()
        for t in (c.q, c.k, c.v, c.dctx):
            t[~rows] = math.nan
        c.fwd(hb)
        c.bwd(hb)
        for t in (c.q, c.k, c.v, c.dctx):
            t[~rows] = 0.0
        c.check()


def test_offsets_of_any_values(hb):
    """Offsets that are out of range or in no order address nothing outside the tensors."""
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        for states in (False, True):
            c = Case("bf16", 2, [[60, 20, 9], [3, 40, 1]], 2, 1, 32, behind=200, seed=4, states=states)
            c.offd = torch.randint(-(1 << 31), (1 << 31) - 1, (2, 4), generator=g).int().cuda() if seed % 2 else \
                torch.randint(-50, c.R + 50, (2, 4), generator=g).int().cuda()
            guard = torch.full((2, 64), MARK, device="cuda")
            c.fwd(hb)
            c.bwd(hb)
            torch.cuda.synchronize()
            assert bool((guard == MARK).all())


def test_workspaces(hb):
    """One workspace of the size for the most rows and sequences serves smaller calls; too little is refused."""
    from paper_2102_02344_amd.binding import HftaError
    need = 0
    for R in (64, 1000, 5000, 20000):
        for nseq in (1, 7, 300):
            for fn in (hb.linear_attention_fwd_workspace_bytes, hb.linear_attention_bwd_workspace_bytes):
                n = fn(2, R, nseq, 4, 2, 64, 1)
                most = fn(2, 20000, 300, 4, 2, 64, 1)
                assert n <= most
    c = Case("bf16", 2, [[2000, 100], [900, 1300]], 2, 2, 64)
    need = hb.linear_attention_bwd_workspace_bytes(*c.size)
    if need:
        with pytest.raises(HftaError):
            c.bwd(hb, torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
        c.bwd(hb, torch.empty(need, dtype=torch.uint8, device="cuda"))
        c.check(("dq", "dk", "dv"))


def test_graphs_streams_and_two_calls_at_once(hb):
    a = Case("bf16", 2, [[600, 50, 3], [20, 400, 90]], 4, 2, 64, behind=4, seed=6, states=True)
    b = Case("bf16", 2, [[600, 50, 3], [20, 400, 90]], 4, 2, 64, behind=4, seed=6, states=True)
    wa, wb = a.ws(hb), b.ws(hb)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    a.fwd(hb, wa)
    b.fwd(hb, wb, other)
    a.bwd(hb, wa)
    b.bwd(hb, wb, other)
    torch.cuda.synchronize()
    names = [m for m, _ in Case.OUT]
    for n in names:
        assert torch.equal(getattr(a, n), getattr(b, n)), n
    want = {n: getattr(a, n).clone() for n in names}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a.fwd(hb, wa)
        a.bwd(hb, wa)
    for i in range(3):
        for n in names:
            getattr(a, n).fill_(MARK)
        wa.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for n, v in want.items():
            assert torch.equal(getattr(a, n), v), (i, n)


def test_past_2_31_elements(hb):
    """The last rows of tensors of more than 2^31 elements, behind a long stretch of zeros."""
    R, H, d = 280000, 64, 128
    g = torch.Generator().manual_seed(1)
    x = torch.zeros(1, R, 3 * H, d, dtype=torch.bfloat16, device="cuda")
    x[0, -40:] = torch.randn(40, 3 * H, d, generator=g).bfloat16().cuda()
    ctx = torch.full((1, R, H, d), MARK, dtype=torch.bfloat16, device="cuda")
    s, cs = (R * 3 * H * d, 3 * H * d, d), (R * H * d, H * d, d)
    off = torch.tensor([[R - 1000, R]], dtype=torch.int32)
    ld = torch.full((1, H), -0.05, device="cuda")
    size = (1, R, 1, H, H, d, 1)
    ws = torch.empty(max(16, hb.linear_attention_fwd_workspace_bytes(*size)), dtype=torch.uint8, device="cuda")
    hb.linear_attention_fwd(*size, x, s, x[:, :, H:], x[:, :, 2 * H:], s, off.cuda(), ld, 0.1, None, ctx, cs, None, ws)
    tail = x[:, -40:].double().cpu()
    args = (tail[:, :, :H], tail[:, :, H:2 * H], tail[:, :, 2 * H:], torch.tensor([[0, 40]]), ld.cpu(), 0.1)
    want = dr.linear_attention(*args)["ctx"]
    b = dr.stored(want, 25 * dr.linear_attention_bounds(*args, dtype="bf16")["ctx"], "bf16")       # (a bound of 1000 rows, not 40)
    assert float(((ctx[:, -40:].double().cpu() - want).abs() - b).max()) <= 0
    assert bool((ctx[:, :R - 1000] == MARK).all()) and not bool(ctx[:, R - 1000:R - 40].any())


# ------------------------------------------------------------------ single tokens
def step_ref(q, k, v, slot, ld, scale, state):
    """Rows one after another.  (ctx, states, and the sums of absolute values of both)"""
    B, n, Hq, d = q.shape
    Hkv = k.shape[2]
    lam = torch.exp(ld.double().clamp(max=0.0))
    ctx, S = torch.zeros_like(q), state.clone()
    actx, A = torch.zeros_like(q), state.abs()
    for b in range(B):
        for i in range(n):
            s = int(slot[b, i])
            if not 0 <= s < state.shape[1]:
                continue
            for h in range(Hkv):
                S[b, s, h] = lam[b, h] * S[b, s, h] + torch.outer(k[b, i, h], v[b, i, h])
                A[b, s, h] = lam[b, h] * A[b, s, h] + torch.outer(k[b, i, h], v[b, i, h]).abs()
                for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    ctx[b, i, g] = scale * (q[b, i, g] @ S[b, s, h])
                    actx[b, i, g] = abs(scale) * (q[b, i, g].abs() @ A[b, s, h])
    return ctx, S, actx, A


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 5, 16, 32, 40, 63, 64, 96, 128])
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (9, 1)])
def test_step(hb, dtype, d, heads):
    Hq, Hkv = heads
    B, n, slots = 2, 7, 11
    g = torch.Generator().manual_seed(d)
    for layout in ("rows", "odd"):
        q, qs = buffers(B, n, Hq, d, dtype, layout)
        k, ks = buffers(B, n, Hkv, d, dtype, layout)
        v, _ = buffers(B, n, Hkv, d, dtype, layout)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g))
        ctx, cs = buffers(B, n, Hq, d, dtype, layout)
        ld = -torch.rand(B, Hkv, generator=g)
        ld[0, 0] = -math.inf
        ld[1, Hkv - 1] = 0.7
        state = torch.randn(B, slots, Hkv, d, d, generator=g)
        # places that no row has, a row without one, one past the end, and a slot three times
        slot = torch.tensor([[3, 0, -1, 3, 10, 3, 11], [5, 4, 9, 2, 1, 0, 1 << 30]], dtype=torch.int32)
        for sl in (slot, None):
            if sl is None:
                sl = torch.arange(n).int().expand(B, -1)
                sd = None
            else:
                sd = sl.cuda()
            want, S, actx, A = step_ref(q.double().cpu(), k.double().cpu(), v.double().cpu(), sl, ld, 0.3, state.double())
            named = torch.zeros(B, slots, dtype=torch.bool)
            for b in range(B):
                for s in sl[b].tolist():
                    if 0 <= s < slots:
                        named[b, s] = True
            took = (sl >= 0) & (sl < slots)
            for alias in (False, True):
                src = state.cuda()
                dst = src if alias else torch.full_like(src, MARK)
                ctx.fill_(MARK)
                hb.linear_attention_step(B, n, slots, Hq, Hkv, d, DT[dtype], q, qs, k, v, ks, sd, ld.cuda(), 0.3, src, ctx, cs, dst)
                # a state: three roundings and the decay's 2 a token, three tokens at most; sums of d products
                bs = 16 * dr.U * A + 1e-30
                keep = named[..., None, None, None]
                ws = torch.where(keep, S, state.double() if alias else torch.full_like(S, MARK))
                assert bool(((dst.double().cpu() - ws).abs() <= torch.where(keep, bs, torch.zeros(()).double())).all())
                wc = torch.where(took[..., None, None], want, torch.full_like(want, MARK))
                bc = torch.where(took[..., None, None], dr.stored(want, (d + 24) * dr.U * actx, dtype), torch.zeros(()).double())
                assert bool(((ctx.double().cpu() - wc).abs() <= bc).all())


def test_step_in_a_graph_with_many_rows(hb):
    B, n, slots, H, d = 2, 700, 900, 2, 32
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(B, n, H, d, generator=g).cuda() for _ in range(3))
    s = (n * H * d, H * d, d)
    ctx, ld = torch.zeros_like(q), -torch.rand(B, H, generator=g).cuda()
    state = torch.randn(B, slots, H, d, d, generator=g).cuda()
    slot = torch.stack([torch.randperm(slots, generator=g)[:n] for _ in range(B)]).int()
    slot[0, 650] = slot[0, 3]
    sd = slot.cuda()
    call = lambda st, c, stream=None: hb.linear_attention_step(B, n, slots, H, H, d, 0, q, s, k, v, s, sd, ld, 0.2, st, c, s, st, stream)
    eager, c2 = state.clone(), torch.zeros_like(ctx)
    graph, inner = torch.cuda.CUDAGraph(), state.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(inner, ctx)
    inner.copy_(state)
    for i in range(3):
        graph.replay()
        call(eager, c2)
        torch.cuda.synchronize()
        assert torch.equal(inner, eager) and torch.equal(ctx, c2), i
    want, S, actx, A = step_ref(q.double().cpu(), k.double().cpu(), v.double().cpu(), slot, ld.cpu(), 0.2, state.double().cpu())
    one, oc = state.clone(), torch.zeros_like(ctx)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(one, oc, other)
    torch.cuda.synchronize()
    assert bool(((one.double().cpu() - S).abs() <= 16 * dr.U * A + 1e-30).all())
    assert bool(((oc.double().cpu() - want).abs() <= (d + 24) * dr.U * actx + 1e-30).all())
