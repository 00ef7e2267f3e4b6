"""Offsets and slots of any values, and workspaces of exactly the size asked for: the operators of a decoder layer write nothing past their
tensors, states and workspaces, and offsets that are in order but out of range give the bits of those taken into it."""
import pytest
import torch

from util import DT, TDT

pytestmark = pytest.mark.gpu
B, GUARD, MARK = 2, 4096, 7.0
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


class Guarded:
    """Tensors and workspaces that lie between guards."""

    def __init__(self):
        self.guards, self.out = [], {}

    def tensor(self, name, dtype, *shape):
        n = 1
        for s in shape:
            n *= s
        flat = torch.full((n + 2 * GUARD,), MARK, dtype=dtype, device="cuda")
        self.guards.append((name, flat, n))
        self.out[name] = flat[GUARD:GUARD + n].view(*shape)
        return self.out[name]

    def space(self, name, size):
        flat = torch.full((size + 2 * GUARD,), 85, dtype=torch.uint8, device="cuda")
        self.guards.append((name, flat, size))
        return flat[GUARD:GUARD + size]

    def check(self):
        torch.cuda.synchronize()
        for name, x, n in self.guards:
            mark = 85 if x.dtype == torch.uint8 else MARK
            assert bool((x[:GUARD] == mark).all()) and bool((x[GUARD + n:] == mark).all()), name


class Attention(Guarded):
    """Linear attention forward and backward, each with a workspace of its own size, or of that for `most` rows and sequences."""

    def __init__(self, hb, dtype, R, off, d, states, Hq=4, Hkv=2, models=B, most=None):
        super().__init__()
        dt, tdt, nseq = DT[dtype], TDT[dtype], len(off[0]) - 1
        g = torch.Generator().manual_seed(R)
        n = lambda *s, t=tdt: torch.randn(*s, generator=g).to(t).cuda()
        O = torch.tensor(off, dtype=torch.int32, device="cuda")
        q, k, v, dctx = n(models, R, Hq, d), n(models, R, Hkv, d), n(models, R, Hkv, d), n(models, R, Hq, d)
        ld = -torch.rand(models, Hkv, generator=g).cuda() * 0.2
        s0, dsf = (n(models, nseq, Hkv, d, d, t=torch.float32) if states else None for _ in range(2))
        o = lambda name, t, *s: self.tensor(name, t, models, *s)
        ctx, dq, dk, dv = o("ctx", tdt, R, Hq, d), o("dq", tdt, R, Hq, d), o("dk", tdt, R, Hkv, d), o("dv", tdt, R, Hkv, d)
        s1, ds0 = (o(m, torch.float32, nseq, Hkv, d, d) if states else None for m in ("s1", "ds0"))
        size, s, ks = (models, R, nseq, Hq, Hkv, d, dt), (R * Hq * d, Hq * d, d), (R * Hkv * d, Hkv * d, d)
        room = size if most is None else (models, *most, Hq, Hkv, d, dt)
        self.fwd_bytes, self.bwd_bytes = hb.linear_attention_fwd_workspace_bytes(*room), hb.linear_attention_bwd_workspace_bytes(*room)
        wf, wb = self.space("workspace forward", self.fwd_bytes), self.space("workspace backward", self.bwd_bytes)
        hb.linear_attention_fwd(*size, q, s, k, v, ks, O, ld, 0.2, s0, ctx, s, s1, wf)
        hb.linear_attention_bwd(*size, q, s, k, v, ks, O, ld, 0.2, s0, dctx, s, dsf, dq, s, dk, dv, ks, ds0, wb)
        self.check()


class Rotary(Guarded):
    def __init__(self, hb, dtype, R, off, d):
        super().__init__()
        g = torch.Generator().manual_seed(R)
        x = torch.randn(B, R, 3, d, generator=g).to(TDT[dtype]).cuda()
        freq, s = torch.rand(B, d // 2, generator=g).cuda(), (R * 3 * d, 3 * d, d)
        O = torch.tensor(off, dtype=torch.int32, device="cuda")
        for inter in (0, 1):
            y = self.tensor("y%d" % inter, TDT[dtype], B, R, 3, d)
            hb.rotary_packed(B, R, len(off[0]) - 1, 3, d, DT[dtype], x, s, None, 1, None, d // 2, freq, inter, O, 0, y, s)
        self.check()


def clamped(off, R):
    return [[min(max(x, 0), R) for x in row] for row in off]


def both(hb, dtype, R, off):
    for d in (16, 40, 128):
        yield lambda o, d=d: Rotary(hb, dtype, R, o, d)
        for states in (False, True):
            if not states or len(off[0]) * d * d < 1 << 23:
                yield lambda o, d=d, states=states: Attention(hb, dtype, R, o, d, states)


def same(a, b):
    for name, t in a.out.items():
        assert torch.equal(t.nan_to_num(123.0), b.out[name].nan_to_num(123.0)), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [80, 700])
@pytest.mark.parametrize("off", [[[-5, 40, 10 ** 6], [LOW, 33, HIGH]], [[80, 80, 89], [-9, -3, -1]], [[LOW, LOW, HIGH], [-1, 81, HIGH]]],
                         ids=["both", "none", "ends"])
def test_out_of_range(hb, dtype, R, off):
    print(dtype, R, off, flush=True)
    for call in both(hb, dtype, R, off):
        same(call(off), call(clamped(off, R)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [80, 3000])
@pytest.mark.parametrize("off", [[[80, 0, 40], [50, 20, 70]], [[HIGH, LOW, 3], [LOW, HIGH, LOW]], [[40, HIGH, 40], [HIGH, 7, LOW]]],
                         ids=["turned", "extreme", "back"])
def test_out_of_order(hb, dtype, R, off):
    print(dtype, R, off, flush=True)
    for call in both(hb, dtype, R, off):
        call(off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [300, 5000])
def test_thousands(hb, dtype, R):
    """Offsets that are searched."""
    print(dtype, R, flush=True)
    g = torch.Generator().manual_seed(3)
    any_ = torch.randint(-R, 2 * R, (B, 2401), generator=g)
    any_[1, ::50] = torch.where(torch.arange(49) % 2 == 0, LOW, HIGH)
    for call in both(hb, dtype, R, any_.tolist()):
        call(any_.tolist())
    off = torch.sort(any_, 1).values.tolist()
    for call in both(hb, dtype, R, off):
        same(call(off), call(clamped(off, R)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("R,lengths,d,Hkv", [(5000, [3000, 2000], 32, 2), (9000, [9000], 128, 1), (2100, [2100], 64, 40), (700, [350, 350], 16, 300)],
                         ids=["summed", "along the sequences", "few blocks", "one block"])
def test_workspaces_of_exactly_their_size(hb, dtype, states, R, lengths, d, Hkv):
    print(dtype, states, R, d, flush=True)
    off = [[0] + torch.tensor(lengths).cumsum(0).tolist()] * B
    a = Attention(hb, dtype, R, off, d, states, Hkv, Hkv)
    assert (a.fwd_bytes > 0 and a.bwd_bytes > 0) == (Hkv * B < 512)
    same(a, Attention(hb, dtype, R, off, d, states, Hkv, Hkv, most=(4 * R, 9)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [16, 63, 128])
def test_slots_of_any_values(hb, dtype, d):
    n, slots, H = 40, 9, 3
    g = torch.Generator().manual_seed(d)
    slot = torch.randint(LOW, HIGH, (B, n), generator=g).int()
    slot[:, ::3] = torch.randint(-3, slots + 3, slot[:, ::3].shape, generator=g).int()
    slot[0, :4] = torch.tensor([LOW, HIGH, slots, -1])
    q, k, v = (torch.randn(B, n, H, d, generator=g).to(TDT[dtype]).cuda() for _ in range(3))
    ld, s = -torch.rand(B, H, generator=g).cuda(), (n * H * d, H * d, d)
    a = Guarded()
    ctx, new = a.tensor("ctx", TDT[dtype], B, n, H, d), a.tensor("new", torch.float32, B, slots, H, d, d)
    state = torch.randn(B, slots, H, d, d, generator=g).cuda()
    hb.linear_attention_step(B, n, slots, H, H, d, DT[dtype], q, s, k, v, s, slot.cuda(), ld, 0.2, state, ctx, s, new)
    a.check()
    for b in range(B):
        took = (slot[b] >= 0) & (slot[b] < slots)
        named = torch.zeros(slots, dtype=torch.bool)
        named[slot[b][took].long()] = True
        assert bool((ctx[b, (~took).cuda()] == MARK).all()) and not bool((ctx[b, took.cuda()] == MARK).flatten(1).all(1).any())
        assert bool((new[b, (~named).cuda()] == MARK).all()) and not bool((new[b, named.cuda()] == MARK).flatten(1).all(1).any())
