"""Log-probabilities of packed sequences and the loss of preferred pairs against the 64-bit forms: vocabularies of any width
and alignment, rows without a label, empty sequences, margins far from zero, labels that are no class, gradients written over
the logits, and tensors past 2^31 elements.

Bounds: a row's log-probability z_y - max - log(sum) takes, with an exponential's argument rounded twice, an error of at most
(n) u for the running sum and its exponentials and u of each term of the difference: lp_b = u (|z_y| + |max| + |lse| + 4) + ep,
ep = u (K / 256 + 40 + 4 max|z|) (a thread's stretch of the row, 256 of them joined in a few steps).  Sums are exact; t is off by
beta times the sum of its rows' errors, the loss by as much (its slope is below 1), the factor of the gradient by beta times that."""
import math

import pytest
import torch

import packed_ref as pr
from util import DT, TDT

pytestmark = pytest.mark.gpu
U = pr.U


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


class Case:
    def __init__(self, dtype, lengths, K, first=0, behind=0, seed=0, spread=2.0, prompts=True):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.B, self.K = dtype, len(lengths), K
        self.R, self.nseq = max(sum(n) for n in lengths) + first + behind, len(lengths[0])
        self.off = pr.offsets(lengths, first)
        self.z = (torch.randn(self.B, self.R, K, generator=g) * spread).to(TDT[dtype])
        self.y = torch.randint(0, K, (self.B, self.R), generator=g).int()
        if prompts:
            self.y[torch.rand(self.B, self.R, generator=g) < 0.3] = -1
        self.ref = torch.randn(self.B, self.nseq, generator=g) * 3
        self.ref = (self.ref.double() + pr.seq_sums(pr.row_logps(self.z.double(), self.y), self.off)).float()
        self.beta = torch.rand(self.B, generator=g) + 0.05
        self.eps = torch.where(torch.arange(self.B) % 2 == 0, 0.0, 0.15)

    def row_bound(self):
        z = self.z.double().abs()
        top = z.amax(-1)
        return U * (3 * top + 2 * math.log(self.K + 1) + 4) + U * (self.K / 256 + 40 + 4 * top)

    def loss(self, hb, dlogits=None, z=None, stream=None):
        B, R, K, pairs = self.B, self.R, self.K, self.nseq // 2
        z = self.z.cuda() if z is None else z
        d = torch.full((B, R, K), 7.0, dtype=TDT[self.dtype], device="cuda") if dlogits is None else dlogits
        loss, logps = torch.empty(B, device="cuda"), torch.empty(B, self.nseq, device="cuda")
        ws = torch.empty(hb.preference_loss_workspace_bytes(B, R, pairs), dtype=torch.uint8, device="cuda").fill_(255)
        hb.preference_loss(B, R, K, pairs, DT[self.dtype], z, self.y.cuda(), self.off.cuda(), self.ref.cuda(), self.beta.cuda(), self.eps.cuda(), loss,
                           logps, d, ws, stream)
        torch.cuda.synchronize()
        return loss.cpu(), logps.cpu(), d.cpu()

    def check_loss(self, got):
        loss, logps, d = (t.double() for t in got)
        z, beta, eps = self.z.double(), self.beta.double(), self.eps.double()
        want, L = pr.preference(z, self.y, self.off, self.ref.double(), beta, eps)
        g = pr.preference_grad(z, self.y, self.off, self.ref.double(), beta, eps)
        rb = torch.where(self.y >= 0, self.row_bound(), 0.0)
        Lb = pr.seq_sums(rb, self.off)
        assert bool(((logps - L).abs() <= Lb + U * L.abs()).all())
        tb = beta[:, None] * (Lb[:, 0::2] + Lb[:, 1::2])
        assert bool(((loss - want).abs() <= tb.mean(1) + 4 * U * want.abs()).all())
        e = pr.HALF[self.dtype]
        is_in, _ = pr.inside(self.off, self.R)
        seq = torch.stack([torch.bucketize(torch.arange(self.R), self.off[b].long(), right=True) - 1 for b in range(self.B)]).clamp(0, self.nseq - 1)
        slope = (beta[:, None] / (self.nseq // 2)).expand_as(tb) * tb          # of the factor: its derivative in t is at most beta / pairs / 4
        cb = slope.repeat_interleave(2, 1).gather(1, seq)[..., None]
        c = (beta / (self.nseq // 2))[:, None, None]
        pb = rb[..., None] + 4 * U * (z.abs() + z.abs().amax(-1, keepdim=True) + 2)
        p = torch.softmax(z, -1)
        one = torch.zeros_like(z).scatter_(2, self.y.long().clamp(min=0)[..., None], 1.0)
        bound = cb * (one + p) + c * (p * pb + 2 * U * (one + p)) + (e + 2 * U) * g.abs()
        rows = is_in[..., None].expand_as(d)
        assert bool((d[~rows] == 7.0).all())
        ok = (d - g).abs() <= bound * (1 + e) + 1e-37
        assert bool(ok[rows].all()), float(((d - g).abs() / bound)[rows].max())
        assert bool((d[(is_in & (self.y < 0))[..., None].expand_as(d)] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,K,first,behind", [
    ([[1, 1]], 1, 0, 0), ([[2, 3], [4, 0]], 5, 0, 1), ([[9, 0, 4, 7], [0, 0, 10, 3]], 17, 2, 3), ([[30, 20]], 1000, 0, 0), ([[3, 4, 5, 1]], 8191, 1, 0),
    ([[3, 4], [4, 2]], 8192, 0, 1), ([[2, 3]], 32001, 0, 0), ([[1] * 40] * 2, 64, 0, 2), ([[200, 150, 1, 90]], 129, 0, 0)],
    ids=lambda x: str(x)[:20].replace(" ", ""))
def test_loss_and_log_probabilities(hb, dtype, lengths, K, first, behind):
    print(dtype, lengths, K, flush=True)
    c = Case(dtype, lengths, K, first, behind, seed=K)
    c.check_loss(c.loss(hb))
    tok, out = torch.full((c.B, c.R), 7.0, device="cuda"), torch.empty(c.B, c.nseq, device="cuda")
    hb.seq_logps(c.B, c.R, K, c.nseq, DT[dtype], c.z.cuda(), c.y.cuda(), c.off.cuda(), tok, out)
    torch.cuda.synchronize()
    t, is_in = pr.row_logps(c.z.double(), c.y), pr.inside(c.off, c.R)[0]
    got = tok.double().cpu()
    assert bool((got[~is_in] == 7.0).all()) and bool((got[is_in & (c.y < 0)] == 0).all())
    assert bool(((got - t).abs() <= c.row_bound())[is_in].all())
    L = pr.seq_sums(t, c.off)
    Lb = pr.seq_sums(torch.where(c.y >= 0, c.row_bound(), 0.0), c.off)
    assert bool(((out.double().cpu() - L).abs() <= Lb + U * L.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_margins_far_from_zero(hb, dtype):
    """beta times the gap at +-2000: the loss is linear on one side and vanishes on the other, nothing overflows."""
    c = Case(dtype, [[5, 6, 4, 4]] * 2, 50, seed=3)
    c.ref[:, 0] += 2000.0
    c.ref[:, 2] -= 2000.0
    c.beta[:] = 1.0
    c.check_loss(c.loss(hb))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [33, 256, 8200])
def test_gradient_over_the_logits(hb, dtype, K):
    c = Case(dtype, [[5, 6, 4, 4]], K, seed=5)
    _, _, want = c.loss(hb)
    z = c.z.cuda()
    _, _, got = c.loss(hb, dlogits=z, z=z)
    assert torch.equal(got, want)


def test_gradient_at_another_alignment(hb):
    c = Case("bf16", [[5, 6]], 1000, seed=6)
    _, _, want = c.loss(hb)
    d = torch.full((c.B * c.R * c.K + 3,), 7.0, dtype=torch.bfloat16, device="cuda")[3:].view(c.B, c.R, c.K)
    _, _, got = c.loss(hb, dlogits=d)
    assert torch.equal(got, want)


def test_labels_that_are_no_class_and_values_that_are_not_finite(hb):
    """They reach their own model's loss and their own pair's gradient; -inf logits are classes that cannot be."""
    a, b = Case("f32", [[5, 6, 4, 4]] * 2, 40, seed=7, prompts=False), Case("f32", [[5, 6, 4, 4]] * 2, 40, seed=7, prompts=False)
    b.y[0, 2] = 40
    la, lpa, da = a.loss(hb)
    lb, lpb, db = b.loss(hb)
    assert math.isnan(lb[0]) and lb[1] == la[1]
    assert bool(db[0, :11].isnan().all()) and torch.equal(db[0, 11:], da[0, 11:]) and torch.equal(db[1], da[1])
    assert math.isnan(lpb[0, 0]) and torch.equal(lpb[0, 1:], lpa[0, 1:])
    b = Case("f32", [[5, 6, 4, 4]] * 2, 40, seed=7, prompts=False)
    b.z[1, 12, 3] = math.nan
    lb, _, db = b.loss(hb)
    assert math.isnan(lb[1]) and lb[0] == la[0] and torch.equal(db[1, :11], da[1, :11]) and bool(db[1, 11:].isnan().any())
    c = Case("f32", [[5, 6, 4, 4]] * 2, 40, seed=7, prompts=False)
    c.z[:, :, ::3] = -math.inf
    c.z[:, :, 1] += 1
    c.y[:] = 1
    c.ref[:] = pr.seq_sums(pr.row_logps(c.z.double(), c.y), c.off).float()
    loss, _, d = c.loss(hb)
    g = pr.preference_grad(c.z.double(), c.y, c.off, c.ref.double(), c.beta.double(), c.eps.double())
    assert bool(torch.isfinite(loss).all()) and bool((d[:, :, ::3] == 0).all()) and float((d.double() - g).abs().max()) < 1e-5


def test_rows_without_a_label_are_not_read(hb):
    a, b = (Case("bf16", [[9, 6]], 300, first=1, behind=2, seed=9) for _ in range(2))
    skip = (b.y < 0) | ~pr.inside(b.off, b.R)[0]
    b.z[skip] = math.nan
    for x, y in zip(a.loss(hb), b.loss(hb)):
        assert torch.equal(x, y)


def test_replays_and_streams(hb):
    a, b = Case("bf16", [[50, 60, 40, 40]] * 2, 1000, seed=11), Case("bf16", [[30, 80, 10, 70]] * 2, 1000, seed=12)
    want = [c.loss(hb) for c in (a, b)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert all(torch.equal(x, y) for x, y in zip(a.loss(hb), want[0]))
    live = [t.cuda() for t in (a.z, a.y, a.off, a.ref, a.beta, a.eps)]
    loss, logps, d = torch.empty(2, device="cuda"), torch.empty(2, 4, device="cuda"), torch.empty(a.z.shape, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(hb.preference_loss_workspace_bytes(2, a.R, 2), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.preference_loss(2, a.R, 1000, 2, 1, *live[:5], live[5], loss, logps, d, ws)
    for k in range(4):
        c = (a, b)[k % 2]
        for t, x in zip(live, (c.z, c.y, c.off, c.ref, c.beta, c.eps)):
            t.copy_(x)
        graph.replay()
        b.loss(hb)
        torch.cuda.synchronize()
        assert all(torch.equal(x.cpu(), y) for x, y in zip((loss, logps, d), want[k % 2])), k


def test_past_two_to_the_31_elements(hb):
    R, K = 60000, 40000
    z = torch.zeros(1, R, K, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(20, K, generator=torch.Generator().manual_seed(3)).bfloat16()
    z[0, R - 20:] = tail.cuda()
    y = torch.full((1, R), -1, dtype=torch.int32)
    y[0, R - 20:] = torch.arange(20, dtype=torch.int32) * 1999 + 3
    off = torch.tensor([[R - 20, R - 9, R]], dtype=torch.int32)
    ref, beta = torch.full((1, 2), -90.0), torch.tensor([0.1])
    loss, logps = torch.empty(1, device="cuda"), torch.empty(1, 2, device="cuda")
    ws = torch.empty(hb.preference_loss_workspace_bytes(1, R, 1), dtype=torch.uint8, device="cuda")
    hb.preference_loss(1, R, K, 1, 1, z, y.cuda(), off.cuda(), ref.cuda(), beta.cuda(), None, loss, logps, z, ws)
    torch.cuda.synchronize()
    t, o = tail.double()[None], torch.tensor([[0, 11, 20]])
    want, L = pr.preference(t, y[:, R - 20:], o, ref.double(), beta.double(), torch.zeros(1).double())
    g = pr.preference_grad(t, y[:, R - 20:], o, ref.double(), beta.double(), torch.zeros(1).double())
    rb = U * (7 * t.abs().max() + 80 + K / 256)
    assert float((logps.double().cpu() - L).abs().max()) <= 11 * rb + U * float(L.abs().max())
    assert float((loss.double().cpu() - want).abs().max()) <= 20 * rb
    got = z[0, R - 20:].double().cpu()[None]
    assert bool(((got - g).abs() <= (2.0 ** -8 + 30 * rb) * g.abs() + 1e-30).all())
    assert not bool(z[0, R - 22:R - 20].any())                  # rows in front of the first sequence: as they were


def test_texts_that_cannot_be(hb):
    """A label whose logit is -inf: as a rejected text it costs nothing and leaves no gradient, smoothed or preferred it costs an infinity,
    with the factor of the gradient at its limit."""
    for side, eps, want in ((1, 0.0, 0.0), (1, 0.25, math.inf), (0, 0.0, math.inf), (0, 1.0, 0.0)):
        c = Case("f32", [[3, 4]], 40, seed=11, prompts=False)
        c.ref = torch.zeros(1, 2)
        c.eps[:] = eps
        row = 3 * side + 1
        rb = float(c.row_bound().max()) * 2 + 4 * U                  # of a probability, relative
        c.z[0, row, int(c.y[0, row])] = -math.inf
        loss, logps, d = c.loss(hb)
        assert float(loss[0]) == want and float(logps[0, side]) == -math.inf and math.isfinite(logps[0, 1 - side])
        f = float(c.beta[0]) * (eps if side else eps - 1)            # sigma(t) is 1 where the rejected text cannot be, or else 0
        p = torch.softmax(c.z.double(), -1)
        one = torch.zeros_like(p).scatter_(2, c.y.long()[..., None], 1.0)
        g = f * (one - p) * torch.tensor([1.0] * 3 + [-1.0] * 4)[:, None]
        assert float((d.double() - g).abs().max()) <= rb * abs(f) and (f != 0 or bool((d == 0).all()))


@pytest.mark.parametrize("lengths", [[[9000, 20011], [20011, 9000]], [[2047, 2049], [1, 2048]]], ids=["long", "steps"])
def test_sums_of_long_sequences(hb, lengths):
    c = Case("f32", lengths, 7, behind=2, seed=12)
    loss, logps, _ = c.loss(hb)
    want, L = pr.preference(c.z.double(), c.y, c.off, c.ref.double(), c.beta.double(), c.eps.double())
    Lb = pr.seq_sums(torch.where(c.y >= 0, c.row_bound(), 0.0), c.off)
    assert bool(((logps.double() - L).abs() <= Lb + U * L.abs()).all())
    assert bool(((loss.double() - want).abs() <= (c.beta.double()[:, None] * Lb).sum(1) + 4 * U * want.abs()).all())
    tok, out = torch.empty(c.B, c.R, device="cuda"), torch.empty(c.B, c.nseq, device="cuda")
    hb.seq_logps(c.B, c.R, c.K, c.nseq, DT["f32"], c.z.cuda(), c.y.cuda(), c.off.cuda(), tok, out)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), logps)
