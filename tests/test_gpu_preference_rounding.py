"""Log-probabilities and the preference gradient where rounding shows: a constant added to all logits of a row (which changes neither), one
class with almost all or all of the probability.  The bounds grow with distances from a row's largest logit, not with the logits.

With d = z - max a term exp(d) is off by 3 u |d| (the difference, its product with log2(e), that constant) and the exponential's 2 u.
The running sum takes a step per stretch of the row, whose factors add 3 u each and whose differences are parts of d, and an addition per term of a
thread, of which there are at least 64:  sum_b = u (3 dbar + K / 64 + 30), dbar the mean of |d| under the row's probabilities.
log(sum) adds 4 u of itself:  lp_b = sum_b + u (|z_y - max| + |lp| + 4 |log(sum)|).  A probability is off by 3 u |d| + 5 u + sum_b of
itself, one minus it by u more."""
import math

import pytest
import torch

import packed_ref as pr
from test_gpu_preference import Case
from util import DT

pytestmark = pytest.mark.gpu
U = pr.U


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def moved(dtype, lengths, K, add, seed):
    """A case whose rows are `add` higher, every other one as much lower (rounded to the storage type first: what the kernels see is exact)."""
    c = Case(dtype, lengths, K, seed=seed)
    z = c.z.float()
    z[:, ::2] += add
    z[:, 1::2] -= add
    c.z = z.to(c.z.dtype)
    c.ref = (pr.seq_sums(pr.row_logps(c.z.double(), c.y), c.off) + torch.randn(c.ref.shape, generator=torch.Generator().manual_seed(seed))).float()
    return c


def bounds(c):
    z = c.z.double()
    d = z - z.amax(-1, keepdim=True)
    p = torch.softmax(z, -1)
    sum_b = U * (3 * (p * d.abs()).sum(-1) + c.K / 64 + 30)
    lp = pr.row_logps(z, c.y)
    at = d.gather(2, c.y.long().clamp(min=0)[..., None])[..., 0]
    lp_b = torch.where(c.y >= 0, sum_b + U * (at.abs() + lp.abs() + 4 * torch.exp(d).sum(-1).log()), 0.0)
    return lp, lp_b, p, p * (U * (3 * d.abs() + 5) + sum_b[..., None])


def check(hb, c):
    lp, lp_b, p, p_b = bounds(c)
    tok, out = torch.empty(c.B, c.R, device="cuda"), torch.empty(c.B, c.nseq, device="cuda")
    hb.seq_logps(c.B, c.R, c.K, c.nseq, DT[c.dtype], c.z.cuda(), c.y.cuda(), c.off.cuda(), tok, out)
    loss, logps, g = (t.double() for t in c.loss(hb))
    over = (tok.double().cpu() - lp).abs() - lp_b
    print(f"  log-probabilities: {float(((tok.double().cpu() - lp).abs() / lp_b.clamp(min=1e-30)).max()):.3f} of their bound", flush=True)
    assert bool((over <= 0).all()), float(over.max())
    assert bool((tok <= 0).all())                              # no class is more than certain
    assert torch.equal(out.double().cpu(), logps)
    beta, eps, pairs = c.beta.double(), c.eps.double(), c.nseq // 2
    want, L = pr.preference(c.z.double(), c.y, c.off, c.ref.double(), beta, eps)
    Lb = pr.seq_sums(lp_b, c.off)
    assert bool(((logps - L).abs() <= Lb + U * L.abs()).all())
    t_b = beta[:, None] * (Lb[:, 0::2] + Lb[:, 1::2])
    assert bool(((loss - want).abs() <= t_b.mean(1) + 4 * U * want.abs()).all())
    # the gradient's factor moves with t by at most beta / (4 pairs), and is at most beta / pairs
    seq = torch.stack([torch.bucketize(torch.arange(c.R), c.off[b].long(), right=True) - 1 for b in range(c.B)]).clamp(0, c.nseq - 1)
    f_b = (beta[:, None] / (4 * pairs) * t_b).repeat_interleave(2, 1).gather(1, seq)[..., None]
    f = (beta / pairs)[:, None, None]
    ref = pr.preference_grad(c.z.double(), c.y, c.off, c.ref.double(), beta, eps)
    one = torch.zeros_like(p).scatter_(2, c.y.long().clamp(min=0)[..., None], 1.0)
    has = (c.y >= 0)[..., None]
    e = pr.HALF[c.dtype]
    bound = (f_b * (one - p).abs() + f * (p_b + U * one)) * (1 + 2 * e) + (e + 4 * U) * ref.abs() + 1e-37
    bad = (g - ref).abs() / bound
    print(f"  gradient: {float(bad[has.expand_as(bad)].max()):.3f} of its bound", flush=True)
    assert bool((bad <= 1).all())
    return tok.cpu(), g, one


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [33, 1000, 8193])
@pytest.mark.parametrize("add", [0.0, 100.0, 1000.0, 30000.0])
def test_a_constant_added_to_a_row(hb, dtype, K, add):
    print(dtype, K, add, flush=True)
    check(hb, moved(dtype, [[5, 4], [3, 6]], K, add, K))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [100, 8200])
@pytest.mark.parametrize("above", [6.0, 15.0, 25.0])
def test_confident_labels(hb, dtype, K, above):
    """A tuned model's rows: the label above all others.  One minus its probability keeps its sign."""
    print(dtype, K, above, flush=True)
    c = moved(dtype, [[5, 4], [3, 6]], K, 40.0, K + 1)
    at = c.y.long().clamp(min=0)[..., None]
    c.z.scatter_(2, at, (c.z.float().amax(-1, keepdim=True) + above).to(c.z.dtype))
    c.ref = pr.seq_sums(pr.row_logps(c.z.double(), c.y), c.off).float()
    _, g, one = check(hb, c)
    z, y = pr.preference_grad(c.z.double(), c.y, c.off, c.ref.double(), c.beta.double(), c.eps.double()), c.y >= 0
    own, want = (t[y].masked_select(one[y] > 0) for t in (g, z))
    assert bool((own * want >= 0).all())


@pytest.mark.parametrize("K", [100, 8200])
@pytest.mark.parametrize("top", [37.3, -1003.7, 30000.123])
def test_all_of_the_probability(hb, K, top):
    """The label 200 above the others: exp(-200) adds nothing to 1 in fp32, so its log-probability and the whole gradient are zeros."""
    c = Case("f32", [[5, 4], [3, 6]], K, seed=K, prompts=False)
    c.z = torch.full_like(c.z, top - 200.0).scatter_(2, c.y.long()[..., None], top)
    c.ref[:] = 0.0
    tok, out = torch.empty(c.B, c.R, device="cuda"), torch.empty(c.B, c.nseq, device="cuda")
    hb.seq_logps(c.B, c.R, K, c.nseq, 0, c.z.cuda(), c.y.cuda(), c.off.cuda(), tok, out)
    loss, logps, g = c.loss(hb)
    assert bool((tok == 0).all()) and bool((out == 0).all()) and bool((logps == 0).all()) and bool((g == 0).all())
    assert float((loss.double() - math.log(2.0)).abs().max()) <= U
