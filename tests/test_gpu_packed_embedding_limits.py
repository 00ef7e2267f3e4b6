"""The table gradient by sorted tokens at the ends of what it takes: the largest number of tokens, rows of absent tokens past 2^31 elements,
and rows past the 65536 up to which the sort's blocks add up the counts before them by themselves."""
import pytest
import torch

import packed_ref as pr
from util import DT, TDT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


@pytest.mark.parametrize("V", [2 ** 30, 2 ** 28 + 77])
def test_the_largest_tables(hb, V):
    """2^30 tokens, and a few more than the clearing takes 64 to a workgroup."""
    R = 70
    idx = torch.randint(0, V, (1, R), generator=torch.Generator().manual_seed(1)).int()
    idx[0, :3] = torch.tensor([0, V - 1, V // 2])
    dy = torch.randn(1, R, 1, generator=torch.Generator().manual_seed(2))
    dt = torch.full((1, V, 1), float("nan"), device="cuda")
    ws = torch.empty(hb.embedding_bwd_sorted_workspace_bytes(1, R, V, 1), dtype=torch.uint8, device="cuda")
    hb.embedding_bwd_sorted(1, R, V, 1, 0, 0, dy.cuda(), idx.cuda(), None, 1.0, dt, ws)
    torch.cuda.synchronize()
    assert len(idx.unique()) == R
    at = idx[0].long().cuda()
    assert torch.equal(dt[0, at].cpu(), dy[0])
    dt[0, at] = 0
    for part in dt.view(-1).split(2 ** 28):
        assert bool((part == 0).all())


def test_absent_tokens_past_two_to_the_31_elements(hb):
    B, R, V, E = 2, 40, 1100000, 1024
    idx = torch.randint(0, V, (B, R), generator=torch.Generator().manual_seed(1)).int()
    idx[:, 20:] = V - 2                                     # the last row of each model's table is one of those that no token has
    dy = torch.randn(B, R, E, generator=torch.Generator().manual_seed(2)).cuda()
    dt = torch.full((B, V, E), float("nan"), device="cuda")
    ws = torch.empty(hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E), dtype=torch.uint8, device="cuda")
    hb.embedding_bwd_sorted(B, R, V, E, 0, 0, dy, idx.cuda(), None, 1.0, dt, ws)
    torch.cuda.synchronize()
    for b in range(B):
        at = idx[b].unique().long().cuda()
        assert bool(torch.isfinite(dt[b, at]).all())
        dt[b, at] = 0
        for part in dt[b].split(1 << 18):
            assert bool((part == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,R,V,E,text", [(2, 65537, 300, 5, False), (1, 65536, 70000, 8, True), (2, 200000, 70000, 4, False), (1, 131073, 1, 3, False),
                                          (3, 90001, 40000, 12, True)])
def test_many_rows(hb, dtype, B, R, V, E, text):
    """Tokens of up to 32 rows have the bits of an fp32 sum in order of the rows; longer ones are within n u of the 64-bit sum."""
    print(dtype, B, R, V, E, flush=True)
    g = torch.Generator().manual_seed(R)
    first, last = 3, R - 7
    off = torch.tensor([[first, first + 11, first + 11, last]] * B, dtype=torch.int32)
    idx = torch.randint(0, V, (B, R), generator=g)
    if text:                                                # half of the rows on a few tokens, the others spread
        idx = torch.where(torch.rand(B, R, generator=g) < 0.5, idx % 7 * (V // 7), idx)
    dy = torch.randn(B, R, E, generator=g).to(TDT[dtype])
    ws = torch.empty(hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E), dtype=torch.uint8, device="cuda").fill_(255)
    for o, lo, hi in ((off, first, last), (None, 0, R)):
        dt = torch.full((B, V, E), float("nan"), device="cuda")
        hb.embedding_bwd_sorted(B, R, V, E, 0 if o is None else 3, DT[dtype], dy.cuda(), idx.int().cuda(), None if o is None else o.cuda(), 1.5, dt, ws)
        torch.cuda.synchronize()
        got = dt.cpu()
        for b in range(B):
            at, rows = idx[b, lo:hi], dy[b, lo:hi].float()
            hits = torch.bincount(at, minlength=V)
            order = torch.argsort(at, stable=True)
            start = torch.cumsum(hits, 0) - hits
            acc = torch.zeros(V, E)
            for k in range(min(32, int(hits.max()))):
                v = (hits > k).nonzero()[:, 0]
                acc[v] += rows[order[start[v] + k]]
            few = hits <= 32
            assert torch.equal(got[b][few], (acc * 1.5)[few])
            want, mag = (torch.zeros(V, E, dtype=torch.float64).index_add_(0, at, x.double()) for x in (rows, rows.abs()))
            bound = 1.5 * mag * (hits[:, None] * 1.01 * pr.U) + 1.5 * want.abs() * pr.U
            assert bool(((got[b].double() - 1.5 * want).abs() <= bound).all())
