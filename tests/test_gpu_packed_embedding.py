"""Embedding of packed sequences and its gradient by sorted tokens: positions that restart, any number of rows, tokens met
once and thousands of times, runs that end at and cross the stretches they are added in, row widths at any alignment."""
import math

import pytest
import torch

import packed_ref as pr
from util import DT, TDT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def lengths(B, R, nseq, seed):
    g = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(B):
        cut = torch.sort(torch.randint(0, R + 1, (nseq - 1,), generator=g)).values.tolist()
        at = [0] + cut + [R]
        out.append([z - a for a, z in zip(at[:-1], at[1:])])
    return out


def tokens(kind, B, R, V, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((B, R), V // 2, dtype=torch.int32)
    if kind == "padded":                        # half of the rows on one token
        i = torch.randint(0, V, (B, R), generator=g)
        i[:, R // 2:] = V - 1
        return i.int()
    if kind == "runs":                          # tokens met 1, 2, .. 70 times, shuffled
        i = torch.repeat_interleave(torch.arange(1, 71) * 3 % V, torch.arange(1, 71))
        return torch.stack([i[torch.randperm(R, generator=g) % len(i)] for _ in range(B)]).int()
    if kind == "outside":                       # some past both ends of the table
        return torch.randint(-3, V + 3, (B, R), generator=g).int()
    return torch.randint(0, V, (B, R), generator=g).int()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,B,R,V,E,nseq,first,behind", [
    ("uniform", 1, 1, 1, 1, 1, 0, 0), ("uniform", 2, 70, 9, 8, 3, 2, 5), ("outside", 2, 300, 256, 72, 7, 0, 1), ("runs", 2, 2485, 255, 40, 30, 1, 0),
    ("one", 1, 33, 5, 65, 2, 0, 0), ("one", 2, 5000, 70, 264, 3, 3, 9), ("padded", 2, 9000, 300, 256, 50, 0, 40), ("uniform", 1, 64, 65536, 12, 64, 0, 0),
    ("uniform", 3, 4097, 70000, 4, 200, 0, 3), ("padded", 1, 20000, 1000, 1028, 90, 0, 0), ("uniform", 1, 100, 17, 2050, 100, 0, 0),
    ("uniform", 2, 3000, 90, 16, 2500, 1, 2)])
def test_rows_and_gradients(hb, dtype, kind, B, R, V, E, nseq, first, behind):
    print(kind, dtype, B, R, V, E, nseq, flush=True)
    g = torch.Generator().manual_seed(R + E)
    off = pr.offsets(lengths(B, R, nseq, 3), first)
    R = R + first + behind
    is_in, place = pr.inside(off, R)
    idx = torch.nn.functional.pad(tokens(kind, B, R - first - behind, V, 5), (first, behind), value=1)
    S = max(1, int(place.max()) - 2)                      # the last places share a position
    table, pos, dy = torch.randn(B, V, E, generator=g).to(TDT[dtype]), torch.randn(S, E, generator=g), torch.randn(B, R, E, generator=g).to(TDT[dtype])
    at = idx.long().clamp(0, V - 1)
    for p in (pos, None):
        out = torch.full((B, R, E), 7.0, dtype=TDT[dtype], device="cuda")
        hb.embedding_packed_fwd(B, R, V, E, nseq, DT[dtype], table.cuda(), idx.cuda(), off.cuda(), 2.0, None if p is None else p.cuda(), S, out)
        ref = 2.0 * torch.stack([table[b][at[b]] for b in range(B)]).float()      # exact, so one rounding with the position and one more
        if p is not None:
            ref = ref + p[place.clamp(max=S - 1)]
        ref = torch.where(is_in[..., None], ref, torch.full_like(ref, 7.0)).to(TDT[dtype])
        assert torch.equal(out.cpu(), ref)
    dt = torch.full((B, V, E), float("nan"), device="cuda")
    ws = torch.empty(hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E), dtype=torch.uint8, device="cuda").fill_(255)
    for o in (off, None):
        hb.embedding_bwd_sorted(B, R, V, E, nseq if o is not None else 0, DT[dtype], dy.cuda(), idx.cuda(), None if o is None else o.cuda(), 1.5, dt, ws)
        torch.cuda.synchronize()
        took = is_in if o is not None else torch.ones_like(is_in)
        x = torch.where(took[..., None], dy.double(), 0.0)
        want, mag, hits = (torch.zeros(B, V, n, dtype=torch.float64) for n in (E, E, 1))
        for b in range(B):
            want[b].index_add_(0, at[b], x[b])
            mag[b].index_add_(0, at[b], x[b].abs())
            hits[b].index_add_(0, at[b], took[b].double()[:, None])
        # a sum of n terms in any order is off by at most (n - 1) u of their magnitudes, the factor 1.5 rounds once more
        bound = 1.5 * mag * (hits * 1.01 * pr.U) + 1.5 * want.abs() * pr.U
        got = dt.double().cpu()
        assert bool(((got - 1.5 * want).abs() <= bound).all()), float(((got - 1.5 * want).abs() - bound).max())
        assert bool((got[(hits == 0).expand_as(got)] == 0).all())


def test_same_bits_alone_twice_and_replayed(hb):
    B, R, V, E, nseq = 2, 6000, 900, 128, 20
    g = torch.Generator().manual_seed(7)
    off = pr.offsets(lengths(B, R, nseq, 3)).cuda()
    dy = torch.randn(B, R, E, generator=g).bfloat16().cuda()
    idx = tokens("padded", B, R, V, 9).cuda()
    other = tokens("uniform", B, R, V, 10).cuda()
    need = hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    dt = [torch.empty(B, V, E, device="cuda") for _ in range(2)]
    call = lambda i, k, s=None: hb.embedding_bwd_sorted(B, R, V, E, nseq, 1, dy, i, off, 1.0, dt[k], ws[k], s)
    want = []
    for i in (idx, other):
        call(i, 0)
        torch.cuda.synchronize()
        want.append(dt[0].clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k, i in enumerate((idx, other)):
        call(i, k, streams[k])
    torch.cuda.synchronize()
    assert torch.equal(dt[0], want[0]) and torch.equal(dt[1], want[1])
    live = idx.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(live, 0)
    for k in range(4):
        live.copy_((idx, other)[k % 2])
        graph.replay()
        call(other, 1)
        torch.cuda.synchronize()
        assert torch.equal(dt[0], want[k % 2]) and torch.equal(dt[1], want[1])


def test_past_two_to_the_31_elements(hb):
    """A table and its gradient of more than 2^31 elements: the last model's last rows."""
    B, R, V, E = 2, 40, 1100000, 1024
    idx = torch.randint(0, V, (B, R), generator=torch.Generator().manual_seed(1)).int()
    idx[1, 30:] = V - 1
    dy = torch.randn(B, R, E, generator=torch.Generator().manual_seed(2))
    dt = torch.empty(B, V, E, device="cuda")
    ws = torch.empty(hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E), dtype=torch.uint8, device="cuda")
    hb.embedding_bwd_sorted(B, R, V, E, 0, 0, dy.cuda(), idx.cuda(), None, 1.0, dt, ws)
    torch.cuda.synchronize()
    for b in range(B):
        for v in idx[b].unique().tolist():
            rows = dy[b][idx[b] == v].double()
            err = (dt[b, v].double().cpu() - rows.sum(0)).abs()
            assert bool((err <= len(rows) * pr.U * rows.abs().sum(0)).all())
    out = torch.empty(B, R, E, device="cuda")
    hb.embedding_packed_fwd(B, R, V, E, 1, 0, dt, idx.cuda(), torch.tensor([[0, R]] * B, dtype=torch.int32, device="cuda"), 1.0, None, 0, out)
    assert torch.equal(out[1, 31], dt[1, V - 1])
