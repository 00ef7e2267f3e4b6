"""Dropout by the counter-based generator: its mask word for word as the generator's definition gives it, at any size and alignment,
past 2^32 elements; values within their roundings; rates of none and all; a captured step that draws anew."""
import math

import pytest
import torch

import decoder_ref as dr
from util import DT, TDT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


SEEDS = [0x0123456789abcdef, 5, (1 << 63) - 1, 0, -2]


def scalars(p, seeds, step):
    return (torch.tensor(p, dtype=torch.float32, device="cuda"), torch.tensor(seeds, dtype=torch.int64, device="cuda"),
            torch.tensor([step], dtype=torch.int32, device="cuda"))


def check(y, x, p, seeds, site, step, dtype):
    for b in range(len(p)):
        keep = dr.keep(x.shape[1], p[b], seeds[b] % (1 << 64), site, step % (1 << 32))
        v = x[b].double().cpu()
        want = torch.where(keep, v / (1 - float(torch.tensor(p[b]).float().clamp(0, 1))), torch.zeros(()).double())
        # 1 - p, its inverse and the product: three roundings of fp32
        bad = (y[b].double().cpu() - want).abs() - dr.stored(want, 4 * dr.U * want.abs(), dtype)
        assert float(bad.max()) <= 0, (b, float(bad.max()))
        assert torch.equal(y[b].cpu() != 0, keep & (v != 0)), b


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 2, 3, 4, 5, 7, 8, 9, 63, 1001, 4096, 70001])
def test_mask_and_values(hb, dtype, count):
    p, B = [0.1, 0.5, 0.0, 0.999, 2.0 ** -30], 5
    pd, sd, st = scalars(p, SEEDS, -7)
    flat = torch.empty(B * count + 3, dtype=TDT[dtype], device="cuda").fill_(9.0)
    x = (torch.randn(B, count, generator=torch.Generator().manual_seed(count)) + 0.001).to(TDT[dtype]).cuda()
    y = flat[1:1 + B * count].view(B, count)                     # (an odd first element, and one behind the last that stays)
    hb.dropout_counter(B, count, DT[dtype], x, pd, sd, st, 0xfffffff0, y)
    check(y, x, p, SEEDS, 0xfffffff0, -7, dtype)
    assert float(flat[0]) == 9.0 and bool((flat[1 + B * count:] == 9.0).all())
    # the backward is the same call, in place too, and a model's mask is its own whatever is beside it
    z = x.clone()
    hb.dropout_counter(B, count, DT[dtype], z, pd, sd, st, 0xfffffff0, z)
    assert torch.equal(z, y)
    one = torch.empty(1, count, dtype=TDT[dtype], device="cuda")
    hb.dropout_counter(1, count, DT[dtype], x[1:2], pd[1:], sd[1:], st, 0xfffffff0, one)
    assert torch.equal(one, y[1:2])


def test_rates_at_the_ends(hb):
    p = [0.0, 1.0, -0.5, 1.5, math.nan]
    pd, sd, _ = scalars(p, SEEDS, 0)
    x = torch.randn(5, 100, generator=torch.Generator().manual_seed(1)).cuda()
    x[:, 7], x[:, 9] = math.nan, math.inf
    y = torch.empty_like(x)
    hb.dropout_counter(5, 100, 0, x, pd, sd, None, 3, y)
    assert torch.equal(y[0].nan_to_num(0.0), x[0].nan_to_num(0.0)) and torch.equal(y[2].nan_to_num(0.0), x[2].nan_to_num(0.0))
    assert not bool(y[1].any()) and not bool(y[3].any())         # what stands in dropped places does not matter
    assert bool(torch.isnan(y[4]).all())
    pd.fill_(0.5)
    hb.dropout_counter(5, 100, 0, x, pd, sd, None, 3, y)
    for b in range(5):
        keep = dr.keep(100, 0.5, SEEDS[b] % (1 << 64), 3, 0)
        assert torch.equal(torch.isfinite(y[b]).cpu(), torch.isfinite(x[b]).cpu() | ~keep)


def test_step_in_a_graph(hb):
    p, seeds, B, n = [0.3, 0.6], [11, 12], 2, 5000
    pd, sd, st = scalars(p, seeds, 1)
    x = (torch.randn(B, n, generator=torch.Generator().manual_seed(1)) + 0.001).cuda()
    y = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    hb.dropout_counter(B, n, 0, x, pd, sd, st, 4, y)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hb.dropout_counter(B, n, 0, x, pd, sd, st, 4, y)
        st.add_(1)
    for step in range(1, 5):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(y, x, p, seeds, 4, step, "f32")
    other = torch.cuda.Stream()
    z = torch.empty_like(x)
    torch.cuda.synchronize()
    hb.dropout_counter(B, n, 0, x, pd, sd, st, 4, z, other)
    torch.cuda.synchronize()
    check(z, x, p, seeds, 4, 5, "f32")


def test_past_2_32_elements(hb):
    n = (1 << 32) + 5
    x = torch.ones(2, n, dtype=torch.bfloat16, device="cuda")
    pd, sd, st = scalars([0.25, 0.5], [3, 4], 9)
    hb.dropout_counter(2, n, 1, x, pd, sd, st, 1, x)
    for b, p in ((0, 0.25), (1, 0.5)):
        for first in (0, (1 << 31) - 40, (1 << 32) - 77, n - 60):
            keep = dr.keep(60, p, 3 + b, 1, 9, first)
            assert torch.equal(x[b, first:first + 60].cpu() != 0, keep), (b, first)
    # of n independent draws the share kept is off by five of its deviations at most
    kept = float(sum((c != 0).sum() for c in x[1].split(1 << 28))) / n
    assert abs(kept - 0.5) < 5 * math.sqrt(0.25 / n)
