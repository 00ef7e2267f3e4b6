"""Rotary positions on packed rows against the 64-bit form, within its count of roundings: positions from the sequences and given,
one axis and several, pairs next to each other and halves apart, widths that fill pieces of 16 bytes and that do not, layouts
at any alignment, in place; far positions; rows of no sequence left as they were; graphs, other streams, tensors past 2^31 elements."""
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


def buffers(B, R, heads, d, dtype, layout):
    if layout == "heads":
        t = torch.full((B, heads, R, d), MARK, dtype=TDT[dtype], device="cuda").permute(0, 2, 1, 3)
    elif layout == "odd":
        hs, rs = d + 3, heads * (d + 3) + 5
        flat = torch.full((B * R * rs + 1,), MARK, dtype=TDT[dtype], device="cuda")
        t = flat[1:].as_strided((B, R, heads, d), (R * rs, rs, hs, 1), flat.storage_offset() + 1)
    else:
        t = torch.full((B, R, heads, d), MARK, dtype=TDT[dtype], device="cuda")
    s = t.stride()
    return t, (s[0], s[1], s[2])


def places(off, R):
    rows, place = dr.inside(off, R)
    return rows, place[..., None].int()


def compare(y, value, bound, dtype, what):
    bad = (y.double().cpu() - value).abs() - dr.stored(value, bound, dtype)
    assert float(bad.max()) <= 0, (what, float(bad.max()))


CASES = [  # B, lengths, first, behind, H, d, pairs, naxes
    (2, [[5, 0, 1, 20], [1, 1, 30, 2]], 2, 3, 3, 16, 8, 1),
    (1, [[300, 7, 260]], 0, 5, 2, 64, 32, 3),
    (3, [[1], [1], [1]], 0, 0, 12, 128, 64, 4),
    (2, [[9, 40], [30, 3]], 1, 0, 5, 40, 11, 2),
    (1, [[33]], 0, 0, 1, 7, 3, 1),
    (1, [[17, 2]], 0, 1, 9, 2, 1, 2),
    (2, [[70], [50]], 0, 0, 2, 300, 140, 1),
    (1, [[12]], 0, 0, 1, 1100, 550, 2),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_values_and_gradient(hb, dtype, interleaved, case):
    B, lengths, first, behind, H, d, pairs, naxes = CASES[case]
    g = torch.Generator().manual_seed(case)
    off = dr.offsets(lengths, first)
    R = int(off.max()) + behind
    rows, place = places(off, R)
    freq = (10000.0 ** (-torch.arange(pairs).double() / pairs) * (1 + torch.arange(B).double()[:, None])).float()
    axis = torch.randint(0, naxes, (pairs,), generator=g).int()
    given = naxes > 1
    pos = torch.randint(-50, 5000, (B, R, naxes), generator=g).int() if given else place
    for layout in ("rows", "heads", "odd"):
        x, xs = buffers(B, R, H, d, dtype, layout)
        x.copy_(torch.randn(B, R, H, d, generator=g))
        for inverse in (0, 1):
            for off_d in (off.cuda(), None):
                if off_d is None and not given:
                    p2, r2 = torch.arange(R).int()[None, :, None].expand(B, -1, 1), torch.ones_like(rows)
                else:
                    p2, r2 = pos, rows if off_d is not None else torch.ones_like(rows)
                value, bound = dr.rotary(x.double().cpu(), p2, axis, freq, bool(interleaved), r2, bool(inverse))
                value = torch.where(r2[..., None, None], value, torch.full_like(value, MARK))
                y, ys = buffers(B, R, H, d, dtype, layout)
                args = (pos.cuda() if given else None, naxes, axis.cuda() if given else None, pairs, freq.cuda(), interleaved, off_d, inverse)
                hb.rotary_packed(B, R, len(lengths[0]), H, d, DT[dtype], x, xs, *args, y, ys)
                compare(y, value, bound, dtype, (layout, inverse, off_d is None))
                z, zs = buffers(B, R, H, d, dtype, layout)
                z.copy_(x)
                hb.rotary_packed(B, R, len(lengths[0]), H, d, DT[dtype], z, zs, *args, z, zs)
                keep = torch.where(r2[..., None, None].cuda(), y, x)
                assert torch.equal(z, keep), (layout, "in place")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions_and_edges_of_axes(hb, dtype):
    B, R, H, d, pairs = 2, 37, 3, 32, 16
    g = torch.Generator().manual_seed(1)
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (B, R, 2), generator=g).int()
    pos[0, 0], pos[0, 1] = (1 << 31) - 1, -(1 << 31)
    freq = (10000.0 ** (-torch.arange(pairs).double() / pairs)).expand(B, -1).float().contiguous()
    axis = torch.randint(-3, 5, (pairs,), generator=g).int()           # taken into [0, 2)
    x, xs = buffers(B, R, H, d, dtype, "rows")
    x.copy_(torch.randn(B, R, H, d, generator=g))
    y, ys = buffers(B, R, H, d, dtype, "rows")
    value, bound = dr.rotary(x.double().cpu(), pos, axis.clamp(0, 1), freq, False, torch.ones(B, R, dtype=torch.bool))
    hb.rotary_packed(B, R, 0, H, d, DT[dtype], x, xs, pos.cuda(), 2, axis.cuda(), pairs, freq.cuda(), 0, None, 0, y, ys)
    # the angle's product of 31 and 24 bits is exact to 2^-53 of itself: up to 2^31 radians that is 2^-22, which the bound counts
    compare(y, value, bound, dtype, "far")


def test_values_that_are_not_finite_stay_in_their_pair(hb):
    x = torch.randn(1, 6, 2, 16, generator=torch.Generator().manual_seed(0)).cuda()
    x[0, 2, 1, 3], x[0, 4, 0, 9] = math.nan, math.inf
    freq = torch.full((1, 8), 0.3, device="cuda")
    y = torch.empty_like(x)
    s = (6 * 32, 32, 16)
    hb.rotary_packed(1, 6, 0, 2, 16, 0, x, s, None, 1, None, 8, freq, 0, None, 0, y, s)
    bad = torch.zeros(1, 6, 2, 16, dtype=torch.bool)
    bad[0, 2, 1, [3, 11]] = True
    bad[0, 4, 0, [1, 9]] = True
    assert torch.equal(~torch.isfinite(y).cpu(), bad)


def test_graph_and_streams(hb):
    B, R, H, d = 2, 500, 4, 64
    x = torch.randn(B, R, H, d, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    s = (R * H * d, H * d, d)
    freq = torch.rand(B, 32, generator=torch.Generator().manual_seed(3)).cuda()
    off = dr.offsets([[200, 250], [100, 399]]).cuda()
    y = torch.zeros_like(x)
    call = lambda out, stream=None: hb.rotary_packed(B, R, 2, H, d, 1, x, s, None, 1, None, 32, freq, 1, off, 0, out, s, stream)
    call(y)
    other, z = torch.cuda.Stream(), torch.zeros_like(x)
    torch.cuda.synchronize()
    call(z, other)
    graph, w = torch.cuda.CUDAGraph(), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(w)
    for n in range(3):
        w.zero_()
        x.copy_(torch.randn(B, R, H, d, generator=torch.Generator().manual_seed(2 + n)))
        graph.replay()
        torch.cuda.synchronize()
        if n == 0:
            assert torch.equal(y, z) and torch.equal(y, w)
        call(y.zero_())
        assert torch.equal(y, w)


def test_past_2_31_elements(hb):
    R, H, d = 300000, 60, 128
    x = torch.zeros(1, R, H, d, dtype=torch.bfloat16, device="cuda")
    x[0, -3:] = torch.randn(3, H, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    freq = (100.0 ** (-torch.arange(64).double() / 64)).float()[None]
    s = (R * H * d, H * d, d)
    tail = x[:, -3:].double().cpu()
    hb.rotary_packed(1, R, 0, H, d, 1, x, s, None, 1, None, 64, freq.cuda(), 0, None, 0, x, s)
    pos = torch.arange(R - 3, R).int()[None, :, None]
    value, bound = dr.rotary(tail, pos, torch.zeros(64, dtype=torch.long), freq, False, torch.ones(1, 3, dtype=torch.bool))
    compare(x[:, -3:], value, bound, "bf16", "tail")
    assert not bool(x[:, :-3].any())
