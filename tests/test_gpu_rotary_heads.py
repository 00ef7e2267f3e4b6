"""Rotary positions where a workgroup takes several heads, one fetched as another is stored: head counts around the four in flight, heads split
over workgroups unevenly, whole pieces and single elements, pairs of both kinds, in place and not, with columns that are only copied."""
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


# 8 models of R rows, with as many rows as a workgroup of 256 threads takes at most: from 1024 workgroups on it has all heads, below it a part
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("pairs", [1, 3, 8])
@pytest.mark.parametrize("R,H", [(33000, 5), (33000, 7), (33000, 9), (20000, 9), (9000, 9), (12000, 11)])
def test_heads_one_after_another(hb, dtype, interleaved, pairs, R, H):
    B, d = 8, 16
    g = torch.Generator(device="cuda").manual_seed(R + H)
    off = torch.tensor([[3, 3 + R // 20 * b, R // 2, R // 2, R - 5 * b] for b in range(1, B + 1)], dtype=torch.int32)
    rows, place = dr.inside(off, R)
    rows, place = rows.cuda(), place[..., None].int().cuda()
    freq = (100.0 ** (-torch.arange(pairs).double() / pairs) * (1 + torch.arange(B).double()[:, None])).float().cuda()
    x = torch.randn(B, R, H, d, device="cuda", generator=g).to(TDT[dtype])
    s = (R * H * d, H * d, d)
    for inverse in (0, 1):
        value, bound = dr.rotary(x.double(), place, torch.zeros(pairs, dtype=torch.long, device="cuda"), freq, bool(interleaved), rows, bool(inverse))
        value = torch.where(rows[..., None, None], value, torch.full_like(value, MARK))
        y = torch.full_like(x, MARK)
        args = (None, 1, None, pairs, freq, interleaved, off.cuda(), inverse)
        hb.rotary_packed(B, R, 4, H, d, DT[dtype], x, s, *args, y, s)
        bad = (y.double() - value).abs() - dr.stored(value, bound, dtype)
        assert float(bad.max()) <= 0, (inverse, float(bad.max()), (bad > 0).nonzero()[:3].tolist())
        z = x.clone()
        hb.rotary_packed(B, R, 4, H, d, DT[dtype], z, s, *args, z, s)
        assert torch.equal(z, torch.where(rows[..., None, None], y, x)), (inverse, "in place")
