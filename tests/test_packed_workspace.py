"""The workspace of packed attention's backward: what serves the largest batch serves every smaller one (no GPU)."""
import itertools

import pytest


@pytest.fixture(scope="module")
def size():
    from paper_2102_02344_amd import binding
    return binding.attention_packed_bwd_workspace_bytes


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,Hq,Hkv,d", [(1, 4, 4, 64), (8, 4, 4, 64), (2, 8, 2, 128), (3, 6, 2, 48), (1, 1, 1, 1), (1, 32, 1, 128), (64, 16, 16, 100), (300, 12, 12, 64)])
def test_grows_with_rows_and_holds_for_any_sequences(size, dtype, B, Hq, Hkv, d):
    before = 0
    for R in sorted({1, 2, 31, 63, 64, 65, 127, 129, 1000, 4032, 4096, 8191, 70000, *range(1, 40000, 257)}):
        need = {size(B, R, nseq, Hq, Hkv, d, dtype) for nseq in (1, 2, 12, 30, R)}
        assert len(need) == 1
        (need,) = need
        assert need >= max(before, B * Hq * R * 4)
        before = need


@pytest.mark.parametrize("dtype", [0, 1])
def test_what_a_call_may_take(size, dtype):
    """D of every head and row, and fp32 sums of dk and dv for as many parts as give 2048 workgroups of 64 keys, up to eight: never less
    than that."""
    for B, Hkv, group, R, d in itertools.product((1, 2, 7), (1, 2, 5), (1, 4), (1, 64, 200, 4100, 16385, 70000), (1, 64, 128)):
        tiles = -(-R // 64) * B * Hkv
        parts = min(8, 2048 // tiles)
        need = B * Hkv * group * R * 4 + (parts * 2 * B * Hkv * R * d * 4 if parts > 1 else 0)
        assert size(B, R, 1, Hkv * group, Hkv, d, dtype) >= need
