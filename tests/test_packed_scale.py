"""Packed attention takes scores in base 2: a scale whose product with log2(e) is no fp32 number is refused before any launch (no GPU)."""
import ctypes as C

import pytest

ONE = C.c_void_p(256)              # never dereferenced
S3 = (C.c_int64 * 3)(4096, 64, 16)


@pytest.mark.parametrize("scale", [3.4e38, 2.4e38])
def test_scales_past_the_range(scale):
    from paper_2102_02344_amd import binding
    raw = binding.raw()
    assert raw.hfta_attention_packed_fwd(2, 64, 3, 4, 2, 16, 1, ONE, S3, ONE, ONE, S3, ONE, scale, 1, ONE, S3, ONE, None) == binding.EINVAL
    assert raw.hfta_attention_packed_bwd(2, 64, 3, 4, 2, 16, 1, ONE, S3, ONE, ONE, S3, ONE, scale, 1, ONE, ONE, S3, ONE, ONE, S3, ONE, ONE, S3,
                                         ONE, 1 << 30, None) == binding.EINVAL
