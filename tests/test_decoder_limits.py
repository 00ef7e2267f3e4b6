"""How large calls of the operators of a decoder layer may be: launches below 2^24 workgroups and 2^32 threads are taken, whatever their
threads (no GPU: a workspace of no size is a refusal, and what else is wrong with a call is found first)."""
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2102_02344_amd import binding
    return binding


# columns, rows of a workgroup, its threads
@pytest.mark.parametrize("E,rows,threads", [(1, 32, 256), (64, 32, 256), (65, 8, 256), (256, 8, 256), (512, 4, 256), (513, 1, 128), (600, 1, 128),
                                            (1024, 1, 128), (1025, 1, 256), (2048, 1, 256), (4096, 1, 512), (4097, 1, 1024), (16384, 1, 1024)])
def test_rows_of_a_norm(lib, E, rows, threads):
    most = rows * min((1 << 24) - 1, ((1 << 32) - 1) // threads)
    need = lib.gated_residual_norm_bwd_workspace_bytes
    assert need(1, most, E) > 0 and need(65535, most, E) > 0
    assert need(1, most + 1, E) == 0 and need(65536, 8, E) == 0


def test_query_heads_of_linear_attention(lib):
    """2^21 - 1 query heads of all models, many of them on few key heads too."""
    import ctypes as C
    one, s3 = C.c_void_p(256), (C.c_int64 * 3)(1 << 30, 1 << 20, 16)
    raw = lib.raw()
    for B, Hq, Hkv in ((1, 4096, 1), (1, 5000, 4), (1, (1 << 20) - 1, 1), (3, 300000, 1), (2, 200000, 100)):
        f, b = (fn(B, 2000, 3, Hq, Hkv, 16, 1) for fn in (lib.linear_attention_fwd_workspace_bytes, lib.linear_attention_bwd_workspace_bytes))
        assert b > f > 0, (B, Hq, Hkv)
        # blocks of tiles as many as the launch has room for: their states, 32 x 32 fp32 of each key head
        assert f >= 4096 * B * Hkv * min(32, ((1 << 21) - 1) // (B * Hq), max(1, 512 // (B * Hkv))), (B, Hq, Hkv)
    for B, Hq, Hkv in ((1, 1 << 21, 1), (3, 700000, 1), (65535, 33, 33)):
        size = (B, 2000, 3, Hq, Hkv, 16, 1)
        assert lib.linear_attention_fwd_workspace_bytes(*size) == 0
        assert raw.hfta_linear_attention_fwd(*size, one, s3, one, one, s3, one, one, 1.0, None, one, s3, None, None, 0, None) == lib.EUNSUPPORTED
        assert raw.hfta_linear_attention_bwd(*size, one, s3, one, one, s3, one, one, 1.0, None, one, s3, None, one, s3, one, one, s3, None, None, 0,
                                             None) == lib.EUNSUPPORTED
