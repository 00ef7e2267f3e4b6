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
