"""Packed attention's backward on a workspace that was sized for more rows and other sequences: the bits of a call on its own, and nothing
written past the size that was asked for."""
import pytest
import torch

from test_gpu_packed_attention import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (4, 1, 128), (2, 2, 24)])
def test_one_workspace_for_all_batches(hb, dtype, Hq, Hkv, d):
    batches = [[4096], [64] * 64, [1000, 1000, 40], [30] * 33, [1], [700]]
    most = hb.attention_packed_bwd_workspace_bytes(1, max(map(sum, batches)), 7, Hq, Hkv, d, int(dtype == "bf16"))
    shared = torch.full((most + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    for n, lengths in enumerate(batches):
        print(dtype, Hq, Hkv, d, len(lengths), sum(lengths), flush=True)
        a, b = (Case(dtype, 1, [lengths], Hq, Hkv, d, seed=n) for _ in range(2))
        need = hb.attention_packed_bwd_workspace_bytes(*b.size)
        assert need <= most
        guarded = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
        a.ws, b.ws = shared[:most], guarded[:need]
        for c in (a, b):
            c.fwd(hb, 1)
            c.bwd(hb, 1)
        torch.cuda.synchronize()
        for (name, x), y in zip(a.outputs().items(), b.outputs().values()):
            assert torch.equal(x, y), name
        assert bool((shared[most:] == 0xa5).all()) and bool((guarded[need:] == 0xa5).all())
