"""The table gradient by sorted tokens at the ends of what it takes: the largest number of tokens."""
import pytest
import torch

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
