"""Gated residual norms where a workgroup of the backward call takes several rows: the next row on its way while one is computed, sums that
alternate between two places, gradients of weights held over rows, the gradient written in place of the one that came; every number of
threads a row can have.  The 64-bit form runs on the GPU here, in elementary operations."""
import pytest
import torch

import decoder_ref as dr
from test_gpu_gated_norm import EPS, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def check(c):
    h = lambda t: None if t is None else t.double()
    names = ("x", "f", "gate", "w1", "b1", "res", "w2", "b2")
    p = {n: h(getattr(c, n)) for n in names}
    q = {n: None if v is None else v.clone().requires_grad_() for n, v in p.items()}
    s, y = dr.gated_norm(c.rms, *[q[n] for n in names], EPS)
    ds, dy = h(c.ds), h(c.dy)
    (y * dy).sum().add(0.0 if ds is None else (s * ds).sum()).backward()
    want = dict(s=s.detach(), y=y.detach(), **{"d" + {"gate": "g"}.get(n, n): v.grad for n, v in q.items() if v is not None})
    bound = dr.gated_norm_bounds(c.rms, *[p[n] for n in names], EPS, ds, dy)
    for n in c.OUT:
        t = getattr(c, n)
        if t is None:
            continue
        b = dr.stored(want[n], bound[n], c.dtype if t.dtype == torch.bfloat16 else "f32")
        bad = (t.double().view(want[n].shape) - want[n]).abs() - b
        assert float(bad.max()) <= 0, (n, float(bad.max()), float(want[n].abs().max()))


# models, rows, columns: 8 and 32 lanes, a wavefront, 128 to 1024 threads, rows in two pieces a thread; a last row group that is not full
SIZES = [(24, 2101, 24), (24, 603, 200), (24, 301, 330), (24, 150, 520), (24, 101, 1500), (8, 101, 3001), (8, 101, 7777), (8, 71, 9001)]
FORMS = [dict(), dict(bias=False), dict(block=False), dict(block=False, bias=False, ds=False), dict(gate=False, ds=False)]


def rows_of_a_group(hb, B, R, E):
    """Rows that each row's threads take, at most: by the workgroups that the workspace has room for."""
    rows = 32 if E <= 64 else 8 if E <= 256 else 4 if E <= 512 else 1
    workgroups = hb.gated_residual_norm_bwd_workspace_bytes(B, R, E) // (B * (4 * E + 4) * 4)
    return -(-R // (workgroups * rows))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("size", SIZES)
def test_rows_one_after_another(hb, dtype, rms, form, size):
    assert rows_of_a_group(hb, *size) >= 2
    c = Case(*size, dtype, rms, seed=size[2] + form, **FORMS[form])
    c.fwd(hb)
    c.bwd(hb)
    check(c)
    if c.ds is not None:                                          # the gradient in place of the one that came, the same bits
        want = {n: getattr(c, n).clone() for n in c.OUT if getattr(c, n) is not None}
        c.dx = c.ds
        c.bwd(hb)
        for n, v in want.items():
            assert torch.equal(getattr(c, n), v), n
