"""The plain 64-bit forms the packed operators are tested against: their gradients are the formula's, autograd's and what
differences of their values give.  And the operators' refusals, which come before any launch (no GPU)."""
import ctypes as C
import math

import pytest
import torch

import packed_ref as pr


def _normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("causal", [0, 1])
def test_attention_gradients(causal):
    B, R, Hq, Hkv, d = 2, 11, 4, 2, 3
    off = pr.offsets([[4, 0, 1, 5], [2, 7, 0, 1]])
    q, k, v, g = _normal(1, B, R, Hq, d), _normal(2, B, R, Hkv, d), _normal(3, B, R, Hkv, d), _normal(4, B, R, Hq, d)
    ref = pr.attention(q, k, v, off, 0.7, causal, g)
    val = lambda *t: (pr.attention(*t, off, 0.7, causal)["ctx"] * g).sum()
    h = 1e-5
    for n, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        t = [q, k, v]
        for at in torch.randperm(t[i].numel(), generator=torch.Generator().manual_seed(5))[:40].tolist():
            step = torch.zeros(t[i].numel(), dtype=torch.float64)
            step[at] = h
            step = step.view_as(t[i])
            up = val(*[x + step if j == i else x for j, x in enumerate(t)])
            dn = val(*[x - step if j == i else x for j, x in enumerate(t)])
            # a central difference is off by h^2/6 of the third derivative and 2^-53 |value| / h: below 1e-8 here
            assert abs(float(ref[n].reshape(-1)[at]) - float(up - dn) / (2 * h)) < 1e-7
    # torch's own derivative of a plain softmax over the same rows
    q, k, v = (x.clone().requires_grad_() for x in (q, k, v))
    total = 0
    for b in range(B):
        o = off[b].tolist()
        for lo, hi in zip(o[:-1], o[1:]):
            for hh in range(Hq):
                x = q[b, lo:hi, hh] @ k[b, lo:hi, hh // 2].T * 0.7
                if causal:
                    x = x.masked_fill(torch.ones(hi - lo, hi - lo, dtype=torch.bool).triu(1), -math.inf)
                total = total + (torch.softmax(x, 1) @ v[b, lo:hi, hh // 2] * g[b, lo:hi, hh]).sum()
    total.backward()
    for n, x in (("dq", q), ("dk", k), ("dv", v)):
        assert float((ref[n] - x.grad).abs().max()) < 1e-13


def test_preference_gradient():
    B, R, K = 2, 12, 7
    off = pr.offsets([[3, 4, 0, 2], [1, 5, 3, 3]])
    z = _normal(1, B, R, K) * 2
    y = torch.randint(0, K, (B, R), generator=torch.Generator().manual_seed(2)).int()
    y[:, ::3] = -1
    ref, beta, eps = _normal(3, B, 4) * 3 - 5, torch.tensor([0.3, 1.2]).double(), torch.tensor([0.0, 0.2]).double()
    d = pr.preference_grad(z, y, off, ref, beta, eps)
    zz = z.clone().requires_grad_()
    pr.preference(zz, y, off, ref, beta, eps)[0].sum().backward()
    assert float((zz.grad - d).abs().max()) < 1e-14
    h = 1e-5
    for at in range(0, z.numel(), 5):
        step = torch.zeros(z.numel(), dtype=torch.float64)
        step[at] = h
        step = step.view_as(z)
        up, dn = (pr.preference(z + s, y, off, ref, beta, eps)[0].sum() for s in (step, -step))
        assert abs(float(d.reshape(-1)[at]) - float(up - dn) / (2 * h)) < 1e-7


# ------------------------------------------------------------------ refusals
@pytest.fixture(scope="module")
def lib():
    from paper_2102_02344_amd import binding
    return binding


ONE = C.c_void_p(256)              # never dereferenced
S3 = (C.c_int64 * 3)(4096, 64, 16)


def test_attention_refusals(lib):
    raw = lib.raw()

    def fwd(B=2, R=64, nseq=3, Hq=4, Hkv=2, d=16, dt=1, Q=ONE, qs=S3, K=ONE, V=ONE, ks=S3, off=ONE, scale=0.25, ctx=ONE, cs=S3, lse=ONE):
        return raw.hfta_attention_packed_fwd(B, R, nseq, Hq, Hkv, d, dt, Q, qs, K, V, ks, off, scale, 1, ctx, cs, lse, None)
    for bad in (dict(B=0), dict(R=0), dict(nseq=0), dict(Hq=0), dict(Hkv=0), dict(d=0), dict(dt=2), dict(dt=-1), dict(Hq=3), dict(Q=None),
                dict(qs=None), dict(K=None), dict(V=None), dict(ks=None), dict(off=None), dict(ctx=None), dict(cs=None), dict(lse=None),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(R=2 ** 31 - 1)):
        assert fwd(**bad) == lib.EINVAL, bad
    assert fwd(d=129) == lib.EUNSUPPORTED
    assert fwd(B=2 ** 20, Hq=4096, R=2 ** 20) == lib.EUNSUPPORTED
    assert fwd(B=1, Hq=1, Hkv=1, R=2 ** 31 - 200) == lib.EUNSUPPORTED
    assert fwd(d=129, Q=None) == lib.EINVAL

    need = raw.hfta_attention_packed_bwd_workspace_bytes(2, 64, 3, 4, 2, 16, 1)
    assert need > 0 and raw.hfta_attention_packed_bwd_workspace_bytes(2, 64, 3, 4, 2, 129, 1) == 0
    assert raw.hfta_attention_packed_bwd_workspace_bytes(2, 64, 3, 3, 2, 16, 1) == 0

    def bwd(d=16, Hq=4, ptr=None, ws=ONE, nws=1 << 30):
        a = dict(Q=ONE, qs=S3, K=ONE, V=ONE, ks=S3, off=ONE, ctx=ONE, dctx=ONE, cs=S3, lse=ONE, dq=ONE, dqs=S3, dk=ONE, dv=ONE, dks=S3)
        if ptr:
            a[ptr] = None
        return raw.hfta_attention_packed_bwd(2, 64, 3, Hq, 2, d, 1, a["Q"], a["qs"], a["K"], a["V"], a["ks"], a["off"], 0.25, 1, a["ctx"],
                                             a["dctx"], a["cs"], a["lse"], a["dq"], a["dqs"], a["dk"], a["dv"], a["dks"], ws, nws, None)
    for p in ("Q", "qs", "K", "V", "ks", "off", "ctx", "dctx", "cs", "lse", "dq", "dqs", "dk", "dv", "dks"):
        assert bwd(ptr=p) == lib.EINVAL, p
    assert bwd(Hq=5) == lib.EINVAL
    assert bwd(d=200) == lib.EUNSUPPORTED
    assert bwd(ws=None) == lib.EWORKSPACE and bwd(nws=need - 1) == lib.EWORKSPACE and bwd(ws=C.c_void_p(258)) == lib.EWORKSPACE


def test_embedding_refusals(lib):
    raw = lib.raw()

    def fwd(B=2, R=64, V=100, E=24, nseq=3, dt=1, table=ONE, idx=ONE, off=ONE, pos=ONE, S=64, out=ONE):
        return raw.hfta_embedding_packed_fwd(B, R, V, E, nseq, dt, table, idx, off, 1.0, pos, S, out, None)
    for bad in (dict(B=0), dict(R=0), dict(V=0), dict(E=0), dict(nseq=0), dict(dt=3), dict(table=None), dict(idx=None), dict(off=None),
                dict(out=None), dict(S=0)):
        assert fwd(**bad) == lib.EINVAL, bad
    assert fwd(B=65536) == lib.EUNSUPPORTED and fwd(R=2 ** 28 + 1) == lib.EUNSUPPORTED and fwd(V=2 ** 30 + 1) == lib.EUNSUPPORTED

    need = raw.hfta_embedding_bwd_sorted_workspace_bytes(2, 64, 100, 24)
    assert need > 0 and raw.hfta_embedding_bwd_sorted_workspace_bytes(0, 64, 100, 24) == 0

    def bwd(B=2, R=64, V=100, E=24, nseq=3, dt=1, dy=ONE, idx=ONE, off=ONE, dtab=ONE, ws=ONE, nws=1 << 30):
        return raw.hfta_embedding_bwd_sorted(B, R, V, E, nseq, dt, dy, idx, off, 1.0, dtab, ws, nws, None)
    for bad in (dict(B=0), dict(R=0), dict(V=0), dict(E=0), dict(nseq=0), dict(dt=3), dict(dy=None), dict(idx=None), dict(dtab=None)):
        assert bwd(**bad) == lib.EINVAL, bad
    assert bwd(B=65536) == lib.EUNSUPPORTED
    assert bwd(ws=None) == lib.EWORKSPACE and bwd(nws=need - 1) == lib.EWORKSPACE and bwd(ws=C.c_void_p(264)) == lib.EWORKSPACE


def test_preference_refusals(lib):
    raw = lib.raw()

    def lps(B=2, R=64, K=100, nseq=4, dt=1, z=ONE, y=ONE, off=ONE, tok=ONE, out=ONE):
        return raw.hfta_seq_logps(B, R, K, nseq, dt, z, y, off, tok, out, None)
    for bad in (dict(B=0), dict(R=0), dict(K=0), dict(nseq=0), dict(dt=2), dict(z=None), dict(y=None), dict(off=None), dict(tok=None),
                dict(out=None)):
        assert lps(**bad) == lib.EINVAL, bad
    assert lps(B=65536) == lib.EUNSUPPORTED and lps(R=2 ** 24 - 1) == lib.EUNSUPPORTED

    need = raw.hfta_preference_loss_workspace_bytes(2, 64, 2)
    assert need > 0 and raw.hfta_preference_loss_workspace_bytes(2, 0, 2) == 0

    def loss(B=2, R=64, K=100, pairs=2, dt=1, ptr=None, ws=ONE, nws=1 << 30):
        a = dict(z=ONE, y=ONE, off=ONE, ref=ONE, beta=ONE, eps=ONE, loss=ONE, lp=ONE, dz=ONE)
        if ptr:
            a[ptr] = None
        return raw.hfta_preference_loss(B, R, K, pairs, dt, a["z"], a["y"], a["off"], a["ref"], a["beta"], a["eps"], a["loss"], a["lp"],
                                        a["dz"], ws, nws, None)
    for bad in (dict(B=0), dict(R=0), dict(K=0), dict(pairs=0), dict(dt=2), *[dict(ptr=p) for p in ("z", "y", "off", "ref", "beta", "loss", "lp", "dz")]):
        assert loss(**bad) == lib.EINVAL, bad
    assert loss(B=65536) == lib.EUNSUPPORTED
    assert loss(ws=None) == lib.EWORKSPACE and loss(nws=need - 1) == lib.EWORKSPACE and loss(ws=C.c_void_p(257)) == lib.EWORKSPACE


def test_too_many_sequences(lib):
    raw, many = lib.raw(), 2 ** 24 - 1
    assert raw.hfta_attention_packed_fwd(2, 64, many, 4, 2, 16, 1, ONE, S3, ONE, ONE, S3, ONE, 0.25, 1, ONE, S3, ONE, None) == lib.EUNSUPPORTED
    assert raw.hfta_attention_packed_bwd_workspace_bytes(2, 64, many, 4, 2, 16, 1) == 0
    assert raw.hfta_embedding_packed_fwd(2, 64, 100, 24, many, 1, ONE, ONE, ONE, 1.0, None, 0, ONE, None) == lib.EUNSUPPORTED
    assert raw.hfta_embedding_bwd_sorted(2, 64, 100, 24, many, 1, ONE, ONE, ONE, 1.0, ONE, ONE, 1 << 30, None) == lib.EUNSUPPORTED
    assert raw.hfta_seq_logps(2, 64, 100, many, 1, ONE, ONE, ONE, ONE, ONE, None) == lib.EUNSUPPORTED
    for pairs in (2 ** 23, 2 ** 31 - 1):
        assert raw.hfta_preference_loss(2, 64, 100, pairs, 1, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, 1 << 40, None) == lib.EUNSUPPORTED
        assert raw.hfta_preference_loss_workspace_bytes(2, 64, pairs) == 0
