"""The packed operators as they are used: one preference step of a small causal transformer array on packed pairs -- reference
log-probabilities, embedding, one layer (attention with grouped heads, feed-forward, residual LayerNorms), decoder, loss, and the
whole backward pass down to every parameter -- against autograd in 64 bits, B models one by one.

Tolerance: every operator of the chain holds 1e-5 (fp32) and 2e-2 (bf16, which rounds each stored tensor by 2^-8) of its
output's largest entry on its own; a gradient at the bottom has passed all of the twelve forward and the twelve backward calls, whose
errors add: 24e-5 of the largest entry in fp32.  In bf16 24 roundings of 2^-8 in a random walk and the two products' inner
ones give 2^-8 sqrt(24 + 6) = 2.2e-2 in the 2-norm; it is held to three times that."""
import math

import pytest
import torch

import packed_ref as pr
from util import DT, TDT

pytestmark = pytest.mark.gpu

B, E, Hq, Hkv, d, F, V, S = 2, 48, 4, 2, 12, 96, 203, 40
LENGTHS = [[17, 12, 0, 9, 33, 1], [5, 24, 20, 20, 2, 8]]
BEHIND = 6


@pytest.fixture(scope="module")
def hb():
    from paper_2102_02344_amd import binding
    return binding


def parameters(dtype):
    g = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g)
    W = (Hq + 2 * Hkv) * d
    p = dict(emb=n(B, V, E) / math.sqrt(E), inw=n(B, E, W) / math.sqrt(E), inb=n(B, W) * 0.1, outw=n(B, Hq * d, E) / math.sqrt(Hq * d),
             outb=n(B, E) * 0.1, ff1w=n(B, E, F) / math.sqrt(E), ff1b=n(B, F) * 0.1, ff2w=n(B, F, E) / math.sqrt(F), ff2b=n(B, E) * 0.1,
             decw=n(B, E, V) / math.sqrt(E), decb=n(B, V) * 0.1)
    p = {k: v.to(TDT[dtype]) for k, v in p.items()}
    for k in ("ln1", "ln2"):
        p[k + "w"], p[k + "b"] = 1 + 0.1 * n(B, E), 0.1 * n(B, E)
    return p


def oracle(p, tokens, labels, off, pos, ref, beta, eps):
    p = {k: v.double().requires_grad_() for k, v in p.items()}
    R = tokens.shape[1]
    is_in, place = pr.inside(off, R)
    logits = []
    for b in range(B):
        x = math.sqrt(E) * p["emb"][b][tokens[b].long()] + pos.double()[place[b]]
        qkv = x @ p["inw"][b] + p["inb"][b]
        ctx = torch.zeros(R, Hq * d, dtype=torch.float64)
        o = off[b].tolist()
        rows = []
        for lo, hi in zip(o[:-1], o[1:]):
            heads = []
            for h in range(Hq):
                q = qkv[lo:hi, h * d:(h + 1) * d]
                k, v = (qkv[lo:hi, (Hq + m * Hkv + h // (Hq // Hkv)) * d:][:, :d] for m in (0, 1))
                a = (q @ k.T / math.sqrt(d)).masked_fill(torch.ones(hi - lo, hi - lo, dtype=torch.bool).triu(1), -math.inf)
                heads.append(torch.softmax(a, 1) @ v)
            rows.append(torch.cat(heads, 1))
        ctx = torch.cat(rows + [ctx[o[-1]:]])
        ln = lambda t, k: torch.nn.functional.layer_norm(t, (E,), p[k + "w"][b], p[k + "b"][b], 1e-5)
        x = ln(x + ctx @ p["outw"][b] + p["outb"][b], "ln1")
        x = ln(x + torch.relu(x @ p["ff1w"][b] + p["ff1b"][b]) @ p["ff2w"][b] + p["ff2b"][b], "ln2")
        logits.append(x @ p["decw"][b] + p["decb"][b])
    loss, L = pr.preference(torch.stack(logits), labels, off, ref.double(), beta.double(), eps.double())
    loss.sum().backward()
    return loss.detach(), L.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_preference_step(hb, dtype):
    dt, tdt = DT[dtype], TDT[dtype]
    g = torch.Generator().manual_seed(5)
    off = pr.offsets(LENGTHS)
    R = int(off[:, -1].max()) + BEHIND
    tokens = torch.randint(0, V, (B, R), generator=g).int()
    tokens[:, ::4] = 7
    labels = torch.randint(0, V, (B, R), generator=g).int()
    labels[torch.rand(B, R, generator=g) < 0.3] = -1
    pos = torch.randn(S, E, generator=g) * 0.3
    beta, eps = torch.tensor([0.1, 0.5]), torch.tensor([0.0, 0.1])
    params = parameters(dtype)
    P = {k: v.cuda() for k, v in params.items()}
    G = {k: torch.empty(v.shape, device="cuda") for k, v in params.items()}
    act = lambda *s: torch.zeros(*s, dtype=tdt, device="cuda")          # rows behind the sequences are zeros, and stay zeros
    W, n, pairs = (Hq + 2 * Hkv) * d, len(LENGTHS[0]), len(LENGTHS[0]) // 2
    T, Y, O = tokens.cuda(), labels.cuda(), off.cuda()
    size, s, cs = (B, R, n, Hq, Hkv, d, dt), (R * W, W, d), (R * Hq * d, Hq * d, d)
    ws = torch.empty(max(16, hb.attention_packed_bwd_workspace_bytes(*size), hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E),
                         hb.preference_loss_workspace_bytes(B, R, pairs), hb.layernorm_bwd_workspace_bytes(B, R, E),
                         *[hb.linear_bwd_workspace_bytes(B, R, a, z, dt) for a, z in ((E, W), (Hq * d, E), (E, F), (F, E), (E, V))]),
                     dtype=torch.uint8, device="cuda")
    x, qkv, ctx, t, s1, x1, h, s2, x2, logits = (act(B, R, k) for k in (E, W, Hq * d, E, E, E, F, E, E, V))
    lse = torch.zeros(B, Hq, R, device="cuda")
    st = [torch.empty(B * R, device="cuda") for _ in range(4)]
    heads = lambda a: a.split([Hq * d, Hkv * d, Hkv * d], 2)
    hb.embedding_packed_fwd(B, R, V, E, n, dt, P["emb"], T, O, math.sqrt(E), pos.cuda(), S, x)
    hb.linear_fwd(B, R, E, W, dt, x, P["inw"], P["inb"], qkv)
    q, k, v = heads(qkv)
    hb.attention_packed_fwd(*size, q, s, k, v, s, O, 1 / math.sqrt(d), 1, ctx, cs, lse)
    hb.linear_fwd(B, R, Hq * d, E, dt, ctx, P["outw"], P["outb"], t)
    hb.add_layernorm_fwd(B, R, E, dt, x, t, s1, P["ln1w"], P["ln1b"], 1e-5, st[0], st[1], x1)
    hb.linear_fwd(B, R, E, F, dt, x1, P["ff1w"], P["ff1b"], h, hb.ACT_RELU)
    hb.linear_fwd(B, R, F, E, dt, h, P["ff2w"], P["ff2b"], t)
    hb.add_layernorm_fwd(B, R, E, dt, x1, t, s2, P["ln2w"], P["ln2b"], 1e-5, st[2], st[3], x2)
    hb.linear_fwd(B, R, E, V, dt, x2, P["decw"], P["decb"], logits)
    # the model as its own reference, a little off
    tok, ref = torch.zeros(B, R, device="cuda"), torch.empty(B, n, device="cuda")
    hb.seq_logps(B, R, V, n, dt, logits, Y, O, tok, ref)
    ref += torch.randn(B, n, generator=g).cuda()
    loss, logps, dlog = torch.empty(B, device="cuda"), torch.empty(B, n, device="cuda"), act(B, R, V)
    hb.preference_loss(B, R, V, pairs, dt, logits, Y, O, ref, beta.cuda(), eps.cuda(), loss, logps, dlog, ws)
    # backward
    da, ds2, dh, dh2, db_, ds1, dc, dqkv, dx, dsum = (act(B, R, z) for z in (E, E, F, F, E, E, Hq * d, W, E, E))
    hb.linear_bwd(B, R, E, V, dt, x2, P["decw"], dlog, da, G["decw"], G["decb"], ws)
    hb.layernorm_bwd(B, R, E, dt, s2, da, P["ln2w"], st[2], st[3], ds2, G["ln2w"], G["ln2b"], ws)
    hb.linear_bwd(B, R, F, E, dt, h, P["ff2w"], ds2, dh, G["ff2w"], G["ff2b"], ws)
    hb.act_bwd(B * R * F, dt, h, dh, dh2, hb.ACT_RELU, 0.0, 1)
    hb.linear_bwd(B, R, E, F, dt, x1, P["ff1w"], dh2, db_, G["ff1w"], G["ff1b"], ws)
    hb.add(B * R * E, dt, ds2, db_, da)
    hb.layernorm_bwd(B, R, E, dt, s1, da, P["ln1w"], st[0], st[1], ds1, G["ln1w"], G["ln1b"], ws)
    hb.linear_bwd(B, R, Hq * d, E, dt, ctx, P["outw"], ds1, dc, G["outw"], G["outb"], ws)
    dq, dk, dv = heads(dqkv)
    hb.attention_packed_bwd(*size, q, s, k, v, s, O, 1 / math.sqrt(d), 1, ctx, dc, cs, lse, dq, s, dk, dv, s, ws)
    hb.linear_bwd(B, R, E, W, dt, x, P["inw"], dqkv, dx, G["inw"], G["inb"], ws)
    hb.add(B * R * E, dt, ds1, dx, dsum)
    hb.embedding_bwd_sorted(B, R, V, E, n, dt, dsum, T, O, math.sqrt(E), G["emb"], ws)
    torch.cuda.synchronize()

    want, L, grads = oracle(params, tokens, labels, off, pos, ref.cpu(), beta, eps)
    tol = 24e-5 if dtype == "f32" else 6.6e-2
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm()) if dtype == "bf16" else float((a.double().cpu() - b).abs().max() / b.abs().max())
    assert rel(logps, L) <= tol and rel(loss, want) <= tol
    for name in sorted(grads):
        e = rel(G[name], grads[name])
        print(f"{dtype} {name}: {e:.2e}", flush=True)
        assert e <= tol, name
