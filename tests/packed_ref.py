"""Plain 64-bit forms of the operators on packed sequences, with the bounds on rounding that their tests count.

Everything is torch on the CPU in float64.  ``u`` is half a step of fp32 (2^-24), ``e`` half a step of what the operator
stores (2^-8 for bf16)."""
import math

import torch

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}


def offsets(lengths, first=0):
    """lengths: one list per model -> int32 [B][nseq + 1]."""
    rows = []
    for n in lengths:
        at, row = first, [first]
        for x in n:
            at += x
            row.append(at)
        rows.append(row)
    return torch.tensor(rows, dtype=torch.int32)


def attention(q, k, v, off, scale, causal, dctx=None, dtype="f32"):
    """q, dctx [B, R, Hq, d], k, v [B, R, Hkv, d] (float64).  Returns values and bounds of the error that a kernel may
    have which holds scores and sums in fp32 and rounds what it feeds to a second product, and its outputs, to `dtype`:

    a score is a sum of d products (d + 2 roundings of its absolute terms), its exponential's argument is rounded where it is
    formed and where the maximum is taken from it, and the exponential itself and the running sum add a few more:
    p is off by a factor of at most 1 + ep.  The rounding of p (and ds) to bf16 adds e of each term of a product."""
    B, R, Hq, d = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    e = HALF[dtype]
    ein = e if dtype == "bf16" else 0.0
    out = {n: torch.zeros_like(q) for n in ("ctx", "ctx_b")}
    out["lse"], out["lse_b"] = (torch.zeros(B, Hq, R, dtype=torch.float64) for _ in range(2))
    for n, like in (("dq", q), ("dk", k), ("dv", v)):
        out[n], out[n + "_b"] = torch.zeros_like(like), torch.zeros_like(like)
    for b in range(B):
        for lo, hi in zip(off[b].tolist()[:-1], off[b].tolist()[1:]):
            n = hi - lo
            if n <= 0:
                continue
            mask = torch.ones(n, n, dtype=torch.bool).tril() if causal else torch.ones(n, n, dtype=torch.bool)
            for h in range(Hq):
                Q, K, V = q[b, lo:hi, h], k[b, lo:hi, h // G], v[b, lo:hi, h // G]
                x = (Q @ K.T * scale).masked_fill(~mask, -math.inf)
                xa = (Q.abs() @ K.abs().T * scale).masked_fill(~mask, 0.0)
                lse = torch.logsumexp(x, 1)
                p = torch.exp(x - lse[:, None])
                ctx = p @ V
                dx = (d + 6) * U * xa.amax(1) + 8 * U * (lse.abs() + xa.amax(1) + 1)
                ep = (2 * dx + (n + 8) * U)[:, None]
                ctx_b = (ep + ein * (1 + 2 * e) + n * U) * (p @ V.abs()) + e * ctx.abs() * (1 + 2 * e) + e * ein * (p @ V.abs())
                out["ctx"][b, lo:hi, h], out["ctx_b"][b, lo:hi, h] = ctx, ctx_b
                out["lse"][b, h, lo:hi], out["lse_b"][b, h, lo:hi] = lse, ep[:, 0] + 4 * U * lse.abs()
                if dctx is None:
                    continue
                g = dctx[b, lo:hi, h]
                dp, dpa = g @ V.T, g.abs() @ V.abs().T
                D, Da = (g * ctx).sum(1, keepdim=True), (g.abs() * ctx.abs()).sum(1, keepdim=True)
                Db = (g.abs() * ctx_b).sum(1, keepdim=True) + (d + 2) * U * Da
                ds = p * (dp - D)
                eq = 2 * ep + 4 * U * (lse.abs()[:, None] + 1)          # p formed again from the rounded lse
                ds_b = p * (Db + (d + 4) * U * dpa + 4 * U * Da) + (eq + ein * (1 + 2 * e)) * ds.abs()
                ds_b = ds_b * (1 + ein + eq)
                more = n * G * U                                        # sums over keys, or over queries and heads of a group
                out["dq"][b, lo:hi, h] = ds @ K * scale
                out["dq_b"][b, lo:hi, h] = scale * (ds_b @ K.abs() + more * (ds.abs() @ K.abs()))
                out["dk"][b, lo:hi, h // G] += ds.T @ Q * scale
                out["dk_b"][b, lo:hi, h // G] += scale * (ds_b.T @ Q.abs() + more * (ds.abs().T @ Q.abs()))
                out["dv"][b, lo:hi, h // G] += p.T @ g
                out["dv_b"][b, lo:hi, h // G] += ((p * (eq + ein * (1 + 2 * e) + more)).T @ g.abs())
    for n in ("dq", "dk", "dv"):                                        # the rounding of the output
        out[n + "_b"] = out[n + "_b"] * (1 + e) + (e + 2 * U) * out[n].abs() + 1e-30
    return out


def inside(off, R):
    """[B, R] truth values: whether a row lies in a sequence, and its place there."""
    B = off.shape[0]
    is_in, place = torch.zeros(B, R, dtype=torch.bool), torch.zeros(B, R, dtype=torch.long)
    for b in range(B):
        for lo, hi in zip(off[b].tolist()[:-1], off[b].tolist()[1:]):
            is_in[b, lo:hi] = True
            place[b, lo:hi] = torch.arange(hi - lo)
    return is_in, place


def row_logps(logits, labels):
    """float64 log-probability of each row's label (0 for a negative one)."""
    z = torch.log_softmax(logits, -1)
    t = z.gather(-1, labels.long().clamp(min=0)[..., None])[..., 0]
    return torch.where(labels >= 0, t, torch.zeros_like(t))


def seq_sums(x, off):
    return torch.stack([torch.stack([x[b, lo:hi].sum() for lo, hi in zip(off[b].tolist()[:-1], off[b].tolist()[1:])])
                        for b in range(x.shape[0])])


def preference(logits, labels, off, ref, beta, eps):
    """Loss [B] and summed log-probabilities [B, 2 pairs]; differentiable."""
    L = seq_sums(row_logps(logits, labels), off)
    gap = L - ref
    t = beta[:, None] * (gap[:, 0::2] - gap[:, 1::2])
    ls = torch.nn.functional.logsigmoid
    return (-(1 - eps[:, None]) * ls(t) - eps[:, None] * ls(-t)).mean(1), L


def preference_grad(logits, labels, off, ref, beta, eps):
    """The gradient of the sum of all models' losses, by formula."""
    _, L = preference(logits, labels, off, ref, beta, eps)
    gap = L - ref
    t = beta[:, None] * (gap[:, 0::2] - gap[:, 1::2])
    c = -beta[:, None] * ((1 - eps[:, None]) * torch.sigmoid(-t) - eps[:, None] * torch.sigmoid(t)) / t.shape[1]
    d = torch.zeros_like(logits)
    p = torch.softmax(logits, -1)
    for b in range(logits.shape[0]):
        o = off[b].tolist()
        for s in range(len(o) - 1):
            for r in range(o[s], o[s + 1]):
                y = int(labels[b, r])
                if y >= 0:
                    d[b, r] = -p[b, r]
                    d[b, r, y] += 1
                    d[b, r] *= c[b, s // 2] * (1 if s % 2 == 0 else -1)
    return d
