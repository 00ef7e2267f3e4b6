"""Plain 64-bit forms of the operators of a decoder layer with a recurrent memory, with the bounds on rounding that their tests count.

Everything is torch on the CPU in float64.  U is half a step of fp32 (2^-24), HALF half a step of what an operator stores (2^-8 for
bf16).  A bound is U times a count of roundings of the absolute terms of a sum, and half a step of the result where it is stored."""
import math

import numpy as np
import torch

from packed_ref import HALF, U, inside, offsets  # noqa: F401


def stored(value, bound, dtype):
    """The bound after rounding to `dtype`."""
    e = HALF[dtype]
    return bound * (1 + e) + (e if dtype == "bf16" else 0.0) * value.abs() + 1e-30


# ------------------------------------------------------------------ rotary positions
def rotary(x, pos, axis, freq, interleaved, rows, inverse=False):
    """x [B, R, H, d]; pos [B, R, naxes]; axis [pairs]; freq [B, pairs]; rows [B, R]: which are turned.  (values, bounds)"""
    pairs = freq.shape[1]
    a = pos.double()[:, :, axis.long()] * freq.double()[:, None]
    s = -1.0 if inverse else 1.0
    c, n = torch.cos(a)[:, :, None], s * torch.sin(a)[:, :, None]
    i = torch.arange(pairs)
    iu, iv = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    out, bound = x.clone(), torch.zeros_like(x)
    u, v = x[..., iu], x[..., iv]
    out[..., iu], out[..., iv] = u * c - v * n, v * c + u * n
    # the angle in turns, 64 bits: 3 roundings of 2^-53; the rest of a turn in fp32: pi U; sine and cosine 4 units in the last place (8 U); products
    # and their sum 3 U
    b = (16 * U + (a.abs() * 2.0 ** -50)[:, :, None]) * (u.abs() + v.abs())
    bound[..., iu], bound[..., iv] = b, b
    m = rows[..., None, None]
    return torch.where(m, out, x), torch.where(m, bound, torch.zeros_like(x))


# ------------------------------------------------------------------ linear attention
def linear_attention(q, k, v, off, log_decay, scale, s0=None, dctx=None, dsf=None):
    """q, dctx [B, R, Hq, d], k, v [B, R, Hkv, d], s0, dsf [B, nseq, Hkv, d, d]: by every pair of rows of a sequence."""
    B, R, Hq, d = q.shape
    Hkv, nseq = k.shape[2], off.shape[1] - 1
    G = Hq // Hkv
    lam = torch.exp(log_decay.double().clamp(max=0.0))
    out = dict(ctx=torch.zeros_like(q), state=torch.zeros(B, nseq, Hkv, d, d, dtype=torch.float64), dq=torch.zeros_like(q),
               dk=torch.zeros_like(k), dv=torch.zeros_like(v), ds0=torch.zeros(B, nseq, Hkv, d, d, dtype=torch.float64))
    for b in range(B):
        o = off[b].tolist()
        for i, (lo, hi) in enumerate(zip(o[:-1], o[1:])):
            n = hi - lo
            t = torch.arange(n, dtype=torch.float64)
            for h in range(Hkv):
                S0 = s0[b, i, h] if s0 is not None else torch.zeros(d, d, dtype=torch.float64)
                D = torch.where(t[:, None] >= t, lam[b, h] ** (t[:, None] - t).clamp(min=0), torch.zeros(()).double())
                up, down = (lam[b, h] ** (t + 1))[:, None], (lam[b, h] ** (n - 1 - t))[:, None]
                K, V = k[b, lo:hi, h], v[b, lo:hi, h]
                full = lam[b, h] ** n
                out["state"][b, i, h] = full * S0 + (K * down).T @ V
                if dsf is not None:
                    out["ds0"][b, i, h] += full * dsf[b, i, h]
                    out["dk"][b, lo:hi, h] += down * (V @ dsf[b, i, h].T)
                    out["dv"][b, lo:hi, h] += down * (K @ dsf[b, i, h])
                for g in range(h * G, (h + 1) * G):
                    Q = q[b, lo:hi, g] * scale
                    P = Q @ K.T * D
                    out["ctx"][b, lo:hi, g] = P @ V + up * (Q @ S0)
                    if dctx is None:
                        continue
                    dO = dctx[b, lo:hi, g]
                    dP = dO @ V.T * D
                    out["dq"][b, lo:hi, g] = scale * (dP @ K + up * (dO @ S0.T))
                    out["dk"][b, lo:hi, h] += dP.T @ Q
                    out["dv"][b, lo:hi, h] += P.T @ dO
                    out["ds0"][b, i, h] += (Q * up).T @ dO
    return out


def linear_attention_bounds(q, k, v, off, log_decay, scale, s0=None, dctx=None, dsf=None, dtype="f32"):
    """With A the same sums of absolute values: products of d terms and sums over the rows and heads of a sequence in fp32, a state that is
    multiplied by decays at most once a row, decays good to 8 U: (2 d + (2 + G) n + 40) U A.  bf16: what the first products and states
    put into the second ones is held in two bf16 words, 2^-16 each of at most three factors; the states that are returned in three."""
    a = lambda x: None if x is None else x.abs()
    A = linear_attention(a(q), a(k), a(v), off, log_decay, abs(scale), a(s0), a(dctx), a(dsf))
    d, G = q.shape[-1], q.shape[2] // k.shape[2]
    n = int((off[:, 1:] - off[:, :-1]).max())
    base = (2 * d + (2 + G) * n + 40) * U
    two = 3 * 2.0 ** -16 if dtype == "bf16" else 0.0
    return {m: (base + (0.0 if m in ("state", "ds0") else two)) * x for m, x in A.items()}


# ------------------------------------------------------------------ norms, gate and residual scale
def gated_norm(rms, x, f, gate, w1, b1, res, w2, b2, eps):
    def norm(z, w, b):
        if not rms:
            z = z - z.mean(-1, keepdim=True)
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps) * w[:, None]
        return z if b is None else z + b[:, None]
    s = x
    if f is not None:
        u = norm(f, w1, b1)
        if gate is not None:
            u = u * torch.sigmoid(gate)
        s = x + (u if res is None else res[:, None, None] * u)
    return s, norm(s, w2, b2)


def gated_norm_bounds(rms, x, f, gate, w1, b1, res, w2, b2, eps, ds, dy):
    """Bounds of s, y and the gradients, with a count C of roundings for each step: sums over a row of E elements are formed by 8 or 16
    per lane and a tree over at most 1024 (30 roundings), a handful of operations around them.  r is how much larger a row's largest
    entry is than its deviation, which is what subtracting the mean and dividing may magnify."""
    C = 60
    B, R, E = x.shape
    z = lambda a, like: torch.zeros_like(like) if a is None else a

    def unit(t):
        c = t if rms else t - t.mean(-1, keepdim=True)
        inv = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
        return c * inv, inv, inv * t.abs().amax(-1, keepdim=True) + 1

    def back(t, dt, hat, dhat, inv, rel):               # |bound| of inv (t - mean t - hat mean(t hat)); dt, dhat: bounds of t and hat; rel: of inv
        a = t.abs()
        m1, m2 = a.mean(-1, keepdim=True), (a * hat.abs()).mean(-1, keepdim=True)
        e = dt + dt.mean(-1, keepdim=True) + hat.abs() * (dt * hat.abs() + a * dhat).mean(-1, keepdim=True) + dhat * m2
        return inv * (e + (C * U + rel) * (a + m1 + hat.abs() * m2))

    def grad(t, hat, inv):
        t = t - hat * (t * hat).mean(-1, keepdim=True)
        return inv * (t if rms else t - t.mean(-1, keepdim=True))

    out = {}
    s, es = x, torch.zeros_like(x)
    if f is not None:
        fh, i1, r1 = unit(f)
        efh = C * U * r1 * (1 + fh.abs())
        u = fh * w1[:, None] + z(b1, w1)[:, None]
        eu = w1.abs()[:, None] * efh + 4 * U * ((fh * w1[:, None]).abs() + z(b1, w1).abs()[:, None])
        h = torch.ones_like(x) if gate is None else torch.sigmoid(gate)
        eh = torch.zeros_like(x) if gate is None else 8 * U * (1 + gate.abs()) * h
        a = (torch.ones(B, dtype=torch.float64) if res is None else res)[:, None, None]
        s = x + a * h * u
        es = a.abs() * (h * eu + eh * u.abs()) + 4 * U * (x.abs() + (a * h * u).abs())
    sh, i2, r2 = unit(s)
    me = es.amax(-1, keepdim=True) * i2                  # what an error of s does to its unit form
    esh = (C * U * r2 + 2 * me) * (1 + sh.abs())
    rel2 = C * U * r2 + 2 * me
    y = sh * w2[:, None] + z(b2, w2)[:, None]
    out["s"], out["y"] = es, w2.abs()[:, None] * esh + 4 * U * ((sh * w2[:, None]).abs() + z(b2, w2).abs()[:, None])
    t = dy * w2[:, None]
    dsm = z(ds, x) + grad(t, sh, i2)
    edsm = back(t, 2 * U * t.abs(), sh, esh, i2, rel2) + 4 * U * (z(ds, x).abs() + dsm.abs())
    out["dx"] = edsm
    n = (R + 60) * U                                     # sums over rows
    out["dw2"] = ((dy.abs() * esh).sum(1) + n * (dy * sh).abs().sum(1))
    out["db2"] = n * dy.abs().sum(1)
    if f is not None:
        du = a * h * dsm
        edu = a.abs() * (h * edsm + eh * dsm.abs()) + 4 * U * du.abs()
        v = du * w1[:, None]
        rel1 = C * U * r1
        out["df"] = back(v, edu * w1.abs()[:, None] + 2 * U * v.abs(), fh, efh, i1, rel1)
        out["dw1"] = (edu * fh.abs() + du.abs() * efh).sum(1) + n * (du * fh).abs().sum(1)
        out["db1"] = edu.sum(1) + n * du.abs().sum(1)
        hd = (h * dsm * u).abs()
        out["dres"] = (h * (edsm * u.abs() + dsm.abs() * eu) + eh * (dsm * u).abs()).sum((1, 2)) + (R + E + 60) * U * hd.sum((1, 2))
        out["dg"] = a.abs() * (hd * (1 - h) * 8 * U + (1 - h) * h * (edsm * u.abs() + dsm.abs() * eu) + eh * (dsm * u).abs() * 2 + 2 * U * hd)
    return out


# ------------------------------------------------------------------ the counter-based generator
def philox(counter, key):
    """Philox4x32-10: counter [n, 4], key (2 words) -> [n, 4] words, as Python's or numpy's whole numbers."""
    c = [np.asarray(counter[:, i], dtype=np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    m = np.uint64(0xffffffff)
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & m, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & m]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return np.stack(c, 1)


def keep(count, p, seed, site, step, first=0):
    """Whether elements first .. first + count - 1 of a model are kept."""
    lo, hi = first // 4, (first + count + 3) // 4
    i = np.arange(lo, hi, dtype=np.uint64)
    ctr = np.stack([i & np.uint64(0xffffffff), i >> np.uint64(32), np.full_like(i, site), np.full_like(i, step)], 1)
    w = philox(ctr, (seed & 0xffffffff, seed >> 32 & 0xffffffff)).reshape(-1)[first - 4 * lo:][:count]
    p = min(max(float(np.float32(p)), 0.0), 1.0)
    return torch.from_numpy(w.astype(np.float64) >= p * 2.0 ** 32)
