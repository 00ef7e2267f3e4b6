"""The operators that a decoder layer with a recurrent memory is made of, for a fused array of language models, one by one.

A user of the library trains B models of one architecture as one job, on packed sequences: each model's R rows hold them
back to back, bounded by ``seq_offsets`` [B][nseq + 1], and rows behind the last one belong to none.  Tuned models then answer
prompts, token by token.  A case is one operator at one size; a pass is what a program calls for it:

``rotary``         query and key heads rotated in place of a packed projection, by positions along one or several axes
``linatt_train``   linear attention with a decay for each head over packed sequences, its forward and its backward
``linatt_prompt``  its forward over prompts, or pieces of them, from states to states
``linatt_step``    one token for each of the sequences in flight: states from a table of slots, and the new ones
``norm``           the block's norm, gate and residual scale, the sum with the residual stream and the next block's norm; and the gradients
``dropout``        dropout by a counter-based generator, a rate and a seed for each model; the same call is its own backward

Sizes follow the repository's language model array (8 models, 4 heads of 64 columns, 2048 tokens, width 256) and go from a few
rows to long sequences, wide rows and odd numbers of everything.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_CODE = {"f32": 0, "bf16": 1}
_EXACT_PAIRS = 1 << 34        # products of queries and keys that the 64-bit form does in well under 20 seconds
_M32 = 0xffffffff


def listed():
    return [
        # one new token of 16 sequences on two small models, full precision: launches and latency
        dict(name="rotary_step", op="rotary", dtype="f32", B=2, R=16, nseq=1, H=12, d=128, axes=3, interleaved=False, far=True),
        # patches of long videos: time, height and width
        dict(name="rotary_video", op="rotary", dtype="bf16", B=2, R=40000, nseq=3, H=10, d=128, axes=3, interleaved=False, far=False),
        # full precision, odd sizes, two query heads to a key head
        dict(name="linatt_train_f32", op="linatt_train", dtype="f32", B=3, R=777, nseq=5, Hq=6, Hkv=3, d=48),
        # the language model on packed text
        dict(name="linatt_train_lm", op="linatt_train", dtype="bf16", B=8, R=2048, nseq=12, Hq=4, Hkv=4, d=64),
        # long documents, wide heads
        dict(name="linatt_train_long", op="linatt_train", dtype="bf16", B=2, R=16384, nseq=3, Hq=8, Hkv=8, d=128),
        # prompts that go on from what came before them
        dict(name="linatt_prompt", op="linatt_prompt", dtype="bf16", B=2, R=4096, nseq=9, Hq=8, Hkv=8, d=128),
        # two models, a few sequences
        dict(name="linatt_step_few", op="linatt_step", dtype="bf16", B=2, n=3, slots=5, Hq=4, Hkv=4, d=64),
        # eight models, full batches, grouped heads
        dict(name="linatt_step_many", op="linatt_step", dtype="bf16", B=8, n=96, slots=128, Hq=16, Hkv=8, d=128),
        # a small array in full precision, odd rows, norms with means
        dict(name="norm_small", op="norm", dtype="f32", B=3, R=201, E=330, rms=False, gate=True),
        # wide rows, a gate computed from the tokens
        dict(name="norm_wide", op="norm", dtype="bf16", B=2, R=8192, E=2048, rms=True, gate=True),
        # a pooled vector's dropout in a small array, an odd number of elements
        dict(name="dropout_small", op="dropout", dtype="f32", B=3, count=8191),
        # activations of the language model's feed-forward blocks
        dict(name="dropout_lm", op="dropout", dtype="bf16", B=8, count=2048 * 1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "linatt_train", "linatt_train", "linatt_prompt", "linatt_step", "norm", "dropout"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    while True:
        c = dict(op=op, dtype=dtype, B=rng.choice((1, 2, 3, 4, 5, 8)))
        if op == "rotary":
            R = _log(rng, 1, 40000)
            c.update(R=R, nseq=max(1, R // _log(rng, 8, 2 * R + 8)), H=rng.randint(1, 12), d=rng.choice((16, 32, 40, 64, 64, 80, 96, 128, 128)),
                     axes=rng.choice((1, 1, 2, 3, 4)), interleaved=rng.random() < 0.5, far=rng.random() < 0.3)
            if c["B"] * R * c["H"] * c["d"] <= 1e8:
                return c
        elif op in ("linatt_train", "linatt_prompt"):
            Hkv, G = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 1, 1, 2, 4))
            R = _log(rng, 16, 16384)
            c.update(R=R, nseq=max(1, R // _log(rng, 8, 2 * R)), Hq=Hkv * G, Hkv=Hkv, d=rng.choice((16, 32, 40, 64, 64, 80, 96, 128, 128)))
            size = c["B"] * R * c["Hq"] * c["d"] * (1 if dtype == "bf16" else 4)
            states = c["B"] * c["nseq"] * Hkv * c["d"] ** 2
            if size <= 3.2e7 and c["B"] * c["nseq"] <= 400 and (op == "linatt_train" or states <= 3e7):
                return c
        elif op == "linatt_step":
            Hkv, G, n = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 1, 2, 4)), _log(rng, 1, 200)
            c.update(n=n, slots=n + _log(rng, 1, 50), Hq=Hkv * G, Hkv=Hkv, d=rng.choice((16, 32, 40, 64, 64, 80, 96, 128, 128)))
            if c["B"] * n * Hkv * c["d"] ** 2 <= 1e8:
                return c
        elif op == "norm":
            c.update(R=_log(rng, 1, 16384), E=rng.choice((8, 8, 8, 4, 1)) * _log(rng, 2, 512), rms=rng.random() < 0.6, gate=rng.random() < 0.7)
            if c["B"] * c["R"] * c["E"] <= 3.3e7:
                return c
        else:
            c.update(count=_log(rng, 1, 2048 * 1024))
            return c


def _lengths(c, seed):
    """Each model's sequence lengths: uneven, an empty one and one of a single token among them where there are several."""
    rng, out = random.Random(seed), []
    for _ in range(c["B"]):
        w = [rng.uniform(0.2, 1.0) for _ in range(c["nseq"])]
        used = c["R"] - (rng.randrange(c["R"] // 50 + 1) if c["nseq"] > 1 else 0)
        n = [int(used * x / sum(w)) for x in w]
        if c["nseq"] >= 4:
            i, j = rng.sample(range(c["nseq"]), 2)
            n[i], n[j] = 0, min(1, used)
        out.append(n)
    return out


def _offsets(lengths):
    return torch.tensor([[0] + list(np.cumsum(n)) for n in lengths], dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed + 1)
    dt, op, B = _DT[c["dtype"]], c["op"], c["B"]

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(scale).to(dtype)

    s = dict(c=c)
    if "nseq" in c:
        lengths = _lengths(c, seed)
        s["off"], s["longest"] = _offsets(lengths), max(1, max(max(n) for n in lengths))
    if op == "rotary":
        R, H, d, axes = c["R"], c["H"], c["d"], c["axes"]
        pairs = d // 2 if rng.random() < 0.7 else max(1, d // 4)
        s["x"] = normal(B, R, H + 2, d)                       # two more heads behind them (values) stay as they are
        s["y"] = s["x"].clone()
        base = torch.tensor([10000.0 * 2 ** rng.uniform(-1, 6) for _ in range(B)], dtype=torch.float64)[:, None]
        s["freq"] = (base ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().cuda()
        s["axis"] = (torch.arange(pairs, device="cuda") * axes // pairs).int() if rng.random() < 0.5 else (torch.arange(pairs, device="cuda") % axes).int()
        s["pos"] = None                                       # a row's place in its sequence
        if axes > 1 or c["far"]:
            top = 1000000 if c["far"] else 4096
            s["pos"] = torch.randint(0, top, (B, R, axes), device="cuda", generator=gen, dtype=torch.int32)
    elif op in ("linatt_train", "linatt_prompt"):
        R, Hq, Hkv, d, nseq = c["R"], c["Hq"], c["Hkv"], c["d"], c["nseq"]
        s["scale"] = 1.0 / math.sqrt(d)
        s["qkv"] = normal(B, R, (Hq + 2 * Hkv) * d)
        # memories of a few dozen up to some thousands of tokens, each model its own
        s["log_decay"] = torch.tensor([[math.log1p(-2.0 ** -(4 + 7 * rng.random())) for _ in range(Hkv)] for _ in range(B)], device="cuda")
        # what the calls write; rows behind the last sequence stay as they are
        s["ctx"] = torch.zeros(B, R, Hq * d, dtype=dt, device="cuda")
        if op == "linatt_train":
            s["dctx"], s["dqkv"] = normal(B, R, Hq * d), torch.zeros_like(s["qkv"])
        else:
            s["state"] = normal(B, nseq, Hkv, d, d, scale=3.0, dtype=torch.float32)
            s["new"] = torch.zeros_like(s["state"])
    elif op == "linatt_step":
        n, slots, Hq, Hkv, d = c["n"], c["slots"], c["Hq"], c["Hkv"], c["d"]
        s["scale"] = 1.0 / math.sqrt(d)
        s["qkv"] = normal(B, n, (Hq + 2 * Hkv) * d)
        s["log_decay"] = torch.tensor([[math.log1p(-2.0 ** -(4 + 7 * rng.random())) for _ in range(Hkv)] for _ in range(B)], device="cuda")
        s["state"] = normal(B, slots, Hkv, d, d, scale=3.0, dtype=torch.float32)
        s["new"] = torch.zeros_like(s["state"])
        s["ctx"] = torch.zeros(B, n, Hq * d, dtype=dt, device="cuda")
        order = torch.rand(B, slots, device="cuda", generator=gen).argsort(1)[:, :n].int()
        if n > 8:                                             # a place of the batch that no sequence holds now
            order[:, n // 2] = -1
        s["slot"] = order.contiguous()
    elif op == "norm":
        R, E = c["R"], c["E"]
        s["x"], s["f"], s["dy"], s["ds"] = normal(B, R, E, scale=2.0), normal(B, R, E), normal(B, R, E), normal(B, R, E)
        s["gate"] = normal(B, R, E) if c["gate"] else None
        s["w1"], s["w2"] = (1.0 + normal(B, E, scale=0.2, dtype=torch.float32) for _ in range(2))
        s["b1"], s["b2"] = (None if c["rms"] else normal(B, E, scale=0.2, dtype=torch.float32) for _ in range(2))
        s["res"] = 0.3 + torch.rand(B, device="cuda", generator=gen)
        s["eps"] = 1e-5
        for k in ("s", "y", "dx", "df"):
            s["out_" + k] = torch.empty_like(s["x"])
        s["out_dg"] = torch.empty_like(s["x"]) if c["gate"] else None
        s["stats"] = [torch.empty(B * R, device="cuda") for _ in range(4)]
        s["sums"] = [torch.empty(B, E, device="cuda") for _ in range(4)] + [torch.empty(B, device="cuda")]
    else:
        s["x"] = normal(B, c["count"])
        s["y"] = torch.empty_like(s["x"])
        s["p"] = torch.tensor([rng.choice((0.0, 0.1, 0.25, 0.5, rng.uniform(0.01, 0.6))) for _ in range(B)], device="cuda")
        s["seed"] = torch.tensor([rng.getrandbits(63) for _ in range(B)], dtype=torch.int64, device="cuda")
        s["step"] = torch.tensor([rng.getrandbits(31)], dtype=torch.int32, device="cuda")
        s["site"] = rng.getrandbits(16)
    return s


# ------------------------------------------------------------------ plain forms
def _places(s):
    """Of every row: whether it lies in a sequence, the sequence and the place in it."""
    off = s["off"].long()
    r = torch.arange(s["c"]["R"], device="cuda")
    seq = (off[:, 1:, None] <= r).sum(1)
    inside = (r >= off[:, :1]) & (r < off[:, -1:])
    seq = seq.clamp(max=off.shape[1] - 2)
    return inside, seq, torch.where(inside, r - off.gather(1, seq), 0)


def _rotary(s):
    c, x = s["c"], s["x"]
    B, R, H, d = c["B"], c["R"], c["H"], c["d"]
    inside, _, place = _places(s)
    pairs = s["freq"].shape[1]
    pos = place[..., None].expand(-1, -1, pairs) if s["pos"] is None else s["pos"].gather(2, s["axis"].long().expand(B, R, -1))
    angle = pos.double() * s["freq"].double()[:, None]                  # (far positions: angles that 32 bits lose)
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    z = x[:, :, :H].float()
    if c["interleaved"]:
        u, v = z[..., 0:2 * pairs:2], z[..., 1:2 * pairs:2]
    else:
        u, v = z[..., :pairs], z[..., pairs:2 * pairs]
    u, v = u * cos - v * sin, v * cos + u * sin
    w = torch.stack([u, v], -1).flatten(-2) if c["interleaved"] else torch.cat([u, v], -1)
    w = torch.cat([w, z[..., 2 * pairs:]], -1).to(x.dtype)
    out = x.clone()
    out[:, :, :H] = torch.where(inside[..., None, None], w, x[:, :, :H])
    return [out]


def _chunks(q, k, v, decay, state, chunk=256):
    """sum over t' <= t of decay^(t - t') (q_t . k_t') v_t', and decay^(t + 1) q_t . state: [.., H, L, d] rows, zeros behind the last, chunk by
    chunk with the state between them.  decay: logarithms [.., H, 1, 1]."""
    L, out = q.shape[-2], []
    for at in range(0, L, chunk):
        a, b, c = (x[..., at:at + chunk, :] for x in (q, k, v))
        n = a.shape[-2]
        t = torch.arange(n, device="cuda")
        gap = t[:, None] - t
        w = torch.where(gap >= 0, (decay * gap.clamp(min=0)).exp(), 0.0)
        up = (decay * (t[:, None] + 1)).exp()
        out.append((a @ b.transpose(-1, -2) * w) @ c + up * (a @ state))
        state = (decay * n).exp() * state + (b * (decay * (n - 1 - t[:, None])).exp()).transpose(-1, -2) @ c
    return torch.cat(out, -2)


def _linear_attention(s, train):
    """The sequences as a padded batch: [B, nseq, heads, longest, d], masked rows zero."""
    c, L = s["c"], s["longest"]
    B, R, H, G, d = c["B"], c["R"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    off = s["off"].long()
    nseq = off.shape[1] - 1
    t = torch.arange(L, device="cuda")
    length = off[:, 1:] - off[:, :-1]
    real = t < length[..., None]
    rows = (off[:, :-1, None] + t).clamp(max=R - 1).reshape(B, -1, 1)

    def padded(x, heads):                    # -> [B, nseq, heads, L, d]
        x = x.float().gather(1, rows.expand(-1, -1, x.shape[2])) * real.reshape(B, -1, 1)
        return x.view(B, nseq, L, heads, d).transpose(2, 3).contiguous()

    inside, seq, place = _places(s)
    back = (seq * L + place)[..., None]

    def packed(x):                           # [B, nseq, heads, L, d] -> [B, R, heads * d]
        x = x.transpose(2, 3).reshape(B, nseq * L, -1)
        return torch.where(inside[..., None], x.gather(1, back.expand(-1, -1, x.shape[2])), 0.0)

    q, k, v = s["qkv"].split([H * G * d, H * d, H * d], 2)
    q = padded(q, H * G) * s["scale"]
    k, v = (padded(x, H).repeat_interleave(G, 2) for x in (k, v))
    g = s["log_decay"].repeat_interleave(G, 1)[:, None, :, None, None]
    zero = torch.zeros(B, nseq, H * G, d, d, device="cuda")
    if not train:
        s0 = s["state"]
        ctx = _chunks(q, k, v, g, s0.repeat_interleave(G, 2))
        one, n = g[:, :, ::G], length[..., None, None, None]
        k, v = k[:, :, ::G], v[:, :, ::G]
        w = (one * (n - 1 - t[:, None]).clamp(min=0)).exp()
        new = (one * n).exp() * s0 + (k * w).transpose(-1, -2) @ v
        return [packed(ctx).to(s["qkv"].dtype), new]
    ctx = _chunks(q, k, v, g, zero)
    do = padded(s["dctx"], H * G)

    def later(a, b, c):                      # the same sums over later rows
        a, b, c = (x.flip(-2) for x in (a, b, c))
        return _chunks(a, b, c, g, zero).flip(-2).view(B, nseq, H, G, L, d).sum(3)

    dq = _chunks(do, v, k, g, zero) * s["scale"]
    dk, dv = later(v, do, q), later(k, q, do)
    return [packed(ctx).to(s["qkv"].dtype), torch.cat([packed(dq), packed(dk), packed(dv)], 2).to(s["qkv"].dtype)]


def _step(s):
    c = s["c"]
    B, n, H, G, d = c["B"], c["n"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    there = s["slot"] >= 0
    which = s["slot"].long().clamp(min=0)
    q, k, v = s["qkv"].float().split([H * G * d, H * d, H * d], 2)
    q, k, v = q.view(B, n, H, G, d), k.view(B, n, H, d, 1), v.view(B, n, H, 1, d)
    model = torch.arange(B, device="cuda")[:, None]
    state = s["log_decay"].exp()[:, None, :, None, None] * s["state"][model, which] + k * v
    ctx = (s["scale"] * (q @ state)).view(B, n, H * G * d)
    ctx = torch.where(there[..., None], ctx, 0.0).to(s["qkv"].dtype)
    new = s["new"].clone()
    new[model.expand(-1, n)[there], which[there]] = state[there]
    return [ctx, new]


def _norm(s):
    c, E = s["c"], s["c"]["E"]
    x, f, dy, ds = (s[k].float() for k in ("x", "f", "dy", "ds"))

    def unit(z):
        mean = 0.0 if c["rms"] else z.mean(-1, keepdim=True)
        inv = ((z - mean).square().mean(-1, keepdim=True) + s["eps"]).rsqrt()
        return (z - mean) * inv, inv

    def back(g, hat, inv):                   # the gradient of what unit() was given
        g = g - hat * (g * hat).mean(-1, keepdim=True)
        return inv * (g if c["rms"] else g - g.mean(-1, keepdim=True))

    def affine(hat, w, b):
        return hat * w[:, None] + (0.0 if b is None else b[:, None])

    def total(z):                            # (long sums)
        return z.double().sum(1).float()

    fh, i1 = unit(f)
    u = affine(fh, s["w1"], s["b1"])
    gate = 1 / (1 + (-s["gate"].float()).exp()) if c["gate"] else torch.ones((), device="cuda")
    res = s["res"][:, None, None]
    sm = x + res * gate * u
    sh, i2 = unit(sm)
    y = affine(sh, s["w2"], s["b2"])
    dsm = ds + back(dy * s["w2"][:, None], sh, i2)
    du = res * gate * dsm
    df = back(du * s["w1"][:, None], fh, i1)
    dt = s["x"].dtype
    out = [sm.to(dt), y.to(dt), dsm.to(dt), df.to(dt)]
    if c["gate"]:
        out.append((res * dsm * u * gate * (1 - gate)).to(dt))
    out += [total(du * fh), total(dy * sh), (dsm * gate * u).double().sum((1, 2)).float()]
    return out if c["rms"] else out + [total(du), total(dy)]


def _mulhilo(a, b):
    """High and low 32 bits of a constant times 32-bit words held in 64 bits."""
    low, high = (b & 0xffff) * a, (b >> 16) * a                    # both below 2^48
    total = low + ((high & 0xffff) << 16)
    return (high >> 16) + (total >> 32), total & _M32


def _dropout(s):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): element i takes word i % 4 of the block of counter (i / 4, site, step) under its model's key."""
    B, count = s["x"].shape
    i = torch.arange((count + 3) // 4, dtype=torch.int64, device="cuda").expand(B, -1)
    w = [i & _M32, i >> 32, torch.full_like(i, s["site"]), (s["step"].long() & _M32).expand_as(i)]
    k0, k1 = (s["seed"] & _M32)[:, None], (s["seed"] >> 32 & _M32)[:, None]
    for _ in range(10):
        h0, l0 = _mulhilo(0xD2511F53, w[0])
        h1, l1 = _mulhilo(0xCD9E8D57, w[2])
        w = [h1 ^ w[1] ^ k0, l1, h0 ^ w[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    word = torch.stack(w, -1).view(B, -1)[:, :count]
    keep = word.double() >= s["p"].double()[:, None] * 2.0 ** 32
    return [torch.where(keep, s["x"].float() * (1 / (1 - s["p"]))[:, None], 0.0).to(s["x"].dtype)]


def _plain(s):
    op = s["c"]["op"]
    if op == "rotary":
        return _rotary(s)
    if op in ("linatt_train", "linatt_prompt"):
        return _linear_attention(s, op == "linatt_train")
    return {"linatt_step": _step, "norm": _norm, "dropout": _dropout}[op](s)


# ------------------------------------------------------------------ the framework's calls
def _workspace(s, nbytes):
    """The scratch memory that a program keeps beside its buffers."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _framework(s):
    from paper_2102_02344_amd import binding as hb
    c = s["c"]
    B, op, dt = c["B"], c["op"], _CODE[c["dtype"]]
    if op == "rotary":
        R, H, d = c["R"], c["H"], c["d"]
        xs = (R * (H + 2) * d, (H + 2) * d, d)                # strides of model, row and head
        hb.rotary_packed(B, R, c["nseq"], H, d, dt, s["x"], xs, s["pos"], c["axes"], s["axis"], s["freq"].shape[1], s["freq"],
                         int(c["interleaved"]), s["off"], 0, s["y"], xs)
        return [s["y"]]
    if op in ("linatt_train", "linatt_prompt"):
        R, nseq, Hq, Hkv, d, width = c["R"], c["nseq"], c["Hq"], c["Hkv"], c["d"], s["qkv"].shape[2]
        size = (B, R, nseq, Hq, Hkv, d, dt)
        ins, cs = (R * width, width, d), (R * Hq * d, Hq * d, d)
        q, k, v = s["qkv"].split([Hq * d, Hkv * d, Hkv * d], 2)
        ws = _workspace(s, max(hb.linear_attention_fwd_workspace_bytes(*size), hb.linear_attention_bwd_workspace_bytes(*size)))
        hb.linear_attention_fwd(*size, q, ins, k, v, ins, s["off"], s["log_decay"], s["scale"], s.get("state"), s["ctx"], cs, s.get("new"), ws)
        if op == "linatt_prompt":
            return [s["ctx"], s["new"]]
        dq, dk, dv = s["dqkv"].split([Hq * d, Hkv * d, Hkv * d], 2)
        hb.linear_attention_bwd(*size, q, ins, k, v, ins, s["off"], s["log_decay"], s["scale"], None, s["dctx"], cs, None, dq, ins, dk, dv, ins,
                                None, ws)
        return [s["ctx"], s["dqkv"]]
    if op == "linatt_step":
        n, Hq, Hkv, d, width = c["n"], c["Hq"], c["Hkv"], c["d"], s["qkv"].shape[2]
        q, k, v = s["qkv"].split([Hq * d, Hkv * d, Hkv * d], 2)
        ins, cs = (n * width, width, d), (n * Hq * d, Hq * d, d)
        hb.linear_attention_step(B, n, c["slots"], Hq, Hkv, d, dt, q, ins, k, v, ins, s["slot"], s["log_decay"], s["scale"], s["state"], s["ctx"],
                                 cs, s["new"])
        return [s["ctx"], s["new"]]
    if op == "norm":
        R, E = c["R"], c["E"]
        kind = hb.NORM_RMS if c["rms"] else hb.NORM_LAYER
        m1, i1, m2, i2 = s["stats"]
        if c["rms"]:
            m1 = m2 = None
        hb.gated_residual_norm_fwd(B, R, E, dt, kind, s["x"], s["f"], s["gate"], s["w1"], s["b1"], s["res"], s["w2"], s["b2"], s["eps"],
                                   s["out_s"], s["out_y"], m1, i1, m2, i2)
        dw1, dw2, db1, db2, dres = s["sums"]
        if c["rms"]:
            db1 = db2 = None
        ws = _workspace(s, hb.gated_residual_norm_bwd_workspace_bytes(B, R, E))
        hb.gated_residual_norm_bwd(B, R, E, dt, kind, s["x"], s["f"], s["gate"], s["w1"], s["b1"], s["res"], s["w2"], m1, i1, m2, i2, s["ds"],
                                   s["dy"], s["out_dx"], s["out_df"], s["out_dg"], dw1, db1, dw2, db2, dres, ws)
        out = [s["out_s"], s["out_y"], s["out_dx"], s["out_df"]] + ([s["out_dg"]] if c["gate"] else []) + [dw1, dw2, dres]
        return out if c["rms"] else out + [db1, db2]
    hb.dropout_counter(B, c["count"], dt, s["x"], s["p"], s["seed"], s["step"], s["site"], s["y"])
    return [s["y"]]


def run(state):
    return _framework(state) if own else _plain(state)


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    B, op = c["B"], c["op"]
    if op == "rotary":
        return {"bytes": 2 * B * c["R"] * c["H"] * c["d"] * es + (B * c["R"] * c["axes"] * 4 if c["axes"] > 1 or c["far"] else 0),
                "flops": 3 * B * c["R"] * c["H"] * c["d"]}
    if op in ("linatt_train", "linatt_prompt"):
        # by the recurrence: a row's key adds d * d products to a state, a query takes as many from it
        qkv, ctx = B * c["R"] * (c["Hq"] + 2 * c["Hkv"]) * c["d"], B * c["R"] * c["Hq"] * c["d"]
        per = 2 * B * c["R"] * c["d"] ** 2
        if op == "linatt_prompt":
            return {"bytes": (qkv + ctx) * es + 8 * B * c["nseq"] * c["Hkv"] * c["d"] ** 2, "flops": per * (c["Hq"] + c["Hkv"])}
        return {"bytes": 2 * (qkv + ctx) * es, "flops": per * (3 * c["Hq"] + 3 * c["Hkv"])}
    if op == "linatt_step":
        rows = B * (c["n"] - (c["n"] > 8))
        return {"bytes": rows * (8 * c["Hkv"] * c["d"] ** 2 + 2 * (c["Hq"] + c["Hkv"]) * c["d"] * es), "flops": 2 * rows * (c["Hq"] + 1.5 * c["Hkv"]) * c["d"] ** 2}
    if op == "norm":
        # forward and backward: x, f, gate, ds, dy, and s, y, dx, df, dgate
        n = B * c["R"] * c["E"]
        return {"bytes": n * es * (10 if c["gate"] else 8), "flops": 40 * n}
    return {"bytes": 2 * B * c["count"] * es, "flops": 20 * B * c["count"]}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_rotary(s):
    """Each pair as a complex number times e^(i angle)."""
    c, off = s["c"], s["off"].tolist()
    n = s["freq"].shape[1]
    out = s["x"].double()
    cols = torch.arange(2 * n, device="cuda").view(n, 2) if c["interleaved"] else torch.arange(2 * n, device="cuda").view(2, n).T
    for b in range(c["B"]):
        for lo, hi in zip(off[b][:-1], off[b][1:]):
            if s["pos"] is None:
                pos = torch.arange(hi - lo, device="cuda", dtype=torch.float64)[:, None]
            else:
                pos = s["pos"][b, lo:hi][:, s["axis"].long()].double()
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos * s["freq"][b].double())
            for h in range(c["H"]):
                z = s["x"][b, lo:hi, h].double()
                z = torch.complex(z[:, cols[:, 0]], z[:, cols[:, 1]]) * turn
                out[b, lo:hi, h, cols[:, 0]], out[b, lo:hi, h, cols[:, 1]] = z.real, z.imag
    return [out]


def _exact_linear_attention(s, train):
    """Every pair of rows of a sequence, without chunks."""
    c = s["c"]
    H, G, d = c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    off, x = s["off"].tolist(), s["qkv"].double()
    ctx = torch.zeros(s["ctx"].shape, dtype=torch.float64, device="cuda")
    grad = torch.zeros_like(x)
    new = torch.zeros(s["new"].shape, dtype=torch.float64, device="cuda") if not train else None
    for b in range(c["B"]):
        for i, (lo, hi) in enumerate(zip(off[b][:-1], off[b][1:])):
            n = hi - lo
            t = torch.arange(n, device="cuda", dtype=torch.float64)
            for h in range(H):
                lam = math.exp(float(s["log_decay"][b, h]))
                decay = torch.pow(lam, (t[:, None] - t).clamp(min=0)).tril()
                kc, vc = (slice((H * G + m * H + h) * d, (H * G + m * H + h + 1) * d) for m in (0, 1))
                k, v = x[b, lo:hi, kc], x[b, lo:hi, vc]
                for hq in range(h * G, (h + 1) * G):
                    qc = slice(hq * d, (hq + 1) * d)
                    q = x[b, lo:hi, qc] * s["scale"]
                    p = q @ k.T * decay
                    ctx[b, lo:hi, qc] = p @ v
                    if train:
                        do = s["dctx"][b, lo:hi, qc].double()
                        dp = do @ v.T * decay
                        grad[b, lo:hi, vc] += p.T @ do
                        grad[b, lo:hi, kc] += dp.T @ q
                        grad[b, lo:hi, qc] = dp @ k * s["scale"]
                    else:
                        ctx[b, lo:hi, qc] += torch.pow(lam, t + 1)[:, None] * (q @ s["state"][b, i, h].double())
                if not train:
                    new[b, i, h] = lam ** n * s["state"][b, i, h].double()
                    if n:
                        new[b, i, h] += (k * decay[-1][:, None]).T @ v
    return [ctx, grad] if train else [ctx, new]


def _exact_step(s):
    c = s["c"]
    H, G, d = c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    x = s["qkv"].double()
    ctx, new = torch.zeros(s["ctx"].shape, dtype=torch.float64, device="cuda"), s["new"].double()
    for b in range(c["B"]):
        lam = s["log_decay"][b].double().exp()[:, None, None]
        for i, slot in enumerate(s["slot"][b].tolist()):
            if slot < 0:
                continue
            q, k, v = x[b, i].split([H * G * d, H * d, H * d])
            new[b, slot] = s["state"][b, slot].double() * lam + k.view(H, d, 1) * v.view(H, 1, d)
            ctx[b, i] = s["scale"] * torch.matmul(q.view(H, G, d), new[b, slot]).reshape(-1)
    return [ctx, new]


def _exact_norm(s):
    """The forward pass as it is defined, and its derivatives by differentiation."""
    c = s["c"]
    need = {k: s[k].double().requires_grad_() for k in ("x", "f", "w1", "w2", "res", "gate", "b1", "b2") if s[k] is not None}

    def norm(z, w, b):
        if not c["rms"]:
            z = z - z.mean(-1, keepdim=True)
        z = z / torch.sqrt(z.pow(2).mean(-1, keepdim=True) + s["eps"]) * w[:, None]
        return z if b is None else z + b[:, None]

    u = norm(need["f"], need["w1"], need.get("b1"))
    if c["gate"]:
        u = u * torch.sigmoid(need["gate"])
    total = need["x"] + need["res"][:, None, None] * u
    y = norm(total, need["w2"], need.get("b2"))
    keys = ["x", "f"] + (["gate"] if c["gate"] else []) + ["w1", "w2", "res"] + ([] if c["rms"] else ["b1", "b2"])
    grads = torch.autograd.grad([total, y], [need[k] for k in keys], [s["ds"].double(), s["dy"].double()])
    return [total.detach(), y.detach()] + list(grads)


def _exact_dropout(s):
    """The generator in 64-bit unsigned words on the host."""
    x = s["x"].double().cpu().numpy()
    B, count = x.shape
    out = np.zeros_like(x)
    mask = np.uint64(_M32)
    for b in range(B):
        key, p = int(s["seed"][b]), float(s["p"][b])
        block = np.arange((count + 3) // 4, dtype=np.uint64)
        a = [block & mask, block >> np.uint64(32), np.full_like(block, s["site"]), np.full_like(block, int(s["step"][0]) & _M32)]
        for r in range(10):
            ka, kb = np.uint64((key + r * 0x9E3779B9) & _M32), np.uint64(((key >> 32) + r * 0xBB67AE85) & _M32)
            m, n = a[0] * np.uint64(0xD2511F53), a[2] * np.uint64(0xCD9E8D57)
            a = [(n >> np.uint64(32)) ^ a[1] ^ ka, n & mask, (m >> np.uint64(32)) ^ a[3] ^ kb, m & mask]
        u = np.stack(a, 1).reshape(-1)[:count].astype(np.float64) / 2.0 ** 32
        kept = u >= p
        out[b, kept] = x[b, kept] / (1.0 - p)
    return [torch.from_numpy(out).cuda()]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    op = c["op"]
    if op == "rotary":
        return _exact_rotary(s) if c["B"] * c["nseq"] * c["H"] <= 20000 else None
    if op in ("linatt_train", "linatt_prompt"):
        if c["B"] * c["Hq"] * c["R"] ** 2 * 1.2 / c["nseq"] > _EXACT_PAIRS or c["B"] * c["nseq"] * c["Hq"] > 10000:
            return None
        return _exact_linear_attention(s, op == "linatt_train")
    return {"linatt_step": _exact_step, "norm": _exact_norm, "dropout": _exact_dropout}[op](s)
