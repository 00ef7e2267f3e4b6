"""The operators a fused array of language models needs to be tuned on packed sequences, one by one.

A user of the library trains B models of one architecture as one job.  Real text comes in sequences of different
lengths; packed, they lie back to back in each model's R rows, bounded by ``seq_offsets`` [B][nseq + 1], and rows
behind the last one belong to none.  A case is one operator at one size; a pass is its forward call, or the forward
and the backward call of a training step:

``attn``        attention over packed sequences with grouped heads: evaluation, and what activation recomputation runs
``attn_train``  its forward and its backward
``embed``       token embedding with positions that restart in every sequence, and the gradient of the table
``logps``       the log-probability of every token of an answer and their sum per sequence: what a reference model is asked for
``pref``        the loss of pairs of answers, one preferred, with the gradient of the logits

Sizes follow the repository's language model array (8 models, 4 heads of 64 columns, 2048 tokens, a vocabulary of
8192) and go from a few dozen tokens to long sequences, large tables and odd numbers of everything.
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


def listed():
    return [
        # a few short sequences on two small models: launches and latency
        dict(name="attn_small", op="attn", dtype="bf16", B=2, R=70, nseq=4, Hq=4, Hkv=4, d=64, causal=True),
        # long documents, four query heads to a key head
        dict(name="attn_long", op="attn", dtype="bf16", B=1, R=16384, nseq=2, Hq=8, Hkv=2, d=128, causal=True),
        # the repository's language model on packed text
        dict(name="attn_train_lm", op="attn_train", dtype="bf16", B=8, R=2048, nseq=12, Hq=4, Hkv=4, d=64, causal=True),
        # longer text, grouped heads of 128 columns
        dict(name="attn_train_gqa", op="attn_train", dtype="bf16", B=2, R=8192, nseq=3, Hq=8, Hkv=2, d=128, causal=True),
        # full precision, an encoder's attention, odd sizes
        dict(name="attn_train_f32", op="attn_train", dtype="f32", B=3, R=777, nseq=5, Hq=6, Hkv=2, d=48, causal=False),
        # a small model's table
        dict(name="embed_small", op="embed", dtype="f32", B=2, R=300, V=1000, E=72, nseq=4),
        # the language model's table under a larger batch
        dict(name="embed_lm", op="embed", dtype="bf16", B=8, R=8192, V=8192, E=256, nseq=48),
        # a large vocabulary, wide rows, many tokens
        dict(name="embed_large", op="embed", dtype="bf16", B=2, R=60000, V=32001, E=1024, nseq=100),
        # a small reference model in full precision
        dict(name="logps_small", op="logps", dtype="f32", B=3, R=200, K=1000, pairs=4),
        # the language model as its own reference
        dict(name="logps_lm", op="logps", dtype="bf16", B=8, R=2048, K=8192, pairs=16),
        # a preference step of the language model
        dict(name="pref_lm", op="pref", dtype="bf16", B=8, R=2048, K=8192, pairs=16),
        # a large vocabulary of odd size: rows that begin at any element
        dict(name="pref_large", op="pref", dtype="bf16", B=4, R=4096, K=32001, pairs=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn", "attn_train", "embed", "logps", "pref"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    while True:
        c = dict(op=op, dtype=dtype, B=rng.choice((1, 2, 3, 4, 5, 8)))
        if op in ("attn", "attn_train"):
            Hkv, G = rng.choice((1, 2, 3, 4)), rng.choice((1, 1, 2, 4))
            R = _log(rng, 16, 8192)
            c.update(R=R, nseq=max(1, R // _log(rng, 8, 2 * R)), Hq=Hkv * G, Hkv=Hkv, d=rng.choice((16, 32, 40, 64, 64, 80, 96, 128, 128)),
                     causal=rng.random() < 0.75)
            pairs = c["B"] * c["Hq"] * c["R"] ** 2 / c["nseq"] * c["d"]
            if pairs <= (2e10 if dtype == "bf16" else 5e9):
                return c
        elif op == "embed":
            R = _log(rng, 16, 60000)
            c.update(R=R, V=_log(rng, 50, 32001), E=8 * _log(rng, 1, 128) + rng.choice((0, 0, 0, 4, 1)), nseq=max(1, R // _log(rng, 16, 2 * R)))
            if c["B"] * (c["R"] + c["V"]) * c["E"] <= 1.5e8 and c["nseq"] <= 1000:
                return c
        else:
            pairs = _log(rng, 1, 40)
            c.update(R=max(_log(rng, 16, 8192), 4 * pairs), K=_log(rng, 33, 40000), pairs=pairs)
            if c["B"] * c["R"] * c["K"] <= 3e8:
                return c


def _lengths(c, seed):
    """Each model's sequence lengths: uneven, an empty one and one of a single token among them where there are several."""
    rng, out = random.Random(seed), []
    nseq = c.get("nseq") or 2 * c["pairs"]
    for _ in range(c["B"]):
        w = [rng.uniform(0.2, 1.0) for _ in range(nseq)]
        used = c["R"] - (rng.randrange(c["R"] // 50 + 1) if nseq > 1 else 0)
        n = [int(used * x / sum(w)) for x in w]
        if nseq >= 4:
            i, j = rng.sample(range(nseq), 2)
            n[i], n[j] = 0, min(1, used)
        out.append(n)
    return out


def _offsets(lengths):
    return torch.tensor([[0] + list(np.cumsum(n)) for n in lengths], dtype=torch.int32, device="cuda")


def _zipf(shape, n, seed, gen):
    """Token numbers with the frequencies of text (1 / rank), the ranks spread over the vocabulary."""
    u = torch.rand(shape, device="cuda", generator=gen, dtype=torch.float64)
    rank = torch.exp(u * math.log(n + 1.0)).long().sub_(1).clamp_(0, n - 1)
    return torch.from_numpy(np.random.default_rng(seed).permutation(n)).cuda()[rank].to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[c["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(scale).to(dtype)

    lengths = _lengths(c, seed)
    s = dict(c=c, off=_offsets(lengths), longest=max(1, max(max(n) for n in lengths)))
    B, R = c["B"], c["R"]
    if c["op"] in ("attn", "attn_train"):
        width = (c["Hq"] + 2 * c["Hkv"]) * c["d"]
        s["scale"] = 1.0 / math.sqrt(c["d"])
        s["qkv"] = normal(B, R, width)
        # what the calls write; rows behind the last sequence stay as they are
        s["ctx"] = torch.zeros(B, R, c["Hq"] * c["d"], dtype=dt, device="cuda")
        s["lse"] = torch.zeros(B, c["Hq"], R, device="cuda")
        if c["op"] == "attn_train":
            s["dctx"] = normal(B, R, c["Hq"] * c["d"])
            s["dqkv"] = torch.zeros_like(s["qkv"])
    elif c["op"] == "embed":
        V, E = c["V"], c["E"]
        s["table"], s["pos"], s["dy"] = normal(B, V, E), normal(s["longest"], E, dtype=torch.float32), normal(B, R, E)
        s["idx"] = _zipf((B, R), V, seed, gen)
        s["scale"] = math.sqrt(E)
        s["out"] = torch.zeros(B, R, E, dtype=dt, device="cuda")
        s["dtable"] = torch.empty(B, V, E, device="cuda")
    else:
        K, n = c["K"], 2 * c["pairs"]
        s["logits"] = normal(B, R, K, scale=2.0)
        labels = torch.randint(0, K, (B, R), device="cuda", generator=gen, dtype=torch.int32).cpu().numpy()
        rng = random.Random(seed + 1)
        for b in range(B):       # the prompt at the head of each sequence and the rows behind the last one have no label
            at = 0
            for m in lengths[b]:
                labels[b, at:at + int(m * rng.uniform(0.1, 0.7))] = -1
                at += m
            labels[b, at:] = -1
        s["labels"] = torch.from_numpy(labels).cuda()
        s["logps"] = torch.empty(B, n, device="cuda")
        if c["op"] == "logps":
            s["tokens"] = torch.zeros(B, R, device="cuda")
        else:
            s["beta"] = torch.tensor([0.05 + 0.1 * rng.random() for _ in range(B)], device="cuda")
            s["smoothing"] = torch.tensor([rng.choice((0.0, 0.1)) for _ in range(B)], device="cuda")
            s["ref"] = (_sequence_logps(s) + 5.0 * torch.randn(B, n, device="cuda", generator=gen)).float()
            s["loss"] = torch.empty(B, device="cuda")
            s["dlogits"] = torch.zeros_like(s["logits"])
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


def _attention(s, train):
    """The sequences as a padded batch: [B, nseq, longest] rows, masked scores, products, and the rows back in place."""
    c, L = s["c"], s["longest"]
    B, R, H, G, d = c["B"], c["R"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    off = s["off"].long()
    nseq = off.shape[1] - 1
    t = torch.arange(L, device="cuda")
    real = t < (off[:, 1:] - off[:, :-1])[..., None]
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
    q = padded(q, H * G).view(B, nseq, H, G * L, d)
    k, v = padded(k, H), padded(v, H)
    mask = real[:, :, None, None, :]
    if c["causal"]:
        mask = mask & (t <= t[:, None])
    mask = mask[:, :, None].expand(-1, -1, 1, G, L, -1)         # [B, nseq, 1, G, L, L]
    x = (q @ k.transpose(-1, -2)).mul_(s["scale"]).view(B, nseq, H, G, L, L).masked_fill_(~mask, -math.inf)
    top = x.amax(-1, keepdim=True).clamp_(min=-1e30)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (top + total.clamp(min=1e-30).log()).view(B, nseq, H * G, L, 1)
    p = x.div_(total.clamp_(min=1e-30)).view(B, nseq, H, G * L, L)
    ctx = (p @ v).view(B, nseq, H * G, L, d)
    out = [packed(ctx).to(s["qkv"].dtype), packed(lse).transpose(1, 2).contiguous()]
    if train:
        do = padded(s["dctx"], H * G).view(B, nseq, H, G * L, d)
        dv = p.transpose(-1, -2) @ do
        dp = do @ v.transpose(-1, -2)
        ds = dp.sub_((dp * p).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
        dq, dk = (ds @ k).view(B, nseq, H * G, L, d), ds.transpose(-1, -2) @ q
        out.append(torch.cat([packed(dq), packed(dk), packed(dv)], 2).to(s["qkv"].dtype))
    return out


def _embedding(s):
    c = s["c"]
    inside, _, place = _places(s)
    idx = s["idx"].long()
    out = s["scale"] * s["table"].float().gather(1, idx[..., None].expand(-1, -1, c["E"])) + s["pos"][place]
    out = torch.where(inside[..., None], out, 0.0).to(s["table"].dtype)
    # (frequent tokens are long sums)
    flat = (torch.arange(c["B"], device="cuda")[:, None] * c["V"] + idx).view(-1)
    dy = torch.where(inside[..., None], s["dy"].double(), 0.0).view(-1, c["E"])
    dt = torch.zeros(c["B"] * c["V"], c["E"], dtype=torch.float64, device="cuda").index_add_(0, flat, dy)
    return [out, (s["scale"] * dt).float().view(c["B"], c["V"], c["E"])]


def _rows(s):
    """Log-softmax of every row's label (0 without one), and what the gradient needs."""
    z = s["logits"].float()
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(-1, keepdim=True)
    y = s["labels"].long()
    term = z.gather(2, y.clamp(min=0)[..., None]) - top - total.log()
    return torch.where(y >= 0, term[..., 0], 0.0), e, total


def _sequence_sums(s, terms):
    """Sums over each sequence's rows, in 64 bits: they are long, and the loss takes differences of them."""
    inside, seq, _ = _places(s)
    n = s["off"].shape[1] - 1
    return torch.zeros(terms.shape[0], n, dtype=torch.float64, device="cuda").scatter_add_(1, seq, torch.where(inside, terms.double(), 0.0))


def _sequence_logps(s):
    return _sequence_sums(s, _rows(s)[0])


def _preference(s):
    c = s["c"]
    terms, e, total = _rows(s)
    logps = _sequence_sums(s, terms)
    gap = logps - s["ref"].double()
    beta, eps = s["beta"].double()[:, None], s["smoothing"].double()[:, None]
    t = beta * (gap[:, 0::2] - gap[:, 1::2])

    def softplus(x):
        return x.clamp(min=0) + (-x.abs()).exp().log1p()

    loss = ((1 - eps) * softplus(-t) + eps * softplus(t)).mean(1)
    coef = -beta * ((1 - eps) / (1 + t.exp()) - eps / (1 + (-t).exp())) / c["pairs"]
    coef = torch.stack([coef, -coef], 2).view(c["B"], -1)
    inside, seq, _ = _places(s)
    coef = torch.where(inside & (s["labels"] >= 0), coef.gather(1, seq), 0.0).float()[..., None]
    y = s["labels"].long().clamp(min=0)[..., None]
    d = e.div_(total).neg_().scatter_add_(2, y, torch.ones_like(coef)).mul_(coef)
    return [loss.float(), logps.float(), d.to(s["logits"].dtype)]


def _plain(s):
    op = s["c"]["op"]
    if op in ("attn", "attn_train"):
        return _attention(s, op == "attn_train")
    if op == "embed":
        return _embedding(s)
    if op == "logps":
        terms = _rows(s)[0]
        return [terms, _sequence_sums(s, terms).float()]
    return _preference(s)


# ------------------------------------------------------------------ the framework's calls
def _workspace(s, nbytes):
    """The scratch memory that a program keeps beside its buffers."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _framework(s):
    from paper_2102_02344_amd import binding as hb
    c = s["c"]
    B, R, op, dt = c["B"], c["R"], c["op"], _CODE[c["dtype"]]
    if op in ("attn", "attn_train"):
        nseq, Hq, Hkv, d, width = c["nseq"], c["Hq"], c["Hkv"], c["d"], s["qkv"].shape[2]
        size = (B, R, nseq, Hq, Hkv, d, dt)
        ins, cs = (R * width, width, d), (R * Hq * d, Hq * d, d)          # strides of model, row and head
        q, k, v = s["qkv"].split([Hq * d, Hkv * d, Hkv * d], 2)
        hb.attention_packed_fwd(*size, q, ins, k, v, ins, s["off"], s["scale"], int(c["causal"]), s["ctx"], cs, s["lse"])
        if op == "attn":
            return [s["ctx"], s["lse"]]
        dq, dk, dv = s["dqkv"].split([Hq * d, Hkv * d, Hkv * d], 2)
        ws = _workspace(s, hb.attention_packed_bwd_workspace_bytes(*size))
        hb.attention_packed_bwd(*size, q, ins, k, v, ins, s["off"], s["scale"], int(c["causal"]), s["ctx"], s["dctx"], cs, s["lse"],
                                dq, ins, dk, dv, ins, ws)
        return [s["ctx"], s["lse"], s["dqkv"]]
    if op == "embed":
        V, E, nseq = c["V"], c["E"], c["nseq"]
        hb.embedding_packed_fwd(B, R, V, E, nseq, dt, s["table"], s["idx"], s["off"], s["scale"], s["pos"], s["longest"], s["out"])
        ws = _workspace(s, hb.embedding_bwd_sorted_workspace_bytes(B, R, V, E))
        hb.embedding_bwd_sorted(B, R, V, E, nseq, dt, s["dy"], s["idx"], s["off"], s["scale"], s["dtable"], ws)
        return [s["out"], s["dtable"]]
    K, pairs = c["K"], c["pairs"]
    if op == "logps":
        hb.seq_logps(B, R, K, 2 * pairs, dt, s["logits"], s["labels"], s["off"], s["tokens"], s["logps"])
        return [s["tokens"], s["logps"]]
    ws = _workspace(s, hb.preference_loss_workspace_bytes(B, R, pairs))
    hb.preference_loss(B, R, K, pairs, dt, s["logits"], s["labels"], s["off"], s["ref"], s["beta"], s["smoothing"], s["loss"],
                       s["logps"], s["dlogits"], ws)
    return [s["loss"], s["logps"], s["dlogits"]]


def run(state):
    return _framework(state) if own else _plain(state)


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    B, R = c["B"], c["R"]
    if c["op"] in ("attn", "attn_train"):
        # uneven lengths: the mean of their squares over the square of their mean, as _lengths() draws them
        n = c["nseq"]
        scores = B * c["Hq"] * R * R / n * (1 + 0.148 * (1 - 1 / n)) * (0.5 if c["causal"] else 1.0)
        qkv, ctx, lse = B * R * (c["Hq"] + 2 * c["Hkv"]) * c["d"] * es, B * R * c["Hq"] * c["d"] * es, B * c["Hq"] * R * 4
        if c["op"] == "attn":
            return {"bytes": qkv + ctx + lse, "flops": 4 * c["d"] * scores}
        return {"bytes": 2 * qkv + 2 * ctx + lse, "flops": 14 * c["d"] * scores}
    if c["op"] == "embed":
        return {"bytes": B * R * (3 * c["E"] * es + 4) + B * c["V"] * c["E"] * 4, "flops": 3 * B * R * c["E"]}
    rows = 0.6 * B * R                     # the rows with a label
    if c["op"] == "logps":
        return {"bytes": rows * c["K"] * es + B * R * 8, "flops": 4 * rows * c["K"]}
    return {"bytes": (rows + B * R) * c["K"] * es + B * R * 4, "flops": 8 * rows * c["K"]}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_attention(s, train):
    c = s["c"]
    H, G, d = c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    off = s["off"].tolist()
    x = s["qkv"].double()
    ctx = torch.zeros(s["ctx"].shape, dtype=torch.float64, device="cuda")
    lse, grad = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda"), torch.zeros_like(x)
    dctx = s["dctx"].double() if train else None
    for b in range(c["B"]):
        for lo, hi in zip(off[b][:-1], off[b][1:]):
            n = hi - lo
            if n == 0:
                continue
            later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1) if c["causal"] else None
            for h in range(H * G):
                cols = [slice(h * d, (h + 1) * d)] + [slice((H * G + m * H + h // G) * d, (H * G + m * H + h // G + 1) * d) for m in (0, 1)]
                q, k, v = (x[b, lo:hi, i] for i in cols)
                a = q @ k.T * s["scale"]
                if later is not None:
                    a[later] = -math.inf
                lse[b, h, lo:hi] = torch.logsumexp(a, 1)
                a = torch.exp(a - lse[b, h, lo:hi, None])
                ctx[b, lo:hi, cols[0]] = a @ v
                if train:
                    g = dctx[b, lo:hi, cols[0]]
                    grad[b, lo:hi, cols[2]] += a.T @ g
                    a *= g @ v.T - (g * ctx[b, lo:hi, cols[0]]).sum(1, keepdim=True)
                    grad[b, lo:hi, cols[0]] = a @ k * s["scale"]
                    grad[b, lo:hi, cols[1]] += a.T @ q * s["scale"]
    return [ctx, lse, grad] if train else [ctx, lse]


def _exact_embedding(s):
    c, off = s["c"], s["off"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    grad = torch.zeros(s["dtable"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        for lo, hi in zip(off[b][:-1], off[b][1:]):
            out[b, lo:hi] = s["scale"] * s["table"][b][s["idx"][b, lo:hi].long()].double() + s["pos"][:hi - lo].double()
        lo, hi = off[b][0], off[b][-1]
        # sums of the rows sorted by token: differences of one running sum would lose what atomics keep
        order = torch.argsort(s["idx"][b, lo:hi], stable=True)
        ids, count = torch.unique_consecutive(s["idx"][b, lo:hi][order], return_counts=True)
        rows = s["dy"][b, lo:hi].double()[order]
        grad[b, ids.long()] = s["scale"] * torch.segment_reduce(rows, "sum", lengths=count, axis=0)
    return [out, grad]


def _exact_logps(s):
    c, off = s["c"], s["off"].tolist()
    logps = torch.zeros(c["B"], len(off[0]) - 1, dtype=torch.float64, device="cuda")
    tokens, soft = torch.zeros(c["B"], c["R"], dtype=torch.float64, device="cuda"), []
    for b in range(c["B"]):
        z = torch.log_softmax(s["logits"][b].double(), 1)
        y = s["labels"][b].long()
        term = z[torch.arange(c["R"], device="cuda"), y.clamp(min=0)]
        term[y < 0] = 0
        tokens[b] = term
        for i, (lo, hi) in enumerate(zip(off[b][:-1], off[b][1:])):
            logps[b, i] = term[lo:hi].sum()
        soft.append(z if c["op"] == "pref" else None)
    return tokens, logps, soft


def _exact_preference(s):
    c, off = s["c"], s["off"].tolist()
    _, logps, soft = _exact_logps(s)
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    loss = torch.zeros(c["B"], dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        beta, eps = float(s["beta"][b]), float(s["smoothing"][b])
        gap = (logps[b] - s["ref"][b].double()).tolist()
        y = s["labels"][b].long()
        for p in range(c["pairs"]):
            t = torch.tensor(beta * (gap[2 * p] - gap[2 * p + 1]), dtype=torch.float64, requires_grad=True)
            one = -(1 - eps) * torch.nn.functional.logsigmoid(t) - eps * torch.nn.functional.logsigmoid(-t)
            one.backward()
            loss[b] += one.item() / c["pairs"]
            for i, sign in ((2 * p, 1.0), (2 * p + 1, -1.0)):
                lo, hi = off[b][i], off[b][i + 1]
                rows = torch.arange(lo, hi, device="cuda")[y[lo:hi] >= 0]
                g = -soft[b][rows].exp()
                g[torch.arange(len(rows), device="cuda"), y[rows]] += 1
                grad[b, rows] = g * (sign * beta * float(t.grad) / c["pairs"])
    return [loss, logps, grad]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] in ("attn", "attn_train"):
        if c["B"] * c["Hq"] * c["R"] ** 2 * 1.2 / c["nseq"] > _EXACT_PAIRS or c["B"] * c["nseq"] * c["Hq"] > 10000:
            return None
        return _exact_attention(s, c["op"] == "attn_train")
    if c["op"] == "embed":
        return _exact_embedding(s)
    return list(_exact_logps(s)[:2]) if c["op"] == "logps" else _exact_preference(s)
