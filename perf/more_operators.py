"""Performance cases of the serving operators: what they are, how their inputs
are made, one pass of each, and what a pass computes in 64 bits.

A program that lets a model of schedule tokens propose configurations makes
these calls for every token: it puts the keys and values of the new tokens into
a paged cache and rotates them and the queries by position (at_paged_append),
attends over everything the cache holds of each sequence (at_paged_attention),
and changes the logits by what the sequence already said, by biases and by what
the schedule's grammar allows (at_adjust_logits), before at_logprobs draws the
alternatives.

  append   new keys and values into their pages, normed and rotated on the way
  attend   causal attention of the new tokens over the cache, grouped heads
  adjust   penalties, biases and masks on rows of logits

`run` takes what `prepare` gives.  With `own` false it computes the operators
in elementary torch operations, in 32 bits (angles in 64), rounded once at the
end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WHOLE = {"i32": torch.int32, "i64": torch.int64}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
EPS = 1e-6


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------
def listed():
    return [
        # serving: the next token of one sequence
        {"name": "append one token", "op": "append", "batch": 1, "new": 1, "ctx": 1000, "ragged": False, "pad": 0,
         "heads": 32, "kv": 8, "dim": 128, "rot": 128, "page": 16, "type": "bf16", "layout": "half", "norm": False,
         "stretch": 1.0},
        # the next token of a large batch, heads normed, some of the batch's places empty
        {"name": "append batch", "op": "append", "batch": 256, "new": 1, "ctx": 4096, "ragged": True, "pad": 8,
         "heads": 32, "kv": 8, "dim": 128, "rot": 128, "page": 16, "type": "bf16", "layout": "half", "norm": True,
         "stretch": 1.0},
        # prompts of different lengths at once
        {"name": "append prompts", "op": "append", "batch": 8, "new": 8192, "ctx": 0, "ragged": True, "pad": 0,
         "heads": 32, "kv": 8, "dim": 128, "rot": 128, "page": 64, "type": "bf16", "layout": "interleaved",
         "norm": False, "stretch": 1.0},
        # an odd head size, half of it rotated, far positions of a stretched range, pages of no power of two
        {"name": "append far", "op": "append", "batch": 3, "new": 700, "ctx": 150000, "ragged": True, "pad": 5,
         "heads": 6, "kv": 2, "dim": 80, "rot": 40, "page": 24, "type": "f32", "layout": "half", "norm": True,
         "stretch": 8.0},
        # serving: one sequence's next token over what it has
        {"name": "attend one token", "op": "attend", "batch": 1, "new": 1, "ctx": 4096, "ragged": False, "pad": 0,
         "heads": 32, "kv": 8, "dim": 128, "page": 16, "type": "bf16", "window": 0},
        # a batch of sequences of very different lengths, a token each
        {"name": "attend batch", "op": "attend", "batch": 64, "new": 1, "ctx": 16384, "ragged": True, "pad": 0,
         "heads": 32, "kv": 8, "dim": 128, "page": 16, "type": "bf16", "window": 0},
        # a chunk of a long prompt over what earlier chunks left
        {"name": "attend chunk", "op": "attend", "batch": 1, "new": 512, "ctx": 32000, "ragged": False, "pad": 0,
         "heads": 32, "kv": 8, "dim": 128, "page": 16, "type": "bf16", "window": 0},
        # a whole prompt
        {"name": "attend prompt", "op": "attend", "batch": 1, "new": 8192, "ctx": 0, "ragged": False, "pad": 0,
         "heads": 32, "kv": 8, "dim": 128, "page": 64, "type": "bf16", "window": 0},
        # an odd head size in fp32, each head its own keys, a window, pages that end inside every tile
        {"name": "attend window", "op": "attend", "batch": 3, "new": 700, "ctx": 900, "ragged": True, "pad": 3,
         "heads": 12, "kv": 12, "dim": 80, "page": 24, "type": "f32", "window": 500},
        # serving: the next token of one sequence under a grammar, with what it said before
        {"name": "adjust one row", "op": "adjust", "n": 1, "vocab": 131072, "type": "f32", "index": "i32", "past": 2000,
         "bias": 20, "masks": 1, "allowed": 0.3, "ragged": False, "penalties": True},
        # the knobs of a batch of configurations: each row its own number of values, values that the schedule rules out
        {"name": "adjust knobs", "op": "adjust", "n": 3584, "vocab": 220, "type": "f32", "index": "i64", "past": 7,
         "bias": 0, "masks": 7, "allowed": 0.7, "ragged": True, "penalties": True},
        # a large batch over a text vocabulary, long pasts, biases, some rows under a grammar
        {"name": "adjust text", "op": "adjust", "n": 512, "vocab": 131072, "type": "bf16", "index": "i32",
         "past": 8192, "bias": 50, "masks": 16, "allowed": 0.5, "ragged": False, "penalties": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "adjust"])
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op == "adjust":
        vocab = _log(rng, 2, 131072)
        return {"op": op, "n": _log(rng, 1, min(8192, (1 << 26) // vocab)), "vocab": vocab, "type": kind,
                "index": rng.choice(["i32", "i64"]), "past": rng.choice([0, _log(rng, 1, 8192)]),
                "bias": rng.choice([0, _log(rng, 1, 300)]), "masks": rng.choice([0, 1, 16]),
                "allowed": rng.choice([0.01, 0.5, 0.99]), "ragged": rng.random() < 0.4,
                "penalties": rng.random() < 0.8}
    kv, group = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 4, 5, 8])
    if op == "append":
        dim = rng.choice([16, 64, 80, 100, 128, 192, 256])
        rot = rng.choice([0, dim, dim, dim // 2 // 2 * 2])
        new = rng.choice([1, 1, _log(rng, 2, 2048)])
        batch = _log(rng, 1, 256 if new == 1 else 8)
        ctx = _log(rng, 1, min(100000, (1 << 26) // (kv * dim * batch)))
        return {"op": op, "batch": batch, "new": new, "ctx": ctx, "ragged": rng.random() < 0.6,
                "pad": rng.choice([0, 0, 3]), "heads": kv * group, "kv": kv, "dim": dim, "rot": rot,
                "page": rng.choice([1, 16, 24, 64, 128]), "type": kind, "layout": rng.choice(["half", "interleaved"]),
                "norm": rng.random() < 0.4, "stretch": rng.choice([1.0, 4.0])}
    dim = rng.choice([16, 64, 80, 100, 128, 128, 256])
    if rng.random() < 0.5:
        new, batch = 1, _log(rng, 1, 64)
        ctx = _log(rng, 1, 16384)
    else:
        new, batch = _log(rng, 2, 1024), rng.choice([1, 2, 5])
        ctx = _log(rng, 1, min(16384, (1 << 29) // (new * batch * kv * group)))
    return {"op": op, "batch": batch, "new": new, "ctx": ctx, "ragged": rng.random() < 0.6, "pad": rng.choice([0, 0, 3]),
            "heads": kv * group, "kv": kv, "dim": dim, "page": rng.choice([1, 16, 24, 64, 128]), "type": kind,
            "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)])}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _sizes(case):
    """New tokens and earlier ones of each sequence of a batch.  The first of each is the longest; a ragged batch's go
    down from there in equal steps, single tokens leave every eighth place empty where the buffers are padded."""
    B = case["batch"]
    new, ctx = np.full(B, case["new"]), np.full(B, case["ctx"])
    if case["ragged"]:
        left = (B - np.arange(B)) / B
        ctx = (ctx * left).astype(np.int64)
        if case["new"] > 1:
            new = np.maximum(1, (new * left).astype(np.int64))
        elif case["pad"]:
            new[7::8] = 0
    return new, ctx


def _plan(case, seed):
    """Whole numbers of a batch: where each sequence's new tokens start, its length with them, and its pages, which lie
    anywhere in the cache.  Unused places of the table name no page."""
    rng = np.random.default_rng(int(seed) + 12345)
    B, ps = case["batch"], case["page"]
    new, ctx = _sizes(case)
    pages = int((-(-new // ps) - (-ctx // ps)).sum()) + 3
    for a in (new, ctx):
        a[1:] = rng.permutation(a[1:])
    lengths = new + ctx
    starts = np.concatenate([[0], np.cumsum(new)])
    need = -(-lengths // ps)
    width = -(-(case["new"] + case["ctx"]) // ps)
    table = np.full((B, width), -1, np.int64)
    table[np.arange(width)[None] < need[:, None]] = rng.permutation(pages)[: int(need.sum())]
    return starts, lengths, table, pages


def _batch(s, case, seed):
    starts, lengths, table, pages = _plan(case, seed)
    put = lambda a: torch.as_tensor(a.astype(np.int32), device=DEV)  # noqa: E731
    s["starts"], s["lengths"], s["table"] = put(starts), put(lengths), put(table)
    s["n"] = case["batch"] * case["new"] + case["pad"]   # a program's buffers hold the most it may have to
    return pages


def _normal(gen, kind, *shape):
    out = torch.empty(*shape, dtype=FLOAT[kind], device=DEV)
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 28):
        m = min(1 << 28, flat.numel() - lo)
        flat[lo: lo + m] = torch.randn(m, generator=gen, device=DEV)
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    op, s = case["op"], {"case": case}
    if op == "adjust":
        n, V, ti = case["n"], case["vocab"], WHOLE[case["index"]]
        rand = lambda *sh: torch.rand(*sh, generator=gen, device=DEV)  # noqa: E731
        x = torch.randn(n, V, generator=gen, device=DEV) * 3.0
        s["logits"] = x.to(FLOAT[case["type"]])
        s["out"] = torch.zeros_like(s["logits"])
        L, B = case["past"], case["bias"]
        # what the sequences said: small tokens most often, one place in fifty holds none
        s["past"] = torch.where(rand(n, L) < 0.02, -1.0, torch.exp(rand(n, L) * math.log(V + 1.0)) - 1.0)
        s["past"] = s["past"].clamp(-1, V - 1).to(ti)
        s["past_len"] = (rand(n) * (L + 1)).int().clamp(max=L)
        s["past_len"][0] = L
        s["prompt_len"] = (s["past_len"] * rand(n)).int()
        s["repetition"] = s["presence"] = s["frequency"] = None
        if case["penalties"]:   # every fourth row has none
            on = (torch.arange(n, device=DEV) % 4 != 3).float()
            s["repetition"] = 1.0 + 0.3 * rand(n) * on
            s["presence"], s["frequency"] = rand(n) * on, rand(n) * 0.2 * on
        s["bias_tokens"] = (rand(n, B) * V).to(ti).clamp(max=V - 1)
        s["bias"] = torch.randn(n, B, generator=gen, device=DEV) * 5.0
        words = (V + 31) // 32
        s["mask"] = s["mask_rows"] = None
        if case["masks"]:
            m = case["masks"]
            bits = (rand(m, words, 32) < case["allowed"]).long() << torch.arange(32, device=DEV)
            bits = bits.sum(2)
            s["mask"] = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
            # with several masks some rows have none
            s["mask_rows"] = (rand(n) * (m + (m > 1) * m // 2)).int()
            s["mask_rows"][s["mask_rows"] >= m] = -1
        s["valid"] = None
        if case["ragged"]:
            s["valid"] = (rand(n) * (V + 1)).int().clamp(max=V)
        return s
    pages, T = _batch(s, case, seed), FLOAT[case["type"]]
    n, H, K, D, ps = s["n"], case["heads"], case["kv"], case["dim"], case["page"]
    s["k_cache"], s["v_cache"] = (_normal(gen, case["type"], pages, ps, K, D) for _ in range(2))
    s["out"] = torch.zeros(n, H, D, dtype=T, device=DEV)
    if op == "append":
        # one product makes queries, keys and values: they lie side by side
        qkv = _normal(gen, case["type"], n, H + 2 * K, D)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H: H + K], qkv[:, H + K:]
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"], s["k_weight"] = ((1.0 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(T) for _ in range(2))
        R = case["rot"]
        s["freqs"] = 10000.0 ** (-torch.arange(0, R, 2, device=DEV, dtype=torch.float64) / max(R, 1)) / case["stretch"]
        s["turn"] = 1.0 + 0.1 * math.log(case["stretch"])
    else:
        # queries that find a few keys: what a trained model's scores spread like
        s["q"] = (_normal(gen, "f32", n, H, D) * 1.5).to(T)
        s["lse"] = torch.zeros(n, H, dtype=torch.float32, device=DEV)
        s["scale"] = 1.0 / math.sqrt(D)
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_1805_08166_amd as P
    case = s["case"]
    if case["op"] == "append":
        P.at_paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["lengths"], q=s["q"],
                          q_out=s["out"], freqs=s["freqs"], interleaved=case["layout"] == "interleaved",
                          rot_scale=s["turn"], k_weight=s["k_weight"], q_weight=s["q_weight"], eps=EPS)
        return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if case["op"] == "attend":
        P.at_paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["lengths"], s["out"],
                             scale=s["scale"], window=case["window"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    P.at_adjust_logits(s["logits"], s["out"], tokens=s["past"], lengths=s["past_len"], prompt_lengths=s["prompt_len"],
                       repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                       bias_tokens=s["bias_tokens"], bias=s["bias"], mask=s["mask"], mask_rows=s["mask_rows"],
                       valid=s["valid"])
    return s["out"]


def _where(s):
    """(sequence, row within it, position, whether there is one) of each of the call's tokens."""
    i = torch.arange(s["n"], device=DEV)
    b = torch.searchsorted(s["starts"].long(), i, right=True) - 1
    real = i < s["starts"][-1]
    b = b.clamp(max=s["case"]["batch"] - 1)
    row = i - s["starts"].long()[b]
    return b, row, s["lengths"].long()[b] - (s["starts"].long()[b + 1] - i), real


def _plain(s):
    return {"append": _plain_append, "attend": _plain_attend, "adjust": _plain_adjust}[s["case"]["op"]](s)


def _plain_append(s):
    case = s["case"]
    b, _, pos, real = _where(s)

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS) * weight.float()
        R = case["rot"]
        t = pos.double()[:, None, None] * s["freqs"]
        cos, sin = torch.cos(t).float(), torch.sin(t).float()
        if case["layout"] == "half":
            a, c = x[..., : R // 2], x[..., R // 2: R]
        else:
            a, c = x[..., 0:R:2], x[..., 1:R:2]
        y = (a * cos - c * sin) * s["turn"], (c * cos + a * sin) * s["turn"]
        y = torch.cat(y, 2) if case["layout"] == "half" else torch.stack(y, 3).flatten(2)
        return torch.cat([y, x[..., R:]], 2).to(FLOAT[case["type"]])

    q = turned(s["q"], s["q_weight"])
    s["out"].copy_(torch.where(real[:, None, None], q, s["out"]))
    ps = case["page"]
    page = s["table"].long()[b, (pos // ps).clamp(0, s["table"].shape[1] - 1)]
    slot = torch.where(real, page * ps + pos % ps, torch.zeros_like(pos))
    for cache, rows in ((s["k_cache"], turned(s["k"], s["k_weight"])), (s["v_cache"], s["v"])):
        flat = cache.view(-1, case["kv"], case["dim"])
        # tokens behind the last sequence are put where the first token goes, as the first token
        first = rows[:1]
        flat[torch.where(real, slot, slot[0])] = torch.where(real[:, None, None], rows, first)
    return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    case = s["case"]
    B, M, K, D = case["batch"], case["new"], case["kv"], case["dim"]
    G, L = case["heads"] // K, case["new"] + case["ctx"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    # all sequences' keys and queries side by side, as long as the longest
    pages = s["table"].long().clamp(min=0)
    keys, values = (c[pages].flatten(1, 2)[:, :L].permute(0, 2, 1, 3).float().contiguous()
                    for c in (s["k_cache"], s["v_cache"]))                                      # [B, K, L, D]
    r = torch.arange(M, device=DEV)
    at = (starts[:-1, None] + r).clamp(max=s["n"] - 1)                                          # [B, M]
    q = s["q"][at].float().view(B, M, K, G, D).permute(0, 2, 3, 1, 4).reshape(B, K, G * M, D)
    x = torch.matmul(q, keys.transpose(2, 3).contiguous()).view(B, K, G, M, L)
    x *= s["scale"]
    pos = (lengths - (starts[1:] - starts[:-1]))[:, None] + r                                   # [B, M]
    j = torch.arange(L, device=DEV)
    hidden = (j > pos[..., None]) | (j >= lengths[:, None, None])
    if case["window"]:
        hidden |= j <= pos[..., None] - case["window"]
    x.masked_fill_(hidden[:, None, None], -math.inf)
    top = x.amax(4, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    x -= top
    x.exp_()
    total = x.sum(4, keepdim=True)
    lse = torch.log(total) + top                                                                # [B, K, G, M, 1]
    x /= torch.where(total > 0, total, torch.ones_like(total))
    out = torch.matmul(x.view(B, K, G * M, L), values).view(B, K, G, M, D)
    b, row, _, real = _where(s)
    row = row.clamp(max=M - 1)
    out = out[b, :, :, row].flatten(1, 2).to(FLOAT[case["type"]])
    lse = lse[b, :, :, row, 0].flatten(1, 2)
    return {"out": torch.where(real[:, None, None], out, s["out"]), "lse": torch.where(real[:, None], lse, s["lse"])}


def _plain_adjust(s):
    case = s["case"]
    n, V = case["n"], case["vocab"]
    x = s["logits"].float()
    ruled = x == -math.inf
    past = s["past"].long()
    place = torch.arange(past.shape[1], device=DEV)
    said = (place < s["past_len"][:, None]) & (past >= 0)
    ones = said.float()
    answer = (said & (place >= s["prompt_len"][:, None])).float()
    at = past.clamp(min=0)
    zeros = lambda: torch.zeros(n, V, device=DEV)  # noqa: E731
    seen, count = zeros().scatter_add_(1, at, ones) > 0, zeros().scatter_add_(1, at, answer)
    if s["repetition"] is not None:
        r = s["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
        x = x - s["frequency"][:, None] * count
        x = torch.where(count > 0, x - s["presence"][:, None], x)
    if case["bias"]:
        # of a token's biases the last one counts
        B = case["bias"]
        last = torch.full((n, V), -1, device=DEV)
        last.scatter_reduce_(1, s["bias_tokens"].long(), torch.arange(B, device=DEV).expand(n, B).contiguous(), "amax")
        x = torch.where(last >= 0, x + torch.gather(s["bias"], 1, last.clamp(min=0)), x)
    x = x.masked_fill(ruled, -math.inf)
    col = torch.arange(V, device=DEV)
    if s["mask"] is not None:
        rows = s["mask_rows"].long()
        words = s["mask"][rows.clamp(min=0)]
        allowed = (words[:, col >> 5] >> (col & 31)) & 1
        x = x.masked_fill((allowed == 0) & (rows >= 0)[:, None], -math.inf)
    x = x.to(FLOAT[case["type"]])
    if s["valid"] is not None:   # columns that a row does not have stay as they were
        x = torch.where(col < s["valid"][:, None], x, s["out"])
    return x


# --------------------------------------------------------------------------
# Work and 64-bit results
# --------------------------------------------------------------------------
def work(case):
    a = SIZE[case["type"]]
    share = 0.5 if case["ragged"] else 1.0
    if case["op"] == "adjust":
        n, V = case["n"], case["vocab"]
        past = n * case["past"] * 0.5 * SIZE[case["index"]]
        masks = min(n, case["masks"]) * V / 8
        return {"bytes": 2 * n * V * share * a + past + n * case["bias"] * (4 + SIZE[case["index"]]) + masks,
                "flops": 2 * n * V * share}
    B, H, K, D = case["batch"], case["heads"], case["kv"], case["dim"]
    new, ctx = (v.astype(np.float64) for v in _sizes(case))
    if case["op"] == "append":
        return {"bytes": 2 * new.sum() * (H + 2 * K) * D * a + B * 12, "flops": 3 * new.sum() * (H + K) * D}
    # which lengths meet which numbers of new tokens is drawn: in the mean every one meets every other
    seen, held = ctx.mean() + (new + 1) / 2, ctx.mean() + new
    if case["window"]:
        seen, held = np.minimum(seen, case["window"]), np.minimum(held, case["window"] + new)
    return {"bytes": 2 * (held * (new > 0)).sum() * K * D * a + 2 * new.sum() * H * D * a + new.sum() * H * 4,
            "flops": 4 * (new * seen).sum() * H * D}


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "adjust": _exact_adjust}[case["op"]](case, prepare(case, seed), seed)


def _exact_append(case, s, seed):
    starts, lengths, table, _ = _plan(case, seed)
    R, ps = case["rot"], case["page"]
    q, k_cache, v_cache = s["out"].double(), s["k_cache"].double(), s["v_cache"].double()

    def turned(x, weight, pos):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x * x).sum(2, keepdim=True) / case["dim"] + EPS) * weight.double()
        if R:
            z = torch.polar(torch.full((), s["turn"], dtype=torch.float64, device=DEV), pos.double()[:, None, None] * s["freqs"])
            pairs = x[..., :R].unflatten(2, (2, R // 2) if case["layout"] == "half" else (R // 2, 2))
            pairs = pairs.transpose(2, 3) if case["layout"] == "half" else pairs
            y = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * z)
            y = y.transpose(2, 3) if case["layout"] == "half" else y
            x = torch.cat([y.flatten(2), x[..., R:]], 2)
        return x

    for b in range(case["batch"]):
        lo, hi = int(starts[b]), int(starts[b + 1])
        p = np.arange(lengths[b] - (hi - lo), lengths[b])
        pos = torch.as_tensor(p, device=DEV)
        page, off = (torch.as_tensor(a, device=DEV) for a in (table[b, p // ps], p % ps))
        q[lo:hi] = turned(s["q"][lo:hi], s["q_weight"], pos)
        k_cache[page, off] = turned(s["k"][lo:hi], s["k_weight"], pos)
        v_cache[page, off] = s["v"][lo:hi].double()
    return {"q": q, "k_cache": k_cache, "v_cache": v_cache}


def _exact_attend(case, s, seed):
    starts, lengths, table, _ = _plan(case, seed)
    K, G, D, ps = case["kv"], case["heads"] // case["kv"], case["dim"], case["page"]
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(case["batch"]):
        lo, hi, n = int(starts[b]), int(starts[b + 1]), int(lengths[b])
        if lo == hi:
            continue
        p = np.arange(n)
        slot = torch.as_tensor(table[b, p // ps] * ps + p % ps, device=DEV)
        k, v = (c.view(-1, K, D)[slot].double() for c in (s["k_cache"], s["v_cache"]))
        mine = torch.arange(n - (hi - lo), n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None]
        seen = j <= mine
        if case["window"]:
            seen &= mine - j < case["window"]
        for h in range(case["heads"]):
            z = s["q"][lo:hi, h].double() @ k[:, h // G].T.contiguous() * s["scale"]
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            total = torch.logsumexp(z, 1)
            lse[lo:hi, h] = total
            out[lo:hi, h] = torch.exp(z - total[:, None]) @ v[:, h // G].contiguous()
    return {"out": out, "lse": lse}


def _exact_adjust(case, s, seed):
    n, V = case["n"], case["vocab"]
    out = s["out"].double()
    host = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    past, past_len, prompt_len = host(s["past"]), host(s["past_len"]), host(s["prompt_len"])
    pen = [host(s[k]) for k in ("repetition", "frequency", "presence")]
    tokens, bias, mask, rows, valid = (host(s[k]) for k in ("bias_tokens", "bias", "mask", "mask_rows", "valid"))
    for i in range(n):
        x = s["logits"][i].double().cpu().numpy()
        ruled = np.isneginf(x)
        h = past[i, : past_len[i]]
        late = h[prompt_len[i]:]
        seen = np.unique(h[h >= 0])
        count = np.bincount(late[late >= 0], minlength=V).astype(np.float64)
        if pen[0] is not None:
            r, f, p = (float(a[i]) for a in pen)
            x[seen] = np.where(x[seen] > 0, x[seen] / r, x[seen] * r)
            x -= f * count + p * (count > 0)
        for t, v in {int(t): float(v) for t, v in zip(tokens[i], bias[i])}.items():
            x[t] += v
        x[ruled] = -np.inf
        if mask is not None and rows[i] >= 0:
            bits = np.unpackbits(mask[rows[i]].view(np.uint8), bitorder="little")[:V]
            x[bits == 0] = -np.inf
        w = V if valid is None else int(valid[i])
        out[i, :w] = torch.as_tensor(x[:w], device=DEV)
    return out
