"""Performance cases of the sequence-model operators: what they are, how their
inputs are made, one pass of each, and what a pass computes in 64 bits.

A program that learns proposals from what a search kept makes these calls: it
turns configurations into knob tokens and embeds them (at_embed), scores the
values of each knob (at_logprobs), and trains on the result
(at_logprobs_grad, at_embed_grad, and at_orthogonalize for the update of its
hidden matrices).  Vocabularies run from one knob's few values, each row with
its own number of them, to the ones of models that write whole schedules as
text.

  embed    rows of a table by token, scaled; tokens of -1 are padding
  egrad    its gradient: rows summed by token
  logp     log probabilities of given tokens, entropies, top alternatives
  lgrad    the gradient of the log probabilities and the entropies
  ortho    Newton-Schulz steps on a batch of equal matrices

`run` takes what `prepare` gives.  With `own` false it computes the operators
in elementary torch operations, in 32 bits, rounded once at the end.
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
COEF = (3.4445, -4.7750, 2.0315)   # of the quintic that Newton-Schulz updates commonly use


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------
def listed():
    return [
        # the 7 knob tokens of 64 chains' 8 best configurations of the 512^3 GEMM, in one table of all knobs' values
        {"name": "embed knobs", "op": "embed", "n": 3584, "vocab": 455, "dim": 128, "type": "f32", "out": "f32",
         "index": "i64", "scale": 11.3125, "spread": "flat"},
        # a training batch of long sequences over a text vocabulary
        {"name": "embed text", "op": "embed", "n": 65536, "vocab": 131072, "dim": 2048, "type": "bf16", "out": "bf16",
         "index": "i32", "scale": 45.25, "spread": "flat"},
        # the loop features of 4096 conv2d configurations as tokens (176 columns of 33 values): few rows, each many times
        {"name": "egrad features", "op": "egrad", "n": 720896, "vocab": 5808, "dim": 128, "type": "bf16", "out": "f32",
         "index": "i32", "scale": 11.3125, "spread": "columns", "add": False},
        # one step's gradient of a text table: a few tokens very often, most never
        {"name": "egrad text", "op": "egrad", "n": 32768, "vocab": 131072, "dim": 1024, "type": "bf16", "out": "f32",
         "index": "i64", "scale": 32.0, "spread": "frequent", "add": False},
        # the same added to what earlier micro-batches left, an odd vocabulary, few tokens
        {"name": "egrad added", "op": "egrad", "n": 2049, "vocab": 32003, "dim": 1000, "type": "f32", "out": "f32",
         "index": "i32", "scale": 1.0, "spread": "frequent", "add": True},
        # serving: the next token of one sequence with its alternatives
        {"name": "logp one token", "op": "logp", "n": 1, "vocab": 131072, "type": "bf16", "k": 20, "pad": 0,
         "ragged": False, "masked": 0.0, "scale": 1.25},
        # a knob's value for every step of a batch: each row has its knob's number of values, some of them ruled out
        {"name": "logp knobs", "op": "logp", "n": 3584, "vocab": 220, "type": "f32", "k": 8, "pad": 0,
         "ragged": True, "masked": 0.1, "scale": 1.0},
        # a training batch, an odd vocabulary in rows of a rounded-up stride
        {"name": "logp text", "op": "logp", "n": 4095, "vocab": 50001, "type": "bf16", "k": 5, "pad": 47,
         "ragged": False, "masked": 0.0, "scale": 1.0},
        # gradients of the knob rows, and of a large batch over a large vocabulary
        {"name": "lgrad knobs", "op": "lgrad", "n": 3584, "vocab": 220, "type": "f32", "pad": 0, "ragged": True,
         "masked": 0.1, "scale": 1.0, "entropy": True},
        {"name": "lgrad text", "op": "lgrad", "n": 8192, "vocab": 131072, "type": "bf16", "pad": 0, "ragged": False,
         "masked": 0.0, "scale": 1.0, "entropy": True},
        # the hidden matrices of a small proposal model
        {"name": "ortho hidden", "op": "ortho", "batch": 8, "rows": 128, "cols": 128, "type": "f32", "steps": 5,
         "rank": 8},
        # two layers' expanding matrices, a wide pair of large ones
        {"name": "ortho wide", "op": "ortho", "batch": 2, "rows": 1024, "cols": 4096, "type": "bf16", "steps": 5,
         "rank": 64},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "egrad", "logp", "lgrad", "ortho"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("embed", "egrad"):
        case = {"op": op, "n": _log(rng, 1, 65536), "vocab": _log(rng, 33, 131072), "dim": _log(rng, 8, 2048),
                "type": kind, "out": rng.choice([kind, "f32"]), "index": rng.choice(["i32", "i64"]),
                "scale": rng.choice([1.0, 0.75, 11.3125]), "spread": rng.choice(["flat", "frequent", "columns"])}
        if op == "egrad":
            case["add"] = rng.random() < 0.3
        return case
    if op == "ortho":
        rows, cols = _log(rng, 16, 1024), _log(rng, 16, 4096)
        if rng.random() < 0.5:
            rows, cols = cols, rows
        return {"op": op, "batch": rng.choice([1, 2, 5]), "rows": rows, "cols": cols, "type": kind,
                "steps": rng.choice([4, 5, 6]), "rank": rng.choice([1, 8, 64])}
    case = {"op": op, "n": _log(rng, 1, 8192), "vocab": _log(rng, 2, 131072), "type": kind,
            "pad": rng.choice([0, 0, 1, 24]), "ragged": rng.random() < 0.4, "masked": rng.choice([0.0, 0.0, 0.1, 0.7]),
            "scale": rng.choice([1.0, 0.5, 1.25])}
    if op == "logp":
        case["k"] = rng.choice([0, 1, 5, 20, 64])
    else:
        case["entropy"] = rng.random() < 0.7
    return case


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _tokens(case, gen):
    """flat: uniform; frequent: token r about as often as 1 / (r + 1); columns: each position its own run of 33 values.
    One in fifty is padding."""
    n, V = case["n"], case["vocab"]
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    if case["spread"] == "flat":
        t = (u * V).long()
    elif case["spread"] == "frequent":
        t = (torch.exp(u * math.log(V + 1.0)) - 1.0).long()
    else:
        columns = max(1, V // 33)
        t = (torch.arange(n, device=DEV) % columns) * 33 + (u * u * 33).long()
    t = t.clamp_(0, V - 1)
    t[torch.rand(n, generator=gen, device=DEV) < 0.02] = -1
    return t.to(WHOLE[case["index"]])


def _logits(case, gen):
    """Scores of a trained model: a wide spread and a few likely values in each row, some values ruled out."""
    n, V = case["n"], case["vocab"]
    x = torch.empty(n, V + case["pad"], dtype=FLOAT[case["type"]], device=DEV)[:, :V]
    step = max(1, (1 << 27) // V)
    for lo in range(0, n, step):
        m = min(step, n - lo)
        y = torch.randn(m, V, generator=gen, device=DEV) * 2.0
        few = torch.randint(0, V, (m, 6), generator=gen, device=DEV)
        y.scatter_add_(1, few, torch.rand(m, 6, generator=gen, device=DEV) * 12.0)
        if case["masked"]:
            y.masked_fill_(torch.rand(m, V, generator=gen, device=DEV) < case["masked"], -math.inf)
        x[lo: lo + m] = y
    valid = None
    if case["ragged"]:   # every row its own number of values; one row in 64 has none
        valid = 1 + (torch.rand(n, generator=gen, device=DEV) * V).int()
        valid = valid.clamp_(max=V)
        valid[torch.rand(n, generator=gen, device=DEV) < 1 / 64] = 0
    width = valid if valid is not None else torch.full((n,), V, device=DEV)
    tokens = (torch.rand(n, generator=gen, device=DEV) * width).long()
    tokens = torch.minimum(tokens, (width.long() - 1).clamp(min=0))
    tokens[torch.rand(n, generator=gen, device=DEV) < 0.02] = -1
    return x, valid, tokens


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    op, s = case["op"], {"case": case}
    if op == "embed":
        s["weight"] = torch.randn(case["vocab"], case["dim"], generator=gen, device=DEV).to(FLOAT[case["type"]])
        s["tokens"] = _tokens(case, gen)
        s["out"] = torch.empty(case["n"], case["dim"], dtype=FLOAT[case["out"]], device=DEV)
    elif op == "egrad":
        s["dout"] = torch.randn(case["n"], case["dim"], generator=gen, device=DEV).to(FLOAT[case["type"]])
        s["tokens"] = _tokens(case, gen)
        shape = (case["vocab"], case["dim"])
        s["before"] = None
        if case["add"]:   # each pass adds to the same earlier sums, so that passes can be compared
            s["before"] = torch.randn(*shape, generator=gen, device=DEV).to(FLOAT[case["out"]])
        s["dweight"] = torch.empty(*shape, dtype=FLOAT[case["out"]], device=DEV)
    elif op in ("logp", "lgrad"):
        s["logits"], s["valid"], s["tokens"] = _logits(case, gen)
        n = case["n"]
        new = lambda *sh: torch.empty(*sh, dtype=torch.float32, device=DEV)  # noqa: E731
        if op == "logp":
            s["logp"], s["entropy"], s["lse"] = new(n), new(n), new(n)
            s["top_logp"], s["top_idx"] = new(n, case["k"]), new(n, case["k"]).int()
        else:   # what the forward pass left, and the gradients that come back to it
            step = max(1, (1 << 26) // case["vocab"])
            got = [_stats64(s, lo, min(n, lo + step)) for lo in range(0, n, step)]
            s["lse"], s["entropy"] = (torch.cat([g[i] for g in got]).float() for i in (0, 1))
            s["dlogp"] = torch.randn(n, generator=gen, device=DEV)
            s["dentropy"] = torch.randn(n, generator=gen, device=DEV) * 0.1 if case["entropy"] else None
            s["dlogits"] = torch.empty(n, case["vocab"], dtype=FLOAT[case["type"]], device=DEV)
    else:
        b, m, n, r = case["batch"], case["rows"], case["cols"], case["rank"]
        r = min(r, m, n)
        # a momentum: a few strong directions of falling weight over the noise of a batch's gradients
        left = torch.randn(b, m, r, generator=gen, device=DEV) * (3.0 / torch.arange(1, r + 1, device=DEV))
        right = torch.randn(b, r, n, generator=gen, device=DEV)
        g = torch.randn(b, m, n, generator=gen, device=DEV) + torch.matmul(left, right)
        s["momentum"] = (g * 1e-3).to(FLOAT[case["type"]])
        s["update"] = torch.empty(b, m, n, dtype=torch.bfloat16, device=DEV)
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_1805_08166_amd as P
    case = s["case"]
    op = case["op"]
    if op == "embed":
        P.at_embed(s["weight"], s["tokens"], s["out"], scale=case["scale"])
        return s["out"]
    if op == "egrad":
        if case["add"]:
            s["dweight"].copy_(s["before"])
        P.at_embed_grad(s["dout"], s["tokens"], s["dweight"], scale=case["scale"], accumulate=case["add"])
        return s["dweight"]
    if op == "logp":
        top = (s["top_logp"], s["top_idx"]) if case["k"] else (None, None)
        P.at_logprobs(s["logits"], s["tokens"], s["logp"], s["entropy"], s["lse"], *top, valid=s["valid"],
                      scale=case["scale"])
        return {"logp": s["logp"], "entropy": s["entropy"], "lse": s["lse"], "top_logp": s["top_logp"],
                "top_idx": s["top_idx"]}
    if op == "lgrad":
        P.at_logprobs_grad(s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogp"], s["dlogits"],
                           dentropy=s["dentropy"], valid=s["valid"], scale=case["scale"])
        return s["dlogits"]
    P.at_orthogonalize(s["momentum"], s["update"], steps=case["steps"], coef=COEF)
    return s["update"]


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "embed":
        t, V = s["tokens"].long(), case["vocab"]
        real = (t >= 0) & (t < V)
        rows = s["weight"][t.clamp(0, V - 1)].float() * case["scale"]
        return (rows * real[:, None]).to(FLOAT[case["out"]])
    if op == "egrad":
        t, V = s["tokens"].long(), case["vocab"]
        t = torch.where((t >= 0) & (t < V), t, torch.full_like(t, V))
        g = torch.zeros(V + 1, case["dim"], device=DEV).index_add_(0, t, s["dout"].float())[:V] * case["scale"]
        if case["add"]:
            g = s["before"].float() + g
        return g.to(FLOAT[case["out"]])
    if op == "logp":
        x = _inside(s, s["logits"].float())
        z = x * case["scale"]
        top = z.amax(1)
        some = top > -math.inf
        base = torch.where(some, top, torch.zeros_like(top))[:, None]
        e = torch.exp(z - base)
        total = e.sum(1)
        lse = torch.where(some, base[:, 0] + torch.log(total), top)
        spread = torch.where(e > 0, e * (z - base), torch.zeros_like(e)).sum(1)
        entropy = torch.where(some, torch.log(total) - spread / total, torch.zeros_like(top))
        t = s["tokens"]
        logp = torch.gather(z, 1, t.clamp(min=0)[:, None])[:, 0] - lse
        logp = torch.where(some, logp, top)
        logp = torch.where(t < 0, torch.zeros_like(logp), logp)
        k, V = case["k"], case["vocab"]
        keep = min(k, V)
        # whole numbers that sort as the values do, the lower index first among equals
        bits = (x + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + (0xFFFFFFFF - torch.arange(V, device=DEV))
        best = 0xFFFFFFFF - (torch.topk(key, keep, 1).values & 0xFFFFFFFF)
        found = torch.gather(z, 1, best)
        index = torch.where(found > -math.inf, best, torch.full_like(best, -1)).int()
        found = torch.where(index >= 0, found - lse[:, None], found)
        more = k - keep
        if more:
            index = torch.cat([index, torch.full((len(x), more), -1, dtype=torch.int32, device=DEV)], 1)
            found = torch.cat([found, torch.full((len(x), more), -math.inf, device=DEV)], 1)
        return {"logp": logp, "entropy": entropy, "lse": lse, "top_logp": found, "top_idx": index}
    if op == "lgrad":
        z = _inside(s, s["logits"].float()) * case["scale"]
        lse, t = s["lse"][:, None], s["tokens"]
        here = z > -math.inf
        logp = torch.where(here, z - lse, torch.zeros_like(z))
        p = torch.where(here, torch.exp(logp), torch.zeros_like(z))
        chosen = (torch.gather(z, 1, t.clamp(min=0)[:, None])[:, 0] > -math.inf) & (t >= 0)
        g = torch.where(chosen, s["dlogp"], torch.zeros_like(s["dlogp"]))
        d = -g[:, None] * p
        d.scatter_add_(1, t.clamp(min=0)[:, None], g[:, None])
        if s["dentropy"] is not None:
            d = d - s["dentropy"][:, None] * p * (logp + s["entropy"][:, None])
        return (d * case["scale"]).to(FLOAT[case["type"]])
    a, b, c = COEF
    x = s["momentum"].float()
    tall = case["rows"] > case["cols"]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for _ in range(case["steps"]):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return (x.transpose(1, 2).contiguous() if tall else x).to(torch.bfloat16)


def _inside(s, x):
    """x with minus infinity in the columns past each row's number of values."""
    if s["valid"] is None:
        return x
    return x.masked_fill(torch.arange(x.shape[1], device=DEV) >= s["valid"][:, None], -math.inf)


# --------------------------------------------------------------------------
# Work and 64-bit results
# --------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("embed", "egrad"):
        n, V, D, a, o = case["n"], case["vocab"], case["dim"], SIZE[case["type"]], SIZE[case["out"]]
        if op == "embed":
            different = V * -math.expm1(-n / V)   # rows that n uniform tokens name
            return {"bytes": n * SIZE[case["index"]] + different * D * a + n * D * o, "flops": n * D}
        return {"bytes": n * SIZE[case["index"]] + n * D * a + V * D * o * (2 if case["add"] else 1), "flops": n * D}
    if op in ("logp", "lgrad"):
        share = 0.5 if case["ragged"] else 1.0
        cells = case["n"] * case["vocab"]
        read = cells * share * SIZE[case["type"]] + case["n"] * 8
        if op == "logp":
            return {"bytes": read + case["n"] * (12 + 8 * case["k"]), "flops": 6 * cells * share}
        return {"bytes": read + case["n"] * 16 + cells * SIZE[case["type"]], "flops": 8 * cells * share}
    s, l = sorted((case["rows"], case["cols"]))
    return {"bytes": case["batch"] * s * l * (SIZE[case["type"]] + 2),
            "flops": case["batch"] * case["steps"] * (3.0 * s * s * l + 1.0 * s * s * s)}


def _stats64(s, lo, hi):
    """(log sum exp, entropy) of rows lo .. hi-1 in 64 bits."""
    z = s["logits"][lo:hi].double() * s["case"]["scale"]
    if s["valid"] is not None:
        z = z.masked_fill(torch.arange(z.shape[1], device=DEV) >= s["valid"][lo:hi, None], -math.inf)
    lse = torch.logsumexp(z, 1)
    logp = z - torch.where(lse > -math.inf, lse, torch.zeros_like(lse))[:, None]
    entropy = -torch.where(z > -math.inf, logp.exp() * logp, torch.zeros_like(z)).sum(1)
    return lse, entropy, z, logp


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        t = s["tokens"].long()
        out = torch.zeros(case["n"], case["dim"], dtype=torch.float64, device=DEV)
        at = torch.nonzero(t >= 0)[:, 0]
        out[at] = s["weight"].double()[t[at]] * case["scale"]
        return out
    if op == "egrad":
        t, d = s["tokens"].long(), s["dout"].double()
        at = torch.nonzero(t >= 0)[:, 0]
        order = at[torch.argsort(t[at], stable=True)]
        total = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device=DEV)
        total.index_put_((t[order],), d[order] * case["scale"], accumulate=True)
        return total + s["before"].double() if case["add"] else total
    if op == "ortho":
        a, b, c = COEF
        out = []
        for g in s["momentum"].double():
            x = g.T.contiguous() if case["rows"] > case["cols"] else g
            x = x / (torch.linalg.vector_norm(x) + 1e-7)
            eye = torch.eye(len(x), dtype=torch.float64, device=DEV)
            for _ in range(case["steps"]):
                gram = x @ x.T.contiguous()
                x = (a * eye + gram @ (b * eye + c * gram)) @ x
            out.append(x.T if case["rows"] > case["cols"] else x)
        return torch.stack(out).contiguous()
    parts, step = [], max(1, (1 << 26) // case["vocab"])
    for lo in range(0, case["n"], step):
        hi = min(case["n"], lo + step)
        lse, entropy, z, logp = _stats64(s, lo, hi)
        t = s["tokens"][lo:hi]
        rows = torch.arange(hi - lo, device=DEV)
        mine = z[rows, t.clamp(min=0)]
        if op == "logp":
            value = torch.where(mine > -math.inf, mine - lse, torch.full_like(mine, -math.inf))
            value = torch.where(t < 0, torch.zeros_like(value), value)
            sort = torch.sort(logp, 1, descending=True).values[:, : case["k"]]   # equal values are equal, whatever their order
            if sort.shape[1] < case["k"]:
                sort = torch.nn.functional.pad(sort, (0, case["k"] - sort.shape[1]), value=-math.inf)
            parts.append({"logp": value, "entropy": entropy, "lse": lse, "top_logp": sort})
            continue
        p = torch.where(z > -math.inf, logp.exp(), torch.zeros_like(z))
        slope = torch.where((t >= 0) & (mine > -math.inf), s["dlogp"][lo:hi].double(), torch.zeros_like(mine))
        d = -p * slope[:, None]
        d[rows, t.clamp(min=0)] += slope
        if s["dentropy"] is not None:
            inner = torch.where(z > -math.inf, logp, torch.zeros_like(z)) + entropy[:, None]
            d -= s["dentropy"][lo:hi, None].double() * p * inner
        parts.append(d * case["scale"])
    if op == "lgrad":
        return torch.cat(parts)
    got = {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    got["top_idx"] = None
    return got
