"""Log probabilities, entropies, alternatives and their gradient on the GPU
against the definition in 64 bits on the CPU.

Tolerances.  With u = 2^-24: the exponent (x - m) scale log2(e) is a
difference and a product, so a term's weight is off by at most about (4 + 4 |y|) u,
|y| e^-|y| < 1; the sum of V terms adds V / 64 + 64 roundings in a lane and
in the joins.  So log sum is off by (80 + V / 64) u, lse by two roundings of
its own size more, log p by those of z too; entropy weighs the same errors with
|log p| <= H-like averages, bounded by lse's own magnitude plus log V."""
import math

import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
INF = math.inf


def say(msg):
    print(f"[gpu-logprobs] {msg}", flush=True)


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make(n, vocab, kind, dtype, pad, gen):
    """[n, vocab] logits on the GPU, the gaps between rows NaN."""
    import torch
    x = torch.randn(n, vocab, generator=gen) * 3.0
    if kind == "ties":          # few different values, so that most are equal
        x = torch.randint(0, 3, (n, vocab), generator=gen).float()
    elif kind == "flat":
        x = torch.zeros(n, vocab)
    elif kind == "masked":      # -inf almost everywhere, one row with nothing
        x[torch.rand(n, vocab, generator=gen) < 0.9] = -INF
        x[n // 2] = -INF
    elif kind == "lowest":      # masked by the type's lowest value instead, one row by nothing else
        x[torch.rand(n, vocab, generator=gen) < 0.5] = torch.finfo(dtype).min
        x[n // 2] = torch.finfo(dtype).min
    elif kind == "peaked":
        x[torch.arange(n), torch.randint(0, vocab, (n,), generator=gen)] += 60.0
    elif kind == "rising":      # every value a new maximum
        x = torch.linspace(-20, 20, vocab).expand(n, vocab).clone()
    elif kind == "far":
        x = x + 500.0
    buf = torch.full((n, vocab + pad), float("nan"), dtype=dtype)
    buf[:, :vocab] = x.to(dtype)
    return buf.to(DEV)[:, :vocab]


def exact(x, tokens, valid, scale, k):
    """lse, entropy, logp in 64 bits; the alternatives' indices (stable order)."""
    import torch
    z = x.cpu().double() * scale
    n, vocab = z.shape
    if valid is not None:
        z = z.masked_fill(torch.arange(vocab)[None] >= valid[:, None], -INF)
    # less the maximum first: a row of the type's lowest value has finite log probabilities
    top = z.amax(1)
    base = torch.where(top > -INF, top, torch.zeros_like(top))[:, None]
    rest = torch.logsumexp(z - base, 1)
    lse = torch.where(top > -INF, base[:, 0] + rest, top)
    lp = (z - base) - torch.where(top > -INF, rest, torch.zeros_like(rest))[:, None]
    p = torch.where(z > -INF, lp.exp(), torch.zeros_like(z))
    H = -torch.where(z > -INF, p * lp, torch.zeros_like(z)).sum(1)
    logp = torch.zeros(n, dtype=torch.float64)
    for i in range(n):
        t = int(tokens[i])
        if t >= 0:
            logp[i] = lp[i, t] if t < vocab and z[i, t] > -INF else -INF
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    idx = torch.full((n, k), -1, dtype=torch.int64)
    idx[:, : order.shape[1]] = order
    found = torch.gather(z, 1, order) > -INF
    idx[:, : order.shape[1]][~found] = -1
    return lse, H, logp, idx, lp, p


CASES = [
    # n, vocab, type, k, pad, kind, ragged, scale
    (1, 1, "f32", 1, 0, "plain", False, 1.0),
    (3, 2, "bf16", 5, 1, "plain", False, 1.0),
    (5, 64, "f32", 64, 0, "plain", False, 0.5),
    (64, 220, "f32", 8, 0, "masked", True, 1.0),
    (33, 220, "f16", 8, 3, "plain", True, 1.25),
    (9, 513, "bf16", 64, 0, "ties", False, 1.0),
    (8, 2048, "f32", 10, 0, "flat", False, 1.0),
    (6, 2049, "f32", 10, 0, "flat", False, 1.0),
    (4, 3000, "bf16", 64, 1, "ties", True, 1.0),
    (7, 5001, "f16", 20, 7, "masked", False, 1.0),
    (5, 10007, "f32", 64, 0, "rising", False, 1.0),
    (6, 4100, "f32", 5, 0, "lowest", True, 1.0),
    (6, 300, "f32", 5, 0, "lowest", False, 0.5),
    (6, 4100, "bf16", 5, 0, "lowest", False, 1.0),
    (1, 131072, "bf16", 20, 0, "plain", False, 1.25),
    (2, 50001, "f32", 64, 47, "peaked", False, 1.0),
    (3, 70000, "f16", 0, 0, "far", True, 1.0),
    (1500, 2100, "bf16", 3, 0, "plain", True, 1.0),
    (1300, 33, "f32", 4, 0, "masked", True, 2.0),
    (3300, 2501, "bf16", 33, 1, "plain", True, 1.0),
    (3201, 4097, "f32", 2, 0, "lowest", False, 1.0),
]


@pytest.mark.parametrize("n,vocab,dt,k,pad,kind,ragged,scale", CASES)
def test_forward(P, n, vocab, dt, k, pad, kind, ragged, scale):
    import torch
    say(f"forward {n} x {vocab} {dt} k {k} {kind} ragged {ragged}")
    gen = torch.Generator().manual_seed(n * 11 + vocab)
    x = make(n, vocab, kind, types()[dt], pad, gen)
    valid = torch.randint(0, vocab + 1, (n,), generator=gen).int() if ragged else None
    if ragged:
        valid[0], valid[-1] = 0, vocab + 5     # nothing, and more than there is
    tokens = torch.randint(0, vocab, (n,), generator=gen)
    tokens[n // 3] = -1
    if n > 4:
        tokens[4] = vocab + 3
    new = lambda *s: torch.full(s, 9.0, device=DEV)  # noqa: E731
    logp, H, lse, top = new(n), new(n), new(n), new(n, k)
    idx = torch.full((n, k), 7, dtype=torch.int32, device=DEV)
    P.at_logprobs(x, tokens.to(DEV), logp, H, lse, top if k else None, idx if k else None,
                  valid=valid.to(DEV) if ragged else None, scale=scale)
    w_lse, w_H, w_logp, w_idx, w_lp, _ = exact(x, tokens, valid, scale, k)
    base = U * (80 + vocab / 64)

    def close(got, want, tol, what):
        got = got.cpu().double()
        fin = torch.isfinite(want)
        assert torch.equal(torch.isfinite(got), fin), what
        assert torch.equal(got[~fin], want[~fin]), what
        err = (got - want)[fin].abs()
        assert bool((err <= tol[fin]).all()), f"{what}: {float(err.max())}"

    size = torch.where(torch.isfinite(w_lse), w_lse.abs(), torch.zeros_like(w_lse))
    zmax = size + 4
    close(lse, w_lse, base + 2 * U * size, "lse")
    close(logp, w_logp, base + 4 * U * (size + w_logp.abs().clamp(max=1e38)), "logp")
    close(H, w_H, base * (2 + w_H) + 4 * U * (math.log(vocab + 1) + w_H), "entropy")
    if k:
        assert torch.equal(idx.cpu().long(), w_idx), "alternatives"
        want = torch.where(w_idx >= 0, torch.gather(w_lp, 1, w_idx.clamp(min=0)), torch.full(w_idx.shape, -INF, dtype=torch.float64))
        close(top, want, (base + 4 * U * (zmax[:, None] + want.abs().clamp(max=1e38))), "alternatives' log probabilities")


def test_outputs_are_optional(P):
    import torch
    gen = torch.Generator().manual_seed(3)
    for vocab in (100, 5000):
        x = make(4, vocab, "plain", torch.float32, 0, gen)
        t = torch.tensor([0, 1, 2, 3], device=DEV)
        new = lambda *s: torch.full(s, 9.0, device=DEV)  # noqa: E731
        a, b, idx = new(4), new(4), torch.empty(4, 3, dtype=torch.int32, device=DEV)
        P.at_logprobs(x, t, a, new(4), new(4), new(4, 3), idx)
        P.at_logprobs(x, t, b)
        assert torch.equal(a, b)
        e1, e2, i2 = new(4), new(4), torch.empty_like(idx)
        P.at_logprobs(x, None, None, e1)
        P.at_logprobs(x, None, None, e2, None, None, i2)
        assert torch.equal(e1, e2) and torch.equal(idx, i2)


@pytest.mark.parametrize("vocab", [70, 3000, 40000])
def test_poisoned_rows(P, vocab):
    """NaN and +inf spoil their own row only; past valid they are not read."""
    import torch
    gen = torch.Generator().manual_seed(4)
    x = make(6, vocab, "plain", torch.float32, 0, gen)
    x[1, vocab // 2] = float("nan")
    x[3, vocab - 1] = INF
    x[4, vocab - 1] = float("nan")
    valid = torch.full((6,), vocab, dtype=torch.int32, device=DEV)
    valid[4] = vocab - 1
    t = torch.zeros(6, dtype=torch.int64, device=DEV)
    out = [torch.empty(6, device=DEV) for _ in range(3)]
    top, idx = torch.empty(6, 4, device=DEV), torch.empty(6, 4, dtype=torch.int32, device=DEV)
    P.at_logprobs(x, t, *out, top, idx, valid=valid)
    bad = torch.tensor([False, True, False, True, False, False])
    for o in out:
        assert torch.equal(torch.isnan(o.cpu()), bad)
    assert torch.equal(torch.isnan(top.cpu()), bad[:, None].expand(6, 4))
    assert torch.equal((idx.cpu() == -1), bad[:, None].expand(6, 4))
    d = torch.empty_like(x)
    P.at_logprobs_grad(x, t, out[2], out[1], torch.ones(6, device=DEV), d, valid=valid)
    d = d.cpu()
    assert torch.equal(torch.isnan(d).any(1), bad)
    assert float(d[4, vocab - 1]) == 0.0


ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.mark.parametrize("n,vocab,dt,pad,kind,ragged,scale,entropy", [
    (1, 1, "f32", 0, "plain", False, 1.0, True),
    (3, 2, "bf16", 1, "plain", False, 1.0, True),
    (64, 220, "f32", 0, "masked", True, 1.0, True),
    (33, 221, "f16", 3, "plain", True, 1.25, False),
    (7, 1025, "bf16", 0, "ties", False, 0.5, True),
    (5, 8192, "bf16", 0, "peaked", False, 1.0, True),
    (4, 8195, "f32", 5, "masked", True, 1.0, True),
    (3, 40001, "f16", 0, "far", False, 1.0, True),
    (6, 300, "f32", 0, "lowest", False, 0.5, True),
    (1200, 40, "bf16", 0, "masked", True, 1.0, True),
])
def test_gradient(P, n, vocab, dt, pad, kind, ragged, scale, entropy):
    """Elementwise: with log p off by d = (8 + 4 |lse| + 4 |z|) u at most (the given
    lse is rounded too), a term is off by p (|g| + |h| (|log p| + |H| + 1)) d
    and a few roundings of the terms, then one to the type."""
    import torch
    say(f"gradient {n} x {vocab} {dt} {kind} ragged {ragged}")
    gen = torch.Generator().manual_seed(n * 13 + vocab)
    x = make(n, vocab, kind, types()[dt], pad, gen)
    valid = torch.randint(0, vocab + 1, (n,), generator=gen).int() if ragged else None
    tokens = torch.randint(0, vocab, (n,), generator=gen)
    tokens[n // 3] = -1
    lse, H, _, _, lp, p = exact(x, tokens, valid, scale, 0)
    g, h = torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    buf = torch.full((n, vocab + pad), 5.0, dtype=x.dtype, device=DEV)
    P.at_logprobs_grad(x, tokens.to(DEV), lse.float().to(DEV), H.float().to(DEV), g.to(DEV), buf[:, :vocab],
                       dentropy=h.to(DEV) if entropy else None, valid=valid.to(DEV) if ragged else None, scale=scale)
    got = buf.cpu()
    assert bool((got[:, vocab:] == 5.0).all()), "wrote past a row"
    got = got[:, :vocab].double()
    g, h = g.double()[:, None], h.double()[:, None] * float(entropy)
    t = tokens.clamp(min=0)[:, None]
    live = (tokens[:, None] >= 0) & (torch.gather(p, 1, t) >= 0) & (torch.gather(lp, 1, t) > -INF)
    if valid is not None:
        live &= t < valid[:, None]
    g = torch.where(live, g, torch.zeros_like(g))
    hot = torch.zeros_like(p).scatter_(1, t, 1.0) * live
    lpf = torch.where(p > 0, lp, torch.zeros_like(lp))
    want = scale * (g * (hot - p) - h * p * (lpf + H[:, None]))
    size = torch.where(torch.isfinite(lse), lse.abs(), torch.zeros_like(lse))[:, None]
    z = torch.where(p > 0, (lp + size).abs() + size, torch.zeros_like(p))
    d = U * (8 + 4 * size + 4 * z)
    mag = g.abs() * (hot + p) + h.abs() * p * (lpf.abs() + H[:, None].abs() + 1)
    tol = scale * (p * (g.abs() + h.abs() * (lpf.abs() + H[:, None].abs() + 1)) * d + 8 * U * mag) + ROUND[dt] * want.abs()
    tol += {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}[dt]
    err = (got - want).abs()
    assert bool((err <= tol).all()), f"largest excess {float((err - tol).max())}"
    if valid is not None:
        assert bool((got[torch.arange(vocab)[None] >= valid[:, None]] == 0).all())
    assert bool((got[(x.cpu().double() == -INF)] == 0).all())


def test_gradient_against_differences(P):
    """Central differences of the 64-bit definition along random directions:
    with step e the truncation is about e^2 times the third derivative, a
    polynomial in p, log p and H of size below 100 here, and the kernel's error
    U-sized: 1e-4 covers both at e = 1e-3."""
    import torch
    gen = torch.Generator().manual_seed(21)
    n, vocab, scale = 40, 150, 0.8
    x = make(n, vocab, "plain", torch.float32, 0, gen)
    valid = torch.randint(5, vocab + 1, (n,), generator=gen).int()
    tokens = (torch.rand(n, generator=gen) * valid).long()
    g, h = torch.randn(n, generator=gen).double(), torch.randn(n, generator=gen).double()

    def value(y):
        lse, H, logp, _, _, _ = exact(y, tokens, valid, scale, 0)
        return g * logp + h * H

    lse, H, _, _, _, _ = exact(x, tokens, valid, scale, 0)
    d = torch.empty_like(x)
    P.at_logprobs_grad(x, tokens.to(DEV), lse.float().to(DEV), H.float().to(DEV), g.float().to(DEV), d,
                       dentropy=h.float().to(DEV), valid=valid.to(DEV), scale=scale)
    e, base = 1e-3, x.cpu().double()
    for _ in range(5):
        v = torch.randn(n, vocab, generator=gen).double()
        slope = (value(base + e * v) - value(base - e * v)) / (2 * e)
        assert float((slope - (d.cpu().double() * v).sum(1)).abs().max()) < 1e-4


def test_long_row_past_32_bits(P):
    """Rows far apart: the last one starts past 2^32 bytes (and 2^31 elements)."""
    import torch
    gen = torch.Generator().manual_seed(6)
    n, vocab, ld = 3, 1000, (1 << 30) + 1
    buf = torch.empty((n - 1) * ld + vocab, dtype=torch.float16, device=DEV)
    x = torch.as_strided(buf, (n, vocab), (ld, 1))
    x.copy_(torch.randn(n, vocab, generator=gen).half().to(DEV))
    t = torch.tensor([5, 6, 7], device=DEV)
    got, want = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    P.at_logprobs(x, t, got)
    P.at_logprobs(x.contiguous(), t, want)
    assert torch.equal(got, want)


def test_gradient_past_32_bits(P):
    """Logits and gradients whose last rows start past 2^31 elements, and 64-bit
    tokens whose low words are in range."""
    import torch
    gen = torch.Generator().manual_seed(7)
    n, vocab, ld = 4, 1000, (1 << 30) + 1
    bufs = [torch.empty((n - 1) * ld + vocab, dtype=torch.float16, device=DEV) for _ in range(2)]
    x, d = (torch.as_strided(b, (n, vocab), (ld, 1)) for b in bufs)
    x.copy_(torch.randn(n, vocab, generator=gen).half().to(DEV))
    t = torch.tensor([5, (1 << 32) + 6, 7, 8], device=DEV)
    logp, lse, g = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.ones(n, device=DEV)
    P.at_logprobs(x, t, logp, lse=lse)
    assert bool(torch.isfinite(lse).all())
    P.at_logprobs_grad(x, t, lse, None, g, d)
    want = torch.empty(n, vocab, dtype=torch.float16, device=DEV)
    P.at_logprobs_grad(x.contiguous(), t, lse, None, g, want)
    assert torch.equal(d, want)
    assert bool((d[1] == 0).all()) and not bool((d[0] == 0).all())


def test_graph_and_streams(P):
    import torch
    gen = torch.Generator().manual_seed(8)
    n, vocab, k = 2, 30000, 6
    x = make(n, vocab, "plain", torch.bfloat16, 0, gen)
    t = torch.randint(0, vocab, (n,), generator=gen).to(DEV)
    new = lambda: (torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV),  # noqa: E731
                   torch.zeros(n, k, device=DEV), torch.zeros(n, k, dtype=torch.int32, device=DEV))
    ws = torch.full((P.at_logprobs_workspace(n, vocab, k),), 0xFF, dtype=torch.uint8, device=DEV)
    a, d = new(), torch.zeros_like(x)
    one = torch.ones(n, device=DEV)
    P.at_logprobs(x, t, *a, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.at_logprobs(x, t, *a, workspace=ws)
        P.at_logprobs_grad(x, t, a[2], a[1], one, d, dentropy=one)
    for k_ in range(4):
        x.copy_(torch.randn(n, vocab, generator=gen).to(torch.bfloat16))
        b, e = new(), torch.empty_like(x)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        P.at_logprobs(x, t, *b, stream=side)
        P.at_logprobs_grad(x, t, b[2], b[1], one, e, dentropy=one, stream=side)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, b)) and torch.equal(d, e), k_
