"""The gradient of log probabilities where a row's lse is far from zero, so that its
fp32 value does not hold the row's log sum: rows of nothing but a mask's value,
large offsets and scales.

Tolerances.  Up to |lse| = 1024 the given lse, rounded to 2^-24 of itself, is part of the
definition: log p is off by 4 u |lse|.  Past that nothing of lse's size is left, and
with b = (80 + V / 64) u for a log sum, log p is off by d = b + u (8 + 4 |log p| + 4 min(|lse|, 1024)).
A term is off by p (|g| + |h| (|log p| + |H| + 1)) d and a few roundings, then one
to the type."""
import math

import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


@pytest.mark.parametrize("n,vocab,dt,pad,offset,mask,scale", [
    (9, 20, "f32", 0, 0.0, -1e9, 1.0),
    (70, 221, "f32", 3, 0.0, -1e9, 0.75),
    (6, 300, "bf16", 0, 0.0, "lowest", 1.0),
    (6, 301, "f16", 1, 0.0, "lowest", 1.0),
    (6, 300, "f32", 0, 0.0, "lowest", 0.5),
    (5, 1100, "f32", 0, 3e5, None, 1.0),
    (4, 2100, "f32", 0, 0.0, None, 1e3),
    (5, 2100, "bf16", 5, 0.0, -1e12, 1.0),
    (4, 9000, "f32", 0, -1e6, -1e20, 1.0),
    (3, 40001, "bf16", 0, 3e4, -1e9, 1.0),
    (600, 40, "f16", 0, 0.0, -6e4, 1.0),
])
def test_gradient(P, n, vocab, dt, pad, offset, mask, scale):
    import torch
    print(f"[gpu-logprobs] far gradient {n} x {vocab} {dt} offset {offset} mask {mask} scale {scale}", flush=True)
    T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dt]
    gen = torch.Generator().manual_seed(n + vocab)
    x = torch.randn(n, vocab, generator=gen) * 3.0 + offset
    if mask is not None:
        low = torch.finfo(T).min if mask == "lowest" else mask
        x[torch.rand(n, vocab, generator=gen) < 0.4] = low
        x[0] = low
        x[n // 2] = low
    x = x.to(T)
    valid = torch.randint(1, vocab + 1, (n,), generator=gen).int()
    valid[0] = vocab
    tokens = (torch.rand(n, generator=gen) * valid).long()
    g, h = torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    z = (x.double() * scale).masked_fill(torch.arange(vocab)[None] >= valid[:, None], -math.inf)
    top = z.amax(1, keepdim=True)
    ls = torch.logsumexp(z - top, 1, keepdim=True)
    lp = z - top - ls
    p = lp.exp()
    lpf = torch.where(p > 0, lp, torch.zeros_like(lp))
    H = -(p * lpf).sum(1)
    lse = (top + ls)[:, 0]
    buf = torch.full((n, vocab + pad), 5.0, dtype=T, device=DEV)
    src = torch.full((n, vocab + pad), math.nan, dtype=T, device=DEV)
    src[:, :vocab] = x.to(DEV)
    P.at_logprobs_grad(src[:, :vocab], tokens.to(DEV), lse.float().to(DEV), H.float().to(DEV), g.to(DEV), buf[:, :vocab],
                       dentropy=h.to(DEV), valid=valid.to(DEV), scale=scale)
    got = buf.cpu()
    assert bool((got[:, vocab:] == 5.0).all())
    got, g, h = got[:, :vocab].double(), g.double()[:, None], h.double()[:, None]
    hot = torch.zeros_like(p).scatter_(1, tokens[:, None], 1.0)
    want = scale * (g * (hot - p) - h * p * (lpf + H[:, None]))
    size = lse.abs().clamp(max=1024.0)[:, None]
    d = U * (80 + vocab / 64) + U * (8 + 4 * lpf.abs() + 4 * size)
    weight = g.abs() + h.abs() * (lpf.abs() + H[:, None].abs() + 1)
    tol = scale * (p * weight * d + 8 * U * (p * weight + g.abs() * hot)) + ROUND[dt] * want.abs() + LEAST[dt]
    err = (got - want).abs()
    assert bool((err <= tol).all()), f"off by {float(err.max())}, {float((err - tol).max())} too much"
    assert bool((got[torch.arange(vocab)[None] >= valid[:, None]] == 0).all())
