"""Log probabilities of rows whose values lie far from zero: masks of finite
negative values, alone in a row, in a lane's columns or in a run of them, and large scales.

Tolerances.  With u = 2^-24, y = (x - m) c is off by 4 u |y| (the difference, the
product, the two roundings of c = scale log2(e)), so a weight 2^y is off by (4 + 4 |y|) u,
where |y| 2^y < 1; the sum of V weights adds V / 64 + 64 roundings: log sum is off by
b = (80 + V / 64) u.  log p = (x_t - m) scale - log sum has the roundings of its two terms
more, and nothing of the size of the row's values: 4 u (|z_t - z_max| + |log sum|).
The entropy is log sum less the mean of y, both as far off."""
import math

import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
INF = math.inf
VEC = {"f32": 4, "bf16": 8, "f16": 8}    # values a lane reads at once


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


def make(n, vocab, dt, mask, gen):
    """Row 0: nothing but the mask; 1: one lane's columns masked; 2: the first run of
    64 lanes' columns; 3: all but one; the others: half of them."""
    import torch
    x = torch.randn(n, vocab, generator=gen) * 3.0
    if mask is not None:
        at = torch.arange(vocab)
        x[0] = mask
        x[1, (at // VEC[dt]) % 64 == 5] = mask
        x[2, : min(64 * VEC[dt], vocab - 1)] = mask
        last = float(x[3, vocab // 3])
        x[3] = mask
        x[3, vocab // 3] = last
        half = torch.rand(n - 4, vocab, generator=gen) < 0.5
        x[4:][half] = mask
    return x.to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dt])


def exact(x, tokens, scale, k):
    import torch
    z = x.double() * scale
    top = z.amax(1, keepdim=True)
    ls = torch.logsumexp(z - top, 1)
    lp = (z - top) - ls[:, None]
    H = -(lp.exp() * lp).nan_to_num().sum(1)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    return top[:, 0], ls, lp, H, order


def close(got, want, tol, what):
    err = (got.cpu().double() - want).abs()
    assert bool((err <= tol).all()), f"{what}: off by {float(err.max())}, {float((err - tol).max())} too much"


CASES = [(n, vocab, dt, mask, 1.0)
         for dt, masks in (("f32", (-1e4, -1e9, -1e10, -1e12, -1e20, -1e30)), ("bf16", (-1e4, -1e10, -1e12, -1e20)),
                           ("f16", (-1e4, -6e4)))
         for mask in masks for n, vocab in ((8, 600), (6, 5003))]
CASES += [(3300, 1100, "f32", -1e10, 1.0), (3300, 2500, "bf16", -1e10, 1.0), (7, 64, "f32", -1e9, 1.0),
          (6, 131072, "bf16", -1e9, 0.5), (8, 600, "f32", None, 1e4), (6, 5003, "bf16", None, 1e3), (8, 600, "f16", None, 4096.0),
          (8, 600, "f32", -1e6, 1e3), (8, 600, "f32", None, 2.0 ** -10)]


@pytest.mark.parametrize("n,vocab,dt,mask,scale", CASES)
def test_forward(P, n, vocab, dt, mask, scale):
    import torch
    print(f"[gpu-logprobs] far {n} x {vocab} {dt} mask {mask} scale {scale}", flush=True)
    gen = torch.Generator().manual_seed(n + vocab)
    x = make(n, vocab, dt, mask, gen)
    tokens = torch.randint(0, vocab, (n,), generator=gen)
    tokens[n // 2] = int(x[n // 2].float().argmax())
    k = 7
    new = lambda *s: torch.full(s, 9.0, device=DEV)  # noqa: E731
    logp, H, lse, top = new(n), new(n), new(n), new(n, k)
    idx = torch.full((n, k), 7, dtype=torch.int32, device=DEV)
    P.at_logprobs(x.to(DEV), tokens.to(DEV), logp, H, lse, top, idx, scale=scale)
    zmax, ls, lp, w_H, w_idx = exact(x, tokens, scale, k)
    b = U * (80 + vocab / 64)
    w_logp, w_top = torch.gather(lp, 1, tokens[:, None])[:, 0], torch.gather(lp, 1, w_idx)
    close(logp, w_logp, b + 4 * U * (w_logp.abs() + 2 * ls.abs()), "logp")
    close(lse, zmax + ls, b + 2 * U * ((zmax + ls).abs() + ls.abs()), "lse")
    close(H, w_H, b * (2 + w_H) + 4 * U * (math.log(vocab + 1) + w_H), "entropy")
    assert torch.equal(idx.cpu().long(), w_idx)
    close(top, w_top, b + 4 * U * (w_top.abs() + 2 * ls.abs()[:, None]), "alternatives' log probabilities")
    assert bool((logp.cpu().double() <= b).all()) and bool((top.cpu().double() <= b).all())


@pytest.mark.parametrize("vocab", [40, 5003])
def test_largest_scale(P, vocab):
    """A scale whose product with log2(e) is past fp32's range: the largest value, twice
    in row 1, has all the probability."""
    import torch
    scale = 3e38
    x = -torch.rand(3, vocab, generator=torch.Generator().manual_seed(2)) - 0.125
    x[:, 7] = 0.0
    x[1, vocab - 2] = 0.0
    x[2] *= 0.5
    t = torch.tensor([7, 7, 9], device=DEV)
    new = lambda *s: torch.full(s, 9.0, device=DEV)  # noqa: E731
    logp, H, lse, top = new(3), new(3), new(3), new(3, 2)
    idx = torch.empty(3, 2, dtype=torch.int32, device=DEV)
    P.at_logprobs(x.to(DEV), t, logp, H, lse, top, idx, scale=scale)
    two, second = math.log(2.0), x[0].topk(2).indices[1]
    want = torch.tensor([0.0, -two, float(x[2, 9]) * scale])
    assert torch.allclose(logp.cpu(), want, rtol=1e-6, atol=1e-6)
    assert torch.allclose(H.cpu(), torch.tensor([0.0, two, 0.0]), atol=1e-6)
    assert torch.allclose(lse.cpu(), torch.tensor([0.0, two, 0.0]), atol=1e-6)
    assert idx[0].tolist() == [7, int(second)] and idx[1].tolist() == [7, vocab - 2]
    assert torch.allclose(top[:2].cpu(), torch.tensor([[0.0, float(x[0, second]) * scale], [-two, -two]]), rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("vocab", [40, 5003])
def test_tokens_far_past_the_row(P, vocab):
    """64-bit tokens past every column are ruled out, however large; negative ones are none."""
    import torch
    x = torch.randn(5, vocab, generator=torch.Generator().manual_seed(3)).to(DEV)
    t = torch.tensor([vocab, 1 << 61, 1 << 62, (1 << 63) - 1, -(1 << 63)], device=DEV)
    logp = torch.full((5,), 9.0, device=DEV)
    P.at_logprobs(x, t, logp)
    assert logp.tolist() == [-INF, -INF, -INF, -INF, 0.0]
