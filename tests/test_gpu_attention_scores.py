"""Attention whose scores are finite but large: what counts is their distance from the row's maximum.

Queries and keys are chosen so that scores come out the same, or exact, in fp32 sums of any order.  Weights are then
off by their own roundings only, with u = 2^-24: 3 u of a distance of at most 32 in the argument of 2^x (67 u of the weight), 2 u in 2^x,
at most six times 2 u where sums are scaled down, 8 u in joining pieces, 89 u together; half a step where weights are rounded to the
type; 2 (L + 8) u in sums over L keys."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


@pytest.fixture(scope="module")
def R():
    import paged_reference
    return paged_reference


# one piece, several pieces, tiles that are shared by waves of rows, and prompts
CALLS = [([1], [40]), ([1, 2], [5000, 700]), ([70, 3], [30, 900]), ([300], [0]), ([40], [6000])]


def check(R, x, scores, lse_off, what):
    """out and lse of x against scores [n, L] (of every head), which are exact but for lse_off."""
    import torch
    for b in range(x.batch):
        t, L, m = x.tokens(b), int(x.len[b]), int(x.new[b])
        page, off = x.where(b)
        v = x.v_cache[page, off].double().repeat_interleave(x.heads // x.kv, 1).transpose(0, 1).contiguous()      # [heads, L, D]
        seen = torch.arange(L, device=DEV)[None] <= torch.arange(L - m, L, device=DEV)[:, None]
        s = torch.where(seen, scores(b, L, m).double().expand(m, L), torch.full((), -math.inf, device=DEV, dtype=torch.float64))
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        p = (p / total).expand(x.heads, m, L)
        want, size = torch.bmm(p, v).transpose(0, 1), torch.bmm(p, v.abs()).transpose(0, 1)
        rel = 2 * (L + 8) * U + 89 * U + (R.step(x.kind) if x.kind != "f32" else 0.0)
        extra = L * 2.0 ** -36 * float(v.abs().max()) + 2.0 ** -25 if x.kind == "f16" else 0.0
        R.close(x.out[t], want, size * rel + want.abs() * R.step(x.kind) * (1 + 2 ** -6) + extra, f"{what} out of {b}")
        lse = (top + torch.log(total)).expand(m, x.heads)
        R.close(x.lse[t], lse, (L + 8 + 89) * U + 4 * U * lse.abs() + lse_off, f"{what} lse of {b}")


# values whose squares, times the number of values, fp32 holds
CONSTANTS = [("f16", 4000.0), ("f16", 4104.0), ("f16", 30000.0), ("bf16", 4000.0), ("bf16", 29952.0), ("bf16", 2.0 ** 30), ("bf16", 2.0 ** 59),
             ("f32", 4000.0), ("f32", 29952.0), ("f32", 1e9), ("f32", 5e17)]


@pytest.mark.parametrize("kind,c", CONSTANTS)
@pytest.mark.parametrize("dim", [64, 128, 192])
def test_equal_scores(P, R, kind, c, dim):
    """All of a row's scores are the same: the mean of its values."""
    import torch
    for new, ctx in CALLS:
        for sign in (1, -1):
            print(f"[gpu-scores] {kind} {c} dim {dim} new {new} ctx {ctx} sign {sign}", flush=True)
            x = R.Batch(kind, new, ctx, 4, 2, dim, page=16, seed=dim)
            x.q.fill_(c)
            for b in range(x.batch):
                page, off = x.where(b)
                x.k_cache[page, off] = sign * c
                x.v_cache[page, off] = torch.where(torch.arange(len(page), device=DEV) % 3 == 0, 3.0, -1.0).to(x.q.dtype)[:, None, None].expand(-1, 2, dim)
            x.attend(P)
            torch.cuda.synchronize()
            score = sign * float(x.q[0, 0, 0]) ** 2 * dim * dim ** -0.5
            check(R, x, lambda b, L, m: torch.full((1, L), score, device=DEV, dtype=torch.float64), (dim + 8) * U * abs(score), "equal")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 128, 256])
def test_large_scores_that_differ(P, R, kind, dim):
    """Scores about 2^30 / 256 whose distances, multiples of a half, are exact; maxima differ from tile to tile and piece to piece."""
    import torch
    for new, ctx in CALLS:
        print(f"[gpu-scores] {kind} differ dim {dim} new {new} ctx {ctx}", flush=True)
        x = R.Batch(kind, new, ctx, 4, 2, dim, page=16, seed=dim)
        rng = np.random.default_rng(dim)
        x.q.zero_()
        x.q[..., 0], x.q[..., 1] = 2.0 ** 15, 1.0
        steps = []
        for b in range(x.batch):
            page, off = x.where(b)
            L = len(page)
            m = torch.as_tensor(np.arange(L) * 24 // L + rng.integers(0, 9, L), device=DEV)
            x.k_cache[page, off] = 0.0
            x.k_cache[page, off, :, 0] = 2.0 ** 15
            x.k_cache[page, off, :, 1] = (128.0 * m).to(x.q.dtype)[:, None].expand(-1, 2)
            steps.append(m)
        x.attend(P, scale=2.0 ** -8)
        torch.cuda.synchronize()
        check(R, x, lambda b, L, m: 2.0 ** 22 + 0.5 * steps[b].double()[None], 0.0, "differ")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_largest_scales(P, R, kind):
    """A scale up to fp32's largest: equal scores weigh the same, others nothing."""
    import torch
    top = torch.finfo(torch.float32).max
    for scale in (top, 2.5e38, 2.0 ** 127):
        for new, ctx in CALLS:
            print(f"[gpu-scores] {kind} scale {scale} new {new} ctx {ctx}", flush=True)
            x = R.Batch(kind, new, ctx, 4, 2, 64, page=16, seed=3)
            x.q.zero_()
            x.attend(P, scale=scale)
            torch.cuda.synchronize()
            check(R, x, lambda b, L, m: torch.zeros(1, L, device=DEV, dtype=torch.float64), 0.0, "zeros")
            if kind == "f16":   # whose products do not come near 2^-120
                continue
            x.q.fill_(2.0 ** -63)
            for b in range(x.batch):
                page, off = x.where(b)
                x.k_cache[page, off] = torch.where(torch.arange(len(page), device=DEV) % 2 == 0, 2.0 ** -63, -2.0 ** -63).to(x.q.dtype)[:, None, None].expand(-1, 2, 64)
            x.attend(P, scale=scale)
            torch.cuda.synchronize()
            check(R, x, lambda b, L, m: 2.0 ** -120 * scale * torch.where(torch.arange(L, device=DEV) % 2 == 0, 1.0, -1.0)[None].double(), 0.0, "tiny")
