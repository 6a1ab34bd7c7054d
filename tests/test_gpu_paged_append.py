"""Appending to a paged cache against a plain 64-bit form: norms, rotations, and where everything goes."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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


def turned(x, pos, freqs, interleaved, scale, weight, eps):
    """(result, magnitude) in 64 bits; magnitude: what relative errors of the inputs to a pair are relative to."""
    import torch
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(2, keepdim=True) + eps) * weight.double()
    r = len(freqs)
    if r == 0:
        return x, x.abs()
    t = pos.double()[:, None, None] * freqs
    i = torch.arange(r, device=DEV)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
    y, big = x.clone(), x.abs().clone()
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = (a * torch.cos(t) - b * torch.sin(t)) * scale
    y[..., ib] = (b * torch.cos(t) + a * torch.sin(t)) * scale
    big[..., ia] = big[..., ib] = (a.abs() + b.abs()) * abs(scale)
    return y, big


def check(P, R, x, rot, interleaved=False, scale=1.0, norm=False, stretch=1.0, with_q=True, eps=1e-6, shift=0):
    """Tolerance: in a pair, sine, cosine, two products, their sum and the factor are off by 8 u of |a| + |b| at most (u =
    2^-24; the reduced angle 2 u of a quarter turn); the norm by (D + 8) u relative; the result half a step of the type."""
    import torch
    n, u = x.n, 2.0 ** -24
    print(f"[gpu-append] {x.kind} new {list(x.new)[:6]} len {list(x.len)[:6]} heads {x.heads}/{x.kv} dim {x.dim} rot {rot} "
          f"page {x.page} interleaved {interleaved} norm {norm}", flush=True)
    k, v = x.randn(n, x.kv, x.dim), x.randn(n, x.kv, x.dim)
    freqs = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1)) / stretch
    kw, qw = ((1 + 0.2 * x.randn(x.dim).float()).to(x.q.dtype) for _ in range(2)) if norm else (None, None)
    before = x.k_cache.clone(), x.v_cache.clone()
    want_k, want_v, want_q = x.k_cache.double(), x.v_cache.double(), x.out.double()
    tol_k, tol_q = torch.zeros_like(want_k), torch.zeros_like(want_q)
    rel = (8 + (x.dim + 8 if norm else 0)) * u
    for b in range(x.batch):
        t = x.tokens(b)
        p = np.arange(x.len[b] - x.new[b], x.len[b]) + shift
        pos = torch.as_tensor(p - shift, device=DEV)
        if len(p) == 0:
            continue
        y, big = turned(x.q[t], pos, freqs, interleaved, scale, qw, eps)
        want_q[t], tol_q[t] = y, big * rel + y.abs() * R.step(x.kind) * (1 + 2 ** -6) + (2.0 ** -25 if x.kind == "f16" else 0)
        page, off = x.where(b, int(x.len[b] - x.new[b]))
        y, big = turned(k[t], pos, freqs, interleaved, scale, kw, eps)
        want_k[page, off], tol_k[page, off] = y, big * rel + y.abs() * R.step(x.kind) * (1 + 2 ** -6) + (2.0 ** -25 if x.kind == "f16" else 0)
        want_v[page, off] = v[t].double()
    q = dict(q=x.q, q_out=x.out, q_weight=qw) if with_q else {}
    P.at_paged_append(k, v, x.k_cache, x.v_cache, x.table, x.starts, x.lengths, freqs=freqs if rot else None,
                      interleaved=interleaved, rot_scale=scale, k_weight=kw, eps=eps, **q)
    torch.cuda.synchronize()
    R.close(x.k_cache, want_k, tol_k, "keys")
    R.close(x.v_cache, want_v, torch.zeros_like(want_v), "values")
    if with_q:
        R.close(x.out, want_q, tol_q, "queries")
    else:
        assert bool((x.out == 77).all())
    return before


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,rot", [(1, 0), (2, 2), (3, 2), (5, 4), (16, 16), (31, 30), (64, 64), (64, 32), (80, 40), (80, 16),
                                     (96, 0), (100, 100), (128, 128), (128, 6), (192, 128), (255, 254), (256, 256), (256, 64)])
def test_sizes(P, R, kind, dim, rot):
    for interleaved in (False, True):
        for norm in (False, True):
            check(P, R, R.Batch(kind, [3, 0, 1, 20], [5, 3, 0, 100], 6, 2, dim, page=16, seed=dim + rot, behind=2), rot,
                  interleaved, 1.25 if norm else 1.0, norm)


@pytest.mark.parametrize("page", [1, 3, 16, 24, 100])
@pytest.mark.parametrize("spread", ["tokens", "heads", "odd"])
def test_pages_and_layouts(P, R, page, spread):
    for kind in ("bf16", "f32"):
        check(P, R, R.Batch(kind, [1, 30, 1], [47, 0, 5], 8, 4, 64, page=page, spread=spread, seed=page), 64)


def test_many_tokens(P, R):
    """A workgroup a token, all heads; more sequences than lanes."""
    check(P, R, R.Batch("bf16", [1500, 40, 700], [9, 0, 3], 40, 8, 128, seed=1), 128)
    check(P, R, R.Batch("bf16", [1] * 300 + [0] * 4000 + [2] * 500, [3] * 4800, 4, 2, 32, page=4, seed=2, behind=9), 32, True)
    check(P, R, R.Batch("f32", [1100], [0], 3, 1, 24, seed=3), 12, True, norm=True)
    check(P, R, R.Batch("f16", [5], [8], 300, 100, 16, seed=4), 8)


@pytest.mark.parametrize("kind,heads,kv,dim,rot", [("bf16", 4, 2, 256, 256), ("f32", 2, 1, 256, 256), ("bf16", 12, 4, 128, 64),
                                                   ("bf16", 32, 8, 128, 128), ("f16", 64, 8, 80, 80), ("f32", 1, 1, 6, 6)])
@pytest.mark.parametrize("norm", [False, True])
def test_workgroups_of_every_size(P, R, kind, heads, kv, dim, rot, norm):
    check(P, R, R.Batch(kind, [800, 3], [9, 70], heads, kv, dim, page=24, seed=dim + heads), rot, norm=norm)


def test_without_queries(P, R):
    check(P, R, R.Batch("bf16", [4, 9], [1, 60], 8, 8, 64, seed=5), 64, with_q=False)


@pytest.mark.parametrize("ctx", [100_000, 5_000_000, 2 ** 31 - 40])
def test_far_positions(P, R, ctx):
    """Angles of far positions, whose product with a frequency 32 bits do not hold."""
    import torch
    x = R.Batch("f32", [20], [0], 4, 2, 64, page=16, seed=6)
    x.lengths += ctx
    x.len = x.len + ctx
    # the same pages, under a table that begins far out: only the last places of the sequence are there
    k, v = x.randn(x.n, 2, 64), x.randn(x.n, 2, 64)
    freqs = 10000.0 ** (-torch.arange(0, 64, 2, device=DEV, dtype=torch.float64) / 64)
    pos = torch.arange(ctx, ctx + 20, device=DEV)
    P.at_paged_append(k, v, x.k_cache, x.v_cache, x.table, x.starts, x.lengths, q=x.q, q_out=x.out, freqs=freqs)
    y, big = turned(x.q, pos, freqs, False, 1.0, None, 0.0)
    # 64-bit products are off by half a step: 2^-53 of the angle, in the oracle's and here, and again in the quarters
    R.close(x.out, y, big * (8 * 2.0 ** -24 + 4 * 2.0 ** -53 * ctx) + y.abs() * 2.0 ** -24)


def test_positions_that_are_not_there(P, R):
    """Not stored, and nothing else is touched; their queries are turned."""
    import torch
    x = R.Batch("bf16", [6, 3], [0, 20], 4, 2, 32, page=8, seed=7, fill=False)
    freqs = torch.ones(16, dtype=torch.float64, device=DEV)
    k, v = x.randn(x.n, 2, 32), x.randn(x.n, 2, 32)

    def stored(lengths, table):
        x.k_cache.fill_(9), x.v_cache.fill_(9)
        P.at_paged_append(k, v, x.k_cache, x.v_cache, table, x.starts, torch.tensor(lengths, dtype=torch.int32, device=DEV),
                          q=x.q, q_out=x.out, freqs=freqs)
        torch.cuda.synchronize()
        a, b = ((c != 9).any(3).any(2).sum() for c in (x.k_cache, x.v_cache))
        assert int(a) == int(b)
        return int(a)

    assert stored([6, 23], x.table) == 9
    assert stored([4, 23], x.table) == 7                      # positions -2 and -1
    assert stored([-5, 0], x.table) == 0
    assert stored([6, 25], x.table) == 8                      # position 24 is past the table's three pages
    assert stored([6, 2 ** 31 - 1], x.table) == 6
    bad = x.table.clone()
    bad[0, 0], bad[1, 2] = x.pages, -1
    assert stored([6, 23], bad) == 0
    assert stored([6, 23], x.table[:, :0]) == 0
    pos = torch.arange(-2, 4, device=DEV)
    P.at_paged_append(k, v, x.k_cache, x.v_cache, x.table, x.starts, torch.tensor([4, 23], dtype=torch.int32, device=DEV),
                      q=x.q, q_out=x.out, freqs=freqs)
    y, big = turned(x.q[:6], pos, freqs, False, 1.0, None, 0.0)
    R.close(x.out[:6], y, big * 2.0 ** -21 + y.abs() * 2.0 ** -8)


def test_in_place_and_inside_one_product(P, R):
    """q_out may be q; queries, keys and values may be parts of one row, at odd addresses."""
    import torch
    for kind, norm in (("bf16", False), ("f32", True)):
        x = R.Batch(kind, [40, 1, 9], [0, 33, 100], 6, 2, 80, page=16, seed=8)
        big = torch.full((x.n, 10 * 80 + 3), 5.0, dtype=x.q.dtype, device=DEV)
        qkv = big[:, 1: 801].unflatten(1, (10, 80))
        qkv.copy_(x.randn(x.n, 10, 80))
        q, k, v = qkv[:, :6], qkv[:, 6:8], qkv[:, 8:]
        w = x.randn(80) if norm else None
        freqs = torch.linspace(1, 0.01, 40, dtype=torch.float64, device=DEV)
        args = (x.k_cache, x.v_cache, x.table, x.starts, x.lengths)
        P.at_paged_append(k.contiguous(), v.contiguous(), *args, q=q.contiguous(), q_out=x.out, freqs=freqs, q_weight=w, k_weight=w)
        kc, vc = x.k_cache.clone(), x.v_cache.clone()
        x.k_cache.fill_(math.nan), x.v_cache.fill_(math.nan)
        for b in range(3):      # what was there before
            page, off = x.where(b, 0, int(x.len[b] - x.new[b]))
            x.k_cache[page, off], x.v_cache[page, off] = kc[page, off], vc[page, off]
        P.at_paged_append(k, v, *args, q=q, q_out=q, freqs=freqs, q_weight=w, k_weight=w)
        torch.cuda.synchronize()
        assert torch.equal(q, x.out)
        assert torch.equal(torch.nan_to_num(kc), torch.nan_to_num(x.k_cache)) and torch.equal(torch.nan_to_num(vc), torch.nan_to_num(x.v_cache))
        assert bool((big[:, 0] == 5).all()) and bool((big[:, 801:] == 5).all())


def test_captured_and_on_a_stream(P, R):
    import torch
    x = R.Batch("bf16", [1, 1, 1], [3, 40, 0], 4, 2, 64, seed=9, fill=False)
    freqs = torch.linspace(1, 0.01, 32, dtype=torch.float64, device=DEV)
    k, v = x.randn(x.n, 2, 64), x.randn(x.n, 2, 64)
    args = (k, v, x.k_cache, x.v_cache, x.table, x.starts, x.lengths)

    def run(**kw):
        P.at_paged_append(*args, q=x.q, q_out=x.out, freqs=freqs, **kw)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    s = torch.cuda.Stream()
    for lengths in ([4, 41, 1], [1, 1, 1], [7, 20, 3]):
        x.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        got = []
        for call in (g.replay, run, lambda: run(stream=s)):
            x.k_cache.fill_(3), x.v_cache.fill_(3), x.out.fill_(3)
            torch.cuda.synchronize()
            call()
            torch.cuda.synchronize()
            got.append((x.k_cache.clone(), x.v_cache.clone(), x.out.clone()))
        for other in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got[0], other))
        assert int((got[0][0] != 3).any(3).any(2).sum()) == 3


def test_offsets_past_32_bits(P, R):
    import torch
    pages = (1 << 32) // (8 * 128 * 128) + 8
    cache = [torch.zeros(pages, 128, 8, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    k, v = (torch.randn(200, 8, 128, device=DEV).bfloat16() for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device=DEV)
    P.at_paged_append(k, v, *cache, table, torch.tensor([0, 200], dtype=torch.int32, device=DEV),
                      torch.tensor([200], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for c, x in zip(cache, (k, v)):
        assert torch.equal(torch.cat([c[pages - 1], c[pages - 3, :72]]), x)
        assert int((c[pages - 3, 72:] != 0).sum()) == 0 and int((c[0] != 0).sum()) == 0
