"""Attention over a paged cache against a plain 64-bit form.  Every place of a
cache that a call must not read holds NaN."""
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


def say(msg):
    print(f"[gpu-attend] {msg}", flush=True)


def check(P, R, x, scale=None, window=0, gone=None, **kw):
    import torch
    scale = x.dim ** -0.5 if scale is None else scale
    say(f"{x.kind} new {list(x.new)[:6]} len {list(x.len)[:6]} heads {x.heads}/{x.kv} dim {x.dim} page {x.page} window {window}")
    want, lse, tol, tol_lse = R.attention64(x, scale, window, gone)
    x.attend(P, scale=scale, window=window, **kw)
    torch.cuda.synchronize()
    R.close(x.lse, lse, tol_lse, "lse")
    R.close(x.out, want, tol, "out")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [1, 3, 16, 31, 32, 40, 64, 80, 100, 127, 128, 136, 192, 248, 256])
def test_head_sizes(P, R, kind, dim):
    """Single tokens and prompts, each head size of every padding, sizes that are no multiple of 16 bytes."""
    check(P, R, R.Batch(kind, [1, 1, 1], [0, 5, 300], 4, 2, dim, page=16, seed=dim))
    check(P, R, R.Batch(kind, [70, 1, 33], [0, 5, 200], 4, 2, dim, page=16, seed=dim + 1))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [72, 80, 88, 96, 104, 120, 160, 176, 192, 208])
def test_padded_heads_in_whole_tiles(P, R, kind, dim):
    """Heads that leave part of their padding unused, over keys of which every query sees whole tiles."""
    check(P, R, R.Batch(kind, [300, 70], [700, 5], 4, 2, dim, page=16, seed=dim))
    check(P, R, R.Batch(kind, [40, 1], [900, 640], 4, 2, dim, page=64, seed=dim + 1), window=500)


@pytest.mark.parametrize("kind,dim", [("f32", 255), ("bf16", 255), ("f16", 132)])
def test_large_heads_of_odd_rows_are_refused(P, R, kind, dim):
    for new in ([1], [70]):
        x = R.Batch(kind, new, [40], 4, 2, dim)
        with pytest.raises(P.ATError) as e:
            x.attend(P)
        assert e.value.status == -2
    x = R.Batch(kind, [1], [40], 4, 2, 192, spread="odd")
    with pytest.raises(P.ATError):
        x.attend(P)


@pytest.mark.parametrize("page", [1, 3])
def test_large_heads_in_odd_pages(P, R, page):
    """Two rows of a move to LDS in different pages."""
    for kind, dim in (("bf16", 256), ("f16", 160), ("f32", 192)):
        check(P, R, R.Batch(kind, [1, 1], [300, 9], 4, 2, dim, page=page, seed=dim))
        check(P, R, R.Batch(kind, [70, 3], [30, 100], 4, 2, dim, page=page, seed=dim))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 5), (7, 1), (12, 3), (32, 8), (40, 1), (64, 2)])
def test_head_groups(P, R, kind, heads, kv):
    check(P, R, R.Batch(kind, [1, 1], [130, 17], heads, kv, 64, seed=heads))
    check(P, R, R.Batch(kind, [3, 40], [130, 17], heads, kv, 64, seed=heads + 1))


@pytest.mark.parametrize("page", [1, 2, 7, 16, 24, 100, 128, 1000])
@pytest.mark.parametrize("spread", ["tokens", "heads", "odd"])
def test_pages_and_layouts(P, R, page, spread):
    """Pages that end inside tiles, and every distance between pages, places and heads."""
    for kind, dim in (("bf16", 64), ("f32", 48), ("bf16", 128)):
        check(P, R, R.Batch(kind, [1, 1, 1], [0, 257, 640], 8, 2, dim, page=page, spread=spread, seed=page))
        check(P, R, R.Batch(kind, [129, 65], [63, 0], 8, 2, dim, page=page, spread=spread, seed=page + 1))


@pytest.mark.parametrize("window", [1, 2, 31, 64, 65, 500, 10 ** 9])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_windows(P, R, kind, window):
    """Places before every token's window hold NaN too."""
    import torch
    for new, ctx, heads in (([1, 1], [700, 3], 8), ([150, 30], [300, 0], 4), ([257], [0], 2)):
        x = R.Batch(kind, new, ctx, heads, 2, 64, page=24, seed=window % 1000)
        for b in range(x.batch):
            page, off = x.where(b, 0, max(0, int(ctx[b]) - window + 1))
            for c in (x.k_cache, x.v_cache):
                c[page, off] = math.nan
        keep = x.k_cache, x.v_cache
        x.k_cache, x.v_cache = (torch.nan_to_num(c) for c in keep)
        want = R.attention64(x, 0.125, window)
        x.k_cache, x.v_cache = keep
        x.attend(P, scale=0.125, window=window)
        torch.cuda.synchronize()
        R.close(x.lse, want[1], want[3], "lse")
        R.close(x.out, want[0], want[2], "out")


@pytest.mark.parametrize("window", [1, 33, 300])
@pytest.mark.parametrize("dim", [65, 80, 96, 100, 112, 128])
def test_narrow_tiles(P, R, dim, window):
    """fp32 under a window that is short of what there is: tiles of 32 keys, whole ones, cut ones, and pages of every end."""
    for new, ctx, heads, page in (([200, 90], [400, 700], 4, 16), ([40], [2500], 2, 24), ([700], [0], 12, 7)):
        x = R.Batch("f32", new, ctx, heads, 2, dim, page=page, seed=dim + window)
        check(P, R, x, window=window)


@pytest.mark.parametrize("window", [64, 1000, 3000, 2 ** 63 - 1])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_windows_of_cut_keys(P, R, kind, window):
    """Pieces start where the window of their rows does."""
    for new, ctx, heads in (([1, 1], [6000, 2500], 4), ([40], [5000], 4), ([300, 20], [4000, 100], 2)):
        check(P, R, R.Batch(kind, new, ctx, heads, 2, 80 if kind == "f32" else 128, page=24, seed=len(new)), window=window)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new,ctx,heads,kv", [([500, 260, 500], [0, 30, 900], 16, 8), ([600], [0], 32, 16), ([1200], [300], 4, 4),
                                              ([64] * 5, [100, 0, 2000, 5, 300], 16, 4), ([2100], [0], 8, 8)])
def test_row_tiles(P, R, kind, new, ctx, heads, kv):
    """Tiles of rows of every size, with keys cut and whole."""
    check(P, R, R.Batch(kind, new, ctx, heads, kv, 64, page=16, seed=len(new)))


@pytest.mark.parametrize("ctx", [0, 1, 31, 32, 33, 63, 64, 127, 128, 129, 511, 512, 513, 2047, 5000])
def test_lengths(P, R, ctx):
    """Lengths around the edges of tiles and of pieces."""
    check(P, R, R.Batch("bf16", [1], [ctx], 8, 2, 128, seed=ctx))
    check(P, R, R.Batch("bf16", [5], [ctx], 8, 2, 128, seed=ctx + 1))
    check(P, R, R.Batch("f16", [37, 1], [ctx, ctx // 2], 8, 2, 64, seed=ctx + 2))


def test_long_and_cut(P, R):
    """Long sequences of few rows, cut into many pieces, beside short and empty ones."""
    check(P, R, R.Batch("bf16", [1, 1, 0, 1, 1], [40000, 3, 900, 0, 7777], 8, 2, 64, page=32, seed=5))
    check(P, R, R.Batch("f32", [2, 0, 1], [20000, 0, 1], 4, 2, 32, page=16, seed=6))
    check(P, R, R.Batch("f16", [300], [9000], 4, 1, 64, page=64, seed=7))
    check(P, R, R.Batch("bf16", [300, 2], [9000, 30], 4, 1, 64, page=64, seed=8), window=2500)


def test_large_batches(P, R):
    """More sequences than a workgroup has threads, most of them short, some with no new tokens."""
    rng = np.random.default_rng(3)
    for many in (257, 1500):
        check(P, R, R.Batch("bf16", rng.integers(0, 2, many), rng.integers(0, 60, many), 4, 2, 32, page=8, seed=many, behind=5))
    check(P, R, R.Batch("bf16", rng.integers(0, 40, 300), rng.integers(0, 60, 300), 2, 2, 32, page=8, seed=9, behind=50))


def test_rows_behind_and_empty_sequences(P, R):
    """Tokens of no sequence keep what was there; a token that sees nothing gets zeros and -inf."""
    import torch
    x = R.Batch("bf16", [0, 3, 0, 1, 0], [5, 9, 0, 0, 70], 4, 2, 64, behind=7, seed=1)
    check(P, R, x)
    assert bool((x.out[4:] == 77).all()) and bool((x.lse[4:] == 77).all())
    # lengths below the number of new tokens: the first of them have no position
    for new in ([6], [200]):
        x = R.Batch("bf16", new, [0], 4, 2, 64, seed=2)
        x.lengths.fill_(4)
        x.attend(P)
        assert bool((x.out[: new[0] - 4] == 0).all()) and bool((x.lse[: new[0] - 4] == -math.inf).all())
        y = R.Batch("bf16", [4], [0], 4, 2, 64, seed=2)
        y.k_cache, y.v_cache, y.table_h, y.q = x.k_cache, x.v_cache, x.table_h, x.q[new[0] - 4:]
        y.out, y.lse = x.out[new[0] - 4:], x.lse[new[0] - 4:]
        want = R.attention64(y, 0.125)
        R.close(y.out, want[0], want[2])
        for bad in (0, -3):
            x.lengths.fill_(bad)
            x.out.fill_(5), x.lse.fill_(5)
            x.attend(P)
            assert bool((x.out == 0).all()) and bool((x.lse == -math.inf).all())
    # a batch of no sequence, and starts that begin after the first tokens
    x = R.Batch("f32", [3, 2], [4, 8], 2, 2, 16, seed=3)
    x.starts += 2
    x.q = torch.cat([x.q, x.q])[:8].contiguous()
    x.out, x.lse = torch.full((8, 2, 16), 77.0, device=DEV), torch.full((8, 2), 77.0, device=DEV)
    x.n, x.starts_h = 8, x.starts_h + 2
    check(P, R, x)
    assert bool((x.out[:2] == 77).all()) and bool((x.out[7:] == 77).all())


def test_pages_that_are_not_there(P, R):
    """Page numbers outside the cache, and positions past the table, hold nothing."""
    import torch
    for new, ctx in (([1, 1], [200, 90]), ([40, 1], [200, 90])):
        x = R.Batch("bf16", new, ctx, 8, 2, 64, page=16, seed=4)
        table = x.table.clone()
        table[0, 3], table[0, 7], table[1, 0] = -1, x.pages, 2 ** 31 - 1
        keep, x.table = x.table, table
        lost = {0: list(range(48, 64)) + list(range(112, 128)), 1: list(range(16))}
        check(P, R, x, gone=lambda b: lost[b])
        # a table that ends early
        x.table = keep[:, :5].contiguous()
        want = R.attention64(x, 0.125, gone=lambda b: list(range(80, 400)))
        x.attend(P, scale=0.125)
        R.close(x.out, want[0], want[2])
    x = R.Batch("bf16", [2], [30], 8, 2, 64, page=16, seed=4)
    x.table = torch.full_like(x.table, -1)
    x.attend(P)
    assert bool((x.out == 0).all()) and bool((x.lse == -math.inf).all())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_not_finite_where_not_seen(P, R, kind, bad):
    """A NaN or infinity in a token's key or value reaches the tokens that see it, and no others."""
    import torch
    for new, ctx, at, window in (([70], [10], 50, 0), ([8], [300], 305, 0), ([20, 3], [100, 5], 60, 30), ([3], [700], 701, 0)):
        for which in ("k_cache", "v_cache"):
            x = R.Batch(kind, new, ctx, 4, 2, 64, page=16, seed=11)
            page, off = x.where(0, at, at + 1)
            c = getattr(x, which)
            clean = c[page, off].clone()
            want = R.attention64(x, 0.125, window)
            c[page, off, :, 5:9] = bad
            x.attend(P, scale=0.125, window=window)
            torch.cuda.synchronize()
            pos = torch.arange(ctx[0], ctx[0] + new[0], device=DEV)
            sees = (pos >= at) & ((pos - at < window) if window else True)
            rows = torch.zeros(x.n, dtype=torch.bool, device=DEV)
            rows[x.tokens(0)] = sees
            R.close(x.out[~rows], want[0][~rows], want[2][~rows], f"{which} {at}")
            R.close(x.lse[~rows], want[1][~rows], want[3][~rows], f"{which} {at} lse")
            if which == "v_cache":
                assert not bool(torch.isfinite(x.out[rows][..., 5:9]).any())
                R.close(x.out[rows][..., 9:], want[0][rows][..., 9:], want[2][rows][..., 9:], "other columns")
            elif math.isnan(bad):
                assert bool(torch.isnan(x.out[rows]).all())
            c[page, off] = clean


@pytest.mark.parametrize("kind,dim", [("f32", 80), ("f32", 96), ("bf16", 80), ("bf16", 192), ("f32", 192)])
def test_not_finite_in_padded_heads(P, R, kind, dim):
    import torch
    for new, ctx, at, window in (([70], [900], 905, 100), ([300], [400], 500, 64), ([5], [600], 602, 0)):
        x = R.Batch(kind, new, ctx, 4, 2, dim, page=16, seed=12)
        page, off = x.where(0, at, at + 1)
        want = R.attention64(x, 0.125, window)
        x.v_cache[page, off, :, dim - 3:] = math.inf
        x.attend(P, scale=0.125, window=window)
        torch.cuda.synchronize()
        pos = torch.arange(ctx[0], ctx[0] + new[0], device=DEV)
        sees = (pos >= at) & ((pos - at < window) if window else True)
        rows = torch.zeros(x.n, dtype=torch.bool, device=DEV)
        rows[x.tokens(0)] = sees
        R.close(x.out[~rows], want[0][~rows], want[2][~rows], f"{at}")
        R.close(x.out[rows][..., :dim - 3], want[0][rows][..., :dim - 3], want[2][rows][..., :dim - 3], "other columns")
        assert not bool(torch.isfinite(x.out[rows][..., dim - 3:]).any())


def test_infinite_queries_and_large_scores(P, R):
    """A row of NaN queries is NaN, its neighbours are not; scores of thousands keep their differences."""
    import torch
    for new in ([4], [60]):
        x = R.Batch("bf16", new, [100], 4, 2, 64, seed=12)
        want = R.attention64(x, 0.125)
        x.q[1, 2] = math.nan
        x.attend(P, scale=0.125)
        assert bool(torch.isnan(x.out[1, 2]).all())
        x.out[1, 2], x.lse[1, 2] = want[0][1, 2].to(x.out.dtype), want[1][1, 2].float()
        R.close(x.out, want[0], want[2] + (want[0].abs() * 2 ** -8))
    for kind in ("f32", "bf16", "f16"):
        x = R.Batch(kind, [5, 90], [1000, 0], 4, 2, 64, seed=13)
        x.q *= 30
        check(P, R, x, scale=1.0)
    # all of a row's scores equal, far from zero
    x = R.Batch("f16", [3], [500], 2, 1, 32, seed=14)
    x.q.fill_(200.0)
    page, off = x.where(0)
    x.k_cache[page, off] = -100.0
    check(P, R, x, scale=1.0)


def test_strides(P, R):
    """Queries and outputs inside larger tensors, at odd addresses."""
    import torch
    x = R.Batch("bf16", [3, 50], [40, 0], 4, 2, 64, seed=15)
    whole = torch.full((x.n, 11, 67), 77.0, dtype=torch.bfloat16, device=DEV)
    big = torch.zeros(x.n, 9, 71, dtype=torch.bfloat16, device=DEV)
    big[:, 1:5, 3:67] = x.q
    x.q, x.out = big[:, 1:5, 3:67], whole[:, 2:6, 1:65]
    check(P, R, x)
    whole[:, 2:6, 1:65] = 77.0
    assert bool((whole == 77).all())
    # heads outside tokens
    x = R.Batch("f32", [3, 50], [40, 0], 4, 2, 64, seed=16)
    x.q = x.q.transpose(0, 1).contiguous().transpose(0, 1)
    x.out = torch.full((4, x.n, 64), 77.0, device=DEV).transpose(0, 1)
    check(P, R, x)


def test_same_bits_again_and_without_lse(P, R):
    import torch
    for new, ctx in (([1] * 5, [3000, 1, 500, 40, 9000]), ([300, 20], [2000, 100])):
        x = R.Batch("bf16", new, ctx, 8, 2, 128, seed=17)
        x.attend(P)
        first = x.out.clone(), x.lse.clone()
        for _ in range(5):
            x.out.zero_()
            x.attend(P)
            assert torch.equal(x.out, first[0]) and torch.equal(x.lse, first[1])
        x.out.zero_()
        P.at_paged_attention(x.q, x.k_cache, x.v_cache, x.table, x.starts, x.lengths, x.out)
        assert torch.equal(x.out, first[0])


def test_streams_and_a_workspace_of_ones_own(P, R):
    import torch
    x = R.Batch("bf16", [1, 1], [9000, 100], 8, 2, 128, seed=18)
    want = R.attention64(x, x.dim ** -0.5)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    x.attend(P, stream=s)
    s.synchronize()
    R.close(x.out, want[0], want[2])
    need = P.at_paged_attention_workspace(x.n, x.batch, x.table.shape[1] * x.page, 8, 2, 128, P.AT_BF16)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)   # NaN wherever it is read before it is written
    x.out.zero_()
    x.attend(P, workspace=ws)
    torch.cuda.synchronize()
    R.close(x.out, want[0], want[2])
    with pytest.raises(P.ATError):
        x.attend(P, workspace=ws[:-16])


def test_captured_and_replayed(P, R):
    """One captured call serves lengths and tables that change between replays; two graphs share a workspace."""
    import torch
    a = R.Batch("bf16", [1] * 4, [6000, 30, 0, 400], 8, 2, 64, seed=19, extra=50)
    c = R.Batch("bf16", [60], [700], 8, 2, 64, seed=20)
    need = max(P.at_paged_attention_workspace(x.n, x.batch, x.table.shape[1] * x.page, 8, 2, 64, P.AT_BF16) for x in (a, c))
    ws = torch.zeros(max(16, need), dtype=torch.uint8, device=DEV)
    graphs = []
    for x in (a, c):
        x.attend(P, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.attend(P, workspace=ws)
        graphs.append(g)
    for lengths in ([6001, 31, 1, 401], [5000, 31, 1, 2], [1, 1, 1, 1], [6001, 2, 1, 333]):
        a.len = np.asarray(lengths)
        a.lengths.copy_(torch.as_tensor(lengths, dtype=torch.int32))
        for x in (a, c):
            x.out.fill_(3.0)
        graphs[0].replay()
        graphs[1].replay()
        eager = torch.randn(1000, device=DEV).sum()
        torch.cuda.synchronize()
        assert math.isfinite(float(eager))
        for x in (a, c):
            want = R.attention64(x, 0.125)
            R.close(x.out, want[0], want[2], str(lengths))


def test_offsets_past_32_bits(P, R):
    """A cache of more than 2^32 elements, its last pages in use."""
    import torch
    dim, kv, page = 128, 8, 128
    pages = (1 << 32) // (dim * kv * page) + 40
    x = R.Batch("bf16", [1, 20], [300, 70], 8, 8, dim, page=page, seed=21)
    small = x.k_cache, x.v_cache
    x.k_cache, x.v_cache = (torch.empty(pages, page, kv, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for i in range(2):
        (x.k_cache, x.v_cache)[i][pages - len(small[i]):] = small[i]
    x.table += pages - len(small[0])
    x.table_h = x.table_h + pages - len(small[0])
    check(P, R, x)
