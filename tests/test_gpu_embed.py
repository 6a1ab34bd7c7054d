"""Embedding lookup and its gradient on the GPU.

The lookup is one product and one rounding, so it is compared bit for bit
with the same two operations on the CPU.  The gradient is compared with the
sum in 64 bits: c terms added in fp32 in any order are within c 2^-24 sum|x|,
the product with scale and the rounding to the output's type add one rounding
each."""
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(msg):
    print(f"[gpu-embed] {msg}", flush=True)


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def rows(shape, dtype, pad, gen):
    """A [n, d] tensor whose rows lie pad elements further apart than d, inside
    a larger buffer of a recognisable value."""
    import torch
    n, d = shape
    buf = torch.full((n, d + pad), 77.0, dtype=dtype)
    buf[:, :d] = torch.randn(n, d, generator=gen).to(dtype)
    return buf.to(DEV)[:, :d]


def make_tokens(kind, n, vocab, gen, wide):
    import torch
    if kind == "one":
        t = torch.full((n,), vocab - 1)
    elif kind == "none":
        t = torch.full((n,), -1)
    elif kind == "frequent":
        t = (torch.rand(n, generator=gen) ** 6 * vocab).long()
    elif kind == "ascending":
        t = torch.arange(n) % vocab
    else:
        t = torch.randint(0, vocab, (n,), generator=gen)
    if kind == "outside":   # padding and out-of-range tokens among the others
        t[::3] = -1
        t[1::5] = vocab
        t[2::7] = 2 ** 31 - 1
    return t.to(torch.int64 if wide else torch.int32)


@pytest.mark.parametrize("n,vocab,dim,wt,ot,pad,kind,wide", [
    (1, 1, 1, "f32", "f32", 0, "flat", True),
    (1, 5, 128, "bf16", "bf16", 0, "flat", False),
    (7, 33, 8, "f16", "f32", 0, "outside", True),
    (64, 455, 128, "f32", "bf16", 0, "flat", True),
    (100, 19, 129, "bf16", "bf16", 3, "outside", False),
    (333, 1000, 1000, "f16", "f16", 1, "flat", True),
    (50, 10, 2047, "bf16", "f32", 0, "frequent", True),
    (17, 100, 4099, "f32", "f32", 5, "flat", False),
    (20000, 300, 64, "bf16", "bf16", 0, "outside", True),
    (9000, 5000, 33, "f32", "f16", 0, "flat", False),
    (5, 3, 16, "f32", "f32", 0, "none", True),
])
def test_lookup(P, n, vocab, dim, wt, ot, pad, kind, wide):
    import torch
    say(f"lookup {n} of {vocab} x {dim} {wt} -> {ot} pad {pad} {kind}")
    gen = torch.Generator().manual_seed(n * 7 + dim)
    T = types()
    w = rows((vocab, dim), T[wt], pad, gen)
    t = make_tokens(kind, n, vocab, gen, wide)
    out = torch.full((n, dim + pad), 5.0, dtype=T[ot], device=DEV)
    scale = 11.3125 if wt != "f16" else 1.5
    P.at_embed(w, t.to(DEV), out[:, :dim], scale=scale)
    real = (t >= 0) & (t < vocab)
    want = torch.where(real[:, None], w.cpu()[t.long().clamp(0, vocab - 1)].float() * scale, torch.zeros(())).to(T[ot])
    got = out.cpu()
    assert torch.equal(got[:, :dim], want)
    assert bool((got[:, dim:] == 5.0).all()), "wrote past a row"


def reference(dout, t, vocab, scale, before):
    """(sum in 64 bits, sum of magnitudes, terms a row)."""
    import torch
    keep = torch.nonzero((t >= 0) & (t < vocab))[:, 0]
    d, k = dout.cpu().double()[keep], t.long()[keep]
    z = torch.zeros(vocab, dout.shape[1], dtype=torch.float64)
    total, size = z.clone().index_add_(0, k, d) * scale, z.clone().index_add_(0, k, d.abs()) * abs(scale)
    count = torch.bincount(k, minlength=vocab)
    if before is not None:
        total = total + before.cpu().double()
        size = size + before.cpu().double().abs()
    return total, size, count


@pytest.mark.parametrize("n,vocab,dim,dt,gt,pad,kind,wide,add", [
    (1, 1, 1, "f32", "f32", 0, "flat", True, False),
    (0, 9, 20, "bf16", "f32", 0, "flat", True, False),
    (1, 1000, 128, "bf16", "bf16", 0, "flat", False, False),
    (448, 455, 128, "f32", "f32", 0, "flat", True, False),
    (448, 455, 128, "f32", "f32", 0, "flat", True, True),
    (2049, 3001, 1000, "f32", "f32", 0, "frequent", False, True),
    (1000, 7, 129, "bf16", "f32", 3, "outside", True, False),
    (3000, 50, 40, "f16", "f16", 0, "frequent", True, False),
    (500, 600, 2050, "bf16", "bf16", 2, "outside", True, True),
    (8192, 1, 64, "bf16", "f32", 0, "one", True, False),
    (8193, 4097, 24, "f32", "f32", 0, "flat", False, False),
    (60000, 33, 8, "bf16", "f32", 0, "flat", True, False),
    (60000, 100, 65, "f16", "f32", 0, "one", False, False),
    (50000, 70000, 16, "bf16", "f32", 0, "frequent", True, False),
    (30000, 300000, 12, "f32", "f32", 0, "flat", False, False),
    (20000, 20000, 100, "bf16", "f32", 0, "ascending", True, False),
    (12000, 64, 200, "f32", "bf16", 0, "none", True, False),
    (12000, 64, 200, "f32", "bf16", 0, "none", True, True),
    (300, 20, 9001, "f32", "f32", 1, "flat", True, False),
    # more entries than a tile each; rows over many workgroups; narrow rows
    (100000, 3000, 40, "bf16", "f32", 0, "outside", True, False),
    (150000, 2, 24, "f16", "f32", 1, "flat", False, True),
    (70000, 70001, 3, "f32", "f32", 0, "frequent", True, False),
    (5000, 40, 7, "bf16", "bf16", 0, "outside", False, True),
    (900, 5, 17, "f16", "bf16", 0, "one", True, True),
])
def test_gradient(P, n, vocab, dim, dt, gt, pad, kind, wide, add):
    import torch
    say(f"gradient {n} of {vocab} x {dim} {dt} -> {gt} {kind} add {add}")
    gen = torch.Generator().manual_seed(n * 3 + dim)
    T = types()
    d = rows((n, dim), T[dt], pad, gen)
    t = make_tokens(kind, n, vocab, gen, wide)
    buf = torch.full((vocab, dim + pad), 5.0, dtype=T[gt], device=DEV)
    before = None
    if add:
        before = torch.randn(vocab, dim, generator=gen).to(T[gt])
        buf[:, :dim] = before.to(DEV)
    P.at_embed_grad(d, t.to(DEV), buf[:, :dim], scale=0.75, accumulate=add)
    got = buf.cpu()
    assert bool((got[:, dim:] == 5.0).all()), "wrote past a row"
    total, size, count = reference(d, t, vocab, 0.75, before)
    tol = (count[:, None] + 3) * 2.0 ** -24 * size + ROUND[gt] * total.abs() + (2.0 ** -24 if gt == "f16" else 0.0)
    err = (got[:, :dim].double() - total).abs()
    assert bool((err <= tol).all()), f"largest excess {float((err - tol).max())}"
    if add:   # rows that no token names keep their bits
        assert torch.equal(got[count == 0][:, :dim], before[count == 0])
    else:
        assert bool((got[count == 0][:, :dim] == 0).all())


@pytest.mark.parametrize("n,vocab,dim,dt,gt,kind,wide,add", [
    # one workgroup's sort, a few entries a thread, tiles
    (1024, 1023, 16, "f32", "f32", "flat", True, False),
    (1025, 1024, 16, "bf16", "f32", "outside", False, False),
    (4096, 2000, 8, "f32", "f32", "frequent", True, False),
    (4097, 2000, 8, "f32", "f32", "frequent", False, True),
    (4097, 1, 8, "f32", "f32", "outside", True, False),
    # one and four entries a thread
    (131072, 1100000, 4, "f32", "f32", "flat", False, False),
    (131073, 70000, 8, "bf16", "f32", "outside", True, False),
    # the most tiles that scan for themselves, and a launch that scans
    (192 * 4096, 1024, 8, "bf16", "f32", "flat", False, False),
    (192 * 4096 + 1, 1023, 8, "bf16", "f32", "outside", True, True),
    (1100000, 3, 8, "bf16", "f32", "outside", False, False),
])
def test_gradient_sort_sizes(P, n, vocab, dim, dt, gt, kind, wide, add):
    """Where the sort changes its launches: numbers of entries, and of bits."""
    test_gradient(P, n, vocab, dim, dt, gt, 0, kind, wide, add)


def test_gradient_is_reproducible(P):
    """The same call gives the same bits, with a given workspace that holds
    another call's leftovers, on another stream, and within a batch of calls."""
    import torch
    gen = torch.Generator().manual_seed(5)
    n, vocab, dim = 40000, 500, 96
    d = torch.randn(n, dim, generator=gen).to(DEV)
    t = make_tokens("frequent", n, vocab, gen, True).to(DEV)
    outs = [torch.empty(vocab, dim, device=DEV) for _ in range(3)]
    P.at_embed_grad(d, t, outs[0])
    ws = torch.full((P.at_embed_grad_workspace(n, vocab, dim),), 0xAB, dtype=torch.uint8, device=DEV)
    P.at_embed_grad(d, t, outs[1], workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    P.at_embed_grad(d, t, outs[2], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_gradient_of_a_broadcast_row(P):
    """A gradient that is one row for every token (distance 0 between rows)."""
    import torch
    row = torch.arange(1, 41, dtype=torch.float32, device=DEV)[None]
    t = torch.tensor([2, 0, 2, 2, -1], device=DEV)
    out = torch.empty(4, 40, device=DEV)
    P.at_embed_grad(row.expand(5, 40), t, out)
    want = torch.tensor([1.0, 0.0, 3.0, 0.0], device=DEV)[:, None] * row
    assert torch.equal(out, want)


def far_rows(shape, dtype, apart, gen):
    """A [n, d] tensor whose rows lie apart elements from one another."""
    import torch
    n, d = shape
    buf = torch.empty((n - 1) * apart + d, dtype=dtype, device=DEV)
    x = torch.as_strided(buf, (n, d), (apart, 1))
    x.copy_(torch.randn(n, d, generator=gen).to(dtype).to(DEV))
    return x


def test_rows_past_32_bits(P):
    """Tables, gradients and outputs whose last rows start past 2^31 elements."""
    import torch
    gen = torch.Generator().manual_seed(9)
    apart = (1 << 30) + 8
    t = torch.tensor([2, 0, 2, 3, 1, 2], device=DEV)
    w = far_rows((3, 100), torch.bfloat16, apart, gen)
    out = far_rows((6, 100), torch.bfloat16, 1 << 29, gen)
    P.at_embed(w, t, out, scale=1.5)
    want = torch.empty(6, 100, dtype=torch.bfloat16, device=DEV)
    P.at_embed(w.contiguous(), t, want, scale=1.5)
    assert torch.equal(out, want)
    for add in (False, True):
        before = w.contiguous()
        P.at_embed_grad(out, t, w, accumulate=add)
        P.at_embed_grad(out.contiguous(), t, before, accumulate=add)
        assert torch.equal(w, before)


def test_tokens_past_32_bits(P):
    """64-bit tokens whose low words are in range are not."""
    import torch
    gen = torch.Generator().manual_seed(10)
    w = torch.randn(5, 40, generator=gen).to(DEV)
    t = torch.tensor([1, (1 << 32) + 1, -(1 << 32) + 2, (1 << 63) - 1, 4, -(1 << 63)], device=DEV)
    out = torch.full((6, 40), 3.0, device=DEV)
    P.at_embed(w, t, out)
    want = torch.zeros_like(out)
    want[0], want[4] = w[1], w[4]
    assert torch.equal(out, want)
    dw = torch.full_like(w, 3.0)
    P.at_embed_grad(torch.ones_like(out), t, dw)
    want = torch.zeros_like(w)
    want[1] = want[4] = 1.0
    assert torch.equal(dw, want)


def test_gradient_against_differences(P):
    """The lookup is linear in the table: <dout, embed(W + E) - embed(W)> is
    <gradient, E> for any E, exactly in exact arithmetic.  Whole numbers and
    a power-of-two scale make it exact in fp32 too."""
    import torch
    gen = torch.Generator().manual_seed(9)
    n, vocab, dim = 700, 90, 48
    ints = lambda *s: torch.randint(-8, 9, s, generator=gen).float()  # noqa: E731
    w, e, d = ints(vocab, dim), ints(vocab, dim), ints(n, dim)
    t = make_tokens("outside", n, vocab, gen, True).to(DEV)
    a, b = torch.empty(n, dim, device=DEV), torch.empty(n, dim, device=DEV)
    P.at_embed(w.to(DEV), t, a, scale=0.5)
    P.at_embed((w + e).to(DEV), t, b, scale=0.5)
    g = torch.empty(vocab, dim, device=DEV)
    P.at_embed_grad(d.to(DEV), t, g, scale=0.5)
    assert float(((b - a).cpu().double() * d.double()).sum()) == float((g.cpu().double() * e.double()).sum())


def test_infinities_and_nan_stay_in_their_rows(P):
    import torch
    w = torch.zeros(4, 16)
    w[1], w[2] = float("inf"), float("nan")
    t = torch.tensor([0, 1, 2, -1], device=DEV)
    out = torch.empty(4, 16, device=DEV)
    P.at_embed(w.to(DEV), t, out, scale=2.0)
    out = out.cpu()
    assert bool((out[0] == 0).all()) and bool(torch.isinf(out[1]).all()) and bool(torch.isnan(out[2]).all())
    assert bool((out[3] == 0).all())
    d = torch.ones(3, 16)
    d[1] = float("nan")     # its token is dropped
    g = torch.empty(4, 16, device=DEV)
    P.at_embed_grad(d.to(DEV), torch.tensor([0, -1, 3], device=DEV), g)
    assert torch.equal(g.cpu(), torch.tensor([1.0, 0, 0, 1.0])[:, None].expand(4, 16))


def test_graph_replays(P):
    """Both calls inside a captured graph, replayed with other inputs between."""
    import torch
    gen = torch.Generator().manual_seed(2)
    n, vocab, dim = 10000, 800, 72
    w, d = torch.randn(vocab, dim, generator=gen).to(DEV), torch.randn(n, dim, generator=gen).to(DEV)
    t = make_tokens("outside", n, vocab, gen, True).to(DEV)
    out, g = torch.empty(n, dim, device=DEV), torch.empty(vocab, dim, device=DEV)
    ws = torch.empty(P.at_embed_grad_workspace(n, vocab, dim), dtype=torch.uint8, device=DEV)
    P.at_embed(w, t, out)
    P.at_embed_grad(d, t, g, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.at_embed(w, t, out)
        P.at_embed_grad(d, t, g, workspace=ws)
    for k in range(4):
        t.copy_(make_tokens("frequent" if k % 2 else "flat", n, vocab, gen, True))
        want_out, want_g = torch.empty_like(out), torch.empty_like(g)
        P.at_embed(w, t, want_out)
        P.at_embed_grad(d, t, want_g)
        out.fill_(1.0)
        g.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_out) and torch.equal(g, want_g), k
