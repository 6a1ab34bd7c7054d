"""How the serving operators are called: in place, two at once, as captured steps, many
sequences, and what autograd hears of it."""
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


def test_outputs_are_marked_as_written(P, R):
    import torch
    x = R.Batch("bf16", [3, 1], [5, 40], 4, 2, 64, page=16)
    where = (x.k_cache, x.v_cache, x.table, x.starts, x.lengths)
    k, v, freqs = x.randn(4, 2, 64), x.randn(4, 2, 64), torch.ones(32, dtype=torch.float64, device=DEV)
    logits, out = torch.zeros(2, 9, device=DEV), torch.zeros(2, 9, device=DEV)
    past = torch.zeros(2, 3, dtype=torch.int64, device=DEV)
    f = torch.ones(2, device=DEV)

    def bumped(call, outs, ins):
        before = [t._version for t in outs], [t._version for t in ins]
        call()
        assert all(t._version > w for t, w in zip(outs, before[0]))
        assert [t._version for t in ins] == before[1]

    bumped(lambda: P.at_paged_append(k, v, *where, q=x.q, q_out=x.out, freqs=freqs), [x.k_cache, x.v_cache, x.out], [k, v, x.q, x.table])
    bumped(lambda: P.at_paged_append(k, v, *where), [x.k_cache, x.v_cache], [k, v, x.out])
    bumped(lambda: P.at_paged_attention(x.q, *where, x.out, lse=x.lse), [x.out, x.lse], [x.q, x.k_cache, x.v_cache])
    bumped(lambda: P.at_paged_attention(x.q, *where, x.out), [x.out], [x.lse])
    bumped(lambda: P.at_adjust_logits(logits, out, tokens=past, frequency=f), [out], [logits, past, f])


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("bf16", 256), ("f32", 80), ("f16", 40)])
@pytest.mark.parametrize("new,ctx", [([1, 1], [900, 3]), ([200, 40], [0, 700]), ([9], [20])])
def test_queries_in_place(P, R, kind, dim, new, ctx):
    import torch
    for window in (0, 7):
        x = R.Batch(kind, new, ctx, 4, 2, dim, page=16, seed=dim)
        x.attend(P, window=window)
        out, lse = x.out.clone(), x.lse.clone()
        P.at_paged_attention(x.q, x.k_cache, x.v_cache, x.table, x.starts, x.lengths, x.q, lse=x.lse, window=window)
        assert torch.equal(x.q, out) and torch.equal(x.lse, lse)


def test_many_sequences(P, R):
    """More sequences than a wave has lanes, of prompts and of single tokens, with pieces of each."""
    import torch
    for kind, many, new, ctx, heads, dim in (("bf16", 70, 260, 0, 1, 64), ("bf16", 65, 3, 300, 2, 128), ("f32", 90, 1, 700, 2, 64),
                                             ("f32", 66, 40, 500, 1, 100)):
        print(f"[gpu-serving] {kind} {many} x {new}", flush=True)
        x = R.Batch(kind, [new] * many, np.random.default_rng(0).integers(0, ctx + 1, many), heads, 1, dim, page=16, seed=many)
        for window in (0, 150):
            want = R.attention64(x, 0.125, window)
            x.attend(P, scale=0.125, window=window)
            torch.cuda.synchronize()
            R.close(x.lse, want[1], want[3], "lse")
            R.close(x.out, want[0], want[2], "out")


def test_two_at_once(P, R):
    """Calls on two streams, each with pieces in a workspace of its own."""
    import torch
    xs = [R.Batch("bf16", [1], [ctx], 8, 2, 128, page=16, seed=ctx) for ctx in (9000, 7000)]
    want = []
    for x in xs:
        x.attend(P)
        want.append((x.out.clone(), x.lse.clone()))
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, s in zip(xs, streams):
            x.attend(P, stream=s)
    torch.cuda.synchronize()
    for x, (out, lse) in zip(xs, want):
        assert torch.equal(x.out, out) and torch.equal(x.lse, lse)


def test_captured_steps(P, R):
    """A step of append, attention and changes to logits, captured once and replayed as sequences grow, beside eager calls."""
    import torch
    B, H, K, D, V, size = 5, 8, 2, 64, 300, 16
    gen = torch.Generator(device=DEV).manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()  # noqa: E731
    table = torch.randperm(B * 8, generator=gen, device=DEV).int().reshape(B, 8)
    starts = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    freqs = torch.logspace(0, -3, D // 2, dtype=torch.float64, device=DEV)
    weight = rand(H * D, V)
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (1, (V + 31) // 32), generator=gen, device=DEV).int()
    rows = torch.zeros(B, dtype=torch.int32, device=DEV)
    penalty = torch.full((B,), 1.5, device=DEV)

    class State:
        def __init__(self):
            self.k_cache, self.v_cache = (torch.zeros(B * 8, size, K, D, device=DEV, dtype=torch.bfloat16) for _ in range(2))
            self.lengths = torch.zeros(B, dtype=torch.int32, device=DEV)
            self.past = torch.full((B, 128), -1, dtype=torch.int64, device=DEV)
            self.qkv = torch.zeros(B, H + 2 * K, D, device=DEV, dtype=torch.bfloat16)
            self.out = torch.zeros(B, H, D, device=DEV, dtype=torch.bfloat16)
            self.logits = torch.zeros(B, V, device=DEV)

        def step(self):
            q, k, v = self.qkv.split([H, K, K], 1)
            where = (self.k_cache, self.v_cache, table, starts, self.lengths)
            P.at_paged_append(k, v, *where, q=q, q_out=self.out, freqs=freqs)
            P.at_paged_attention(self.out, *where, self.out)
            torch.matmul(self.out.reshape(B, H * D).float(), weight.float(), out=self.logits)
            P.at_adjust_logits(self.logits, self.logits, tokens=self.past, lengths=self.lengths, repetition=penalty, mask=mask, mask_rows=rows)

    eager, captured = State(), State()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for c in (captured.k_cache, captured.v_cache):
        c.zero_()
    for n in range(120):
        qkv = rand(B, H + 2 * K, D)
        for s in (eager, captured):
            s.qkv.copy_(qkv)
            s.lengths.add_(1)
        eager.step()
        graph.replay()
        assert torch.equal(eager.logits, captured.logits) and torch.equal(eager.out, captured.out), n
        assert bool(torch.isfinite(eager.logits).any(1).all()) and bool((eager.logits == -math.inf).any())
        token = eager.logits.argmax(1)
        for s in (eager, captured):
            s.past[:, n] = token
    assert torch.equal(eager.k_cache, captured.k_cache) and torch.equal(eager.v_cache, captured.v_cache)


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("new,ctx,fewer", [([5, 1], [30, 900], 1), ([9], [40], 4), ([200, 90], [50, 700], 33), ([300, 1, 1], [0, 20, 5000], 150),
                                           ([40], [6000], 25)])
def test_fewer_tokens_than_starts_name(P, R, kind, dim, new, ctx, fewer):
    """Buffers that end before the last sequence's new tokens do: tokens keep their positions, in the cache and in what they see."""
    import torch
    for window in (0, 20):
        x = R.Batch(kind, new, ctx, 4, 2, dim, page=16, seed=fewer)
        want = R.attention64(x, 0.125, window)
        n, keep = x.n - fewer, (x.k_cache.clone(), x.v_cache.clone())
        places = [x.where(b, int(x.len[b] - x.new[b])) for b in range(x.batch)]
        page, off = (torch.cat(p) for p in zip(*places))
        k, v = (c[page, off] for c in keep)
        for c in (x.k_cache, x.v_cache):
            c[page, off] = math.nan
        where = (x.k_cache, x.v_cache, x.table, x.starts, x.lengths)
        P.at_paged_append(k[:n], v[:n], *where)
        for c, whole in zip((x.k_cache, x.v_cache), keep):
            assert torch.equal(c[page, off][:n], whole[page, off][:n]) and bool(torch.isnan(c[page, off][n:]).all())
        P.at_paged_attention(x.q[:n], *where, x.out[:n], scale=0.125, window=window, lse=x.lse[:n])
        torch.cuda.synchronize()
        R.close(x.out[:n], want[0][:n], want[2][:n], "out")
        R.close(x.lse[:n], want[1][:n], want[3][:n], "lse")
        assert bool((x.out[n:] == 77).all()) and bool((x.lse[n:] == 77).all())


def test_more_workgroups_than_a_launch_holds(P):
    """2^32 threads and more, by 65535 heads of 257 sequences: each token sees one key, whose value it gets."""
    import torch
    B, H, D = 257, 65535, 8
    gen = torch.Generator(device=DEV).manual_seed(0)
    k_cache, v_cache, q = (torch.randn(B, H, D, generator=gen, device=DEV).bfloat16() for _ in range(3))
    table = torch.randperm(B, generator=gen, device=DEV).int()[:, None].contiguous()
    starts = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    lengths = torch.ones(B, dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q, 77.0), torch.full((B, H), 77.0, device=DEV)
    P.at_paged_attention(q, k_cache[:, None], v_cache[:, None], table, starts, lengths, out, scale=1.0, lse=lse)
    torch.cuda.synchronize()
    page = table[:, 0].long()
    assert torch.equal(out, v_cache[page])
    products = q.float() * k_cache[page].float()   # exact
    # sums of eight products, and the maximum's scaling, in fp32
    assert bool(((lse - products.double().sum(2)).abs() <= 2.0 ** -24 * (12 * products.abs().sum(2) + 4)).all())


def test_size_one_axes_have_any_stride(P, R):
    """One token in place whose output has another distance between tokens; one head, page or place at odd distances."""
    import torch
    for dim in (64, 192):
        x = R.Batch("bf16", [1], [15], 4, 1, dim, page=16, seed=dim)
        want = R.attention64(x, 0.125)
        big = torch.zeros(4 * dim + 8, dtype=torch.bfloat16, device=DEV)
        q, out = big.as_strided((1, 4, dim), (4 * dim, dim, 1)), big.as_strided((1, 4, dim), (4 * dim + 3, dim, 1))
        q.copy_(x.q)
        odd = [c.as_strided((x.pages, 16, 1, dim), (16 * dim, dim, 7, 1)) for c in (x.k_cache, x.v_cache)]
        P.at_paged_attention(q, *odd, x.table, x.starts, x.lengths, out, scale=0.125, lse=x.lse)
        R.close(out, want[0], want[2], "out")
        k, v = x.randn(1, 1, dim), x.randn(1, 1, dim)
        freqs = torch.linspace(1, 0.01, dim // 2, dtype=torch.float64, device=DEV)
        q.copy_(x.q)
        for q_, o_ in ((x.q, x.out), (q, out)):
            P.at_paged_append(k, v, *odd, x.table, x.starts, x.lengths, q=q_, q_out=o_, freqs=freqs)
        assert torch.equal(out, x.out)


def test_a_quarter_of_a_million_sequences(P):
    """The time of a call goes with the number of its sequences, not with the square, which would be a second here; some have no new
    token, and some two."""
    import torch
    B, H, D = 1 << 18, 2, 16
    gen = torch.Generator(device=DEV).manual_seed(0)
    new = torch.randint(0, 3, (B,), generator=gen, device=DEV)
    starts = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int64), new.cumsum(0)]).int()
    n = int(starts[-1])
    k_cache, v_cache = (torch.randn(B, 2, H, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    table = torch.randperm(B, generator=gen, device=DEV).int()[:, None].contiguous()
    q = torch.randn(n, H, D, generator=gen, device=DEV).bfloat16()
    out, lse = torch.full_like(q, 77.0), torch.full((n, H), 77.0, device=DEV)
    call = lambda: P.at_paged_attention(q, k_cache, v_cache, table, starts, new.int(), out, scale=0.25, lse=lse)  # noqa: E731
    call()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    call()
    end.record()
    torch.cuda.synchronize()
    b = torch.repeat_interleave(torch.arange(B, device=DEV), new)
    page, second = table[b, 0].long(), (torch.arange(n, device=DEV) > starts[b])[:, None, None]
    k, v = k_cache[page].double(), v_cache[page].double()                       # [n, 2, H, D]
    s = 0.25 * (q.double()[:, None] * k).sum(3)
    size = 0.25 * (q.double()[:, None] * k).abs().sum(3).amax(1)
    s[:, 1] = torch.where(second[..., 0], s[:, 1], torch.full_like(s[:, 1], -math.inf))
    want_lse = torch.logsumexp(s, 1)
    p = torch.exp(s - want_lse[:, None])[..., None]
    want, big, u = (p * v).sum(1), (p * v.abs()).sum(1), 2.0 ** -24
    # scores of 16 products, twice in a weight, whose rounding to bf16 is 2^-8 and the result's again
    assert bool(((out.double() - want).abs() <= big * (48 * u * size[..., None] + 40 * u + 2.0 ** -8) + want.abs() * 2.0 ** -8 * (1 + 2 ** -6)).all())
    assert bool(((lse.double() - want_lse).abs() <= 24 * u * size + 20 * u + 4 * u * want_lse.abs()).all())
    took = begin.elapsed_time(end)
    print(f"[gpu-serving] {took:.2f} ms", flush=True)
    assert took < 100.0
