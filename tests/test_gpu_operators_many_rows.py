"""Calls of more rows than one launch holds threads for (2^32, at 4 to 256 threads
a row): every row is worked on, those on both sides of a cut among them."""
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


@pytest.fixture(autouse=True)
def memory():
    """The tensors here are large: none stays behind."""
    import torch
    yield
    torch.cuda.empty_cache()


def room(gib):
    import torch
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def rows_to_look_at(n, cuts, count, gen):
    """Rows around every cut, the ends, and some in between."""
    import torch
    near = [c + d for c in cuts for d in (-2, -1, 0, 1)] + [0, 1, n - 2, n - 1]
    some = torch.randint(0, n, (count,), generator=gen)
    return torch.unique(torch.cat([torch.tensor([r for r in near if 0 <= r < n]), some])).to(DEV)


def test_log_probabilities(P):
    """2^26 + 5 rows of three values, a wave each."""
    import torch
    room(8)
    n, vocab, k = (1 << 26) + 5, 3, 2
    print(f"[gpu-rows] log probabilities {n} x {vocab}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(n, vocab, generator=gen, device=DEV)
    tokens = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    valid = torch.randint(1, vocab + 1, (n,), generator=gen, device=DEV, dtype=torch.int32)
    logp, H, lse = (torch.full((n,), 9.0, device=DEV) for _ in range(3))
    top, idx = torch.full((n, k), 9.0, device=DEV), torch.full((n, k), 7, dtype=torch.int32, device=DEV)
    P.at_logprobs(x, tokens, logp, H, lse, top, idx, valid=valid)
    for lo in range(0, n, 1 << 24):     # every row, in 32 bits
        s = slice(lo, lo + (1 << 24))
        z = x[s].masked_fill(torch.arange(vocab, device=DEV) >= valid[s, None], -torch.inf)
        lp = torch.log_softmax(z, 1)
        want = torch.gather(lp, 1, tokens[s, None].long())[:, 0]
        assert torch.allclose(logp[s], want, rtol=1e-5, atol=1e-5)
        assert torch.allclose(lse[s], torch.logsumexp(z, 1), rtol=1e-5, atol=1e-5)
        assert torch.allclose(H[s], -(lp.exp() * lp).nan_to_num().sum(1), rtol=1e-5, atol=1e-5)
        best = z.argmax(1)
        assert torch.equal(idx[s, 0].long(), best)
        assert torch.allclose(top[s, 0], torch.gather(lp, 1, best[:, None])[:, 0], rtol=1e-5, atol=1e-5)
        assert torch.equal(idx[s, 1] < 0, valid[s] < 2)


def test_log_probabilities_gradient(P):
    """2^29 + 37 rows of one value, 32 a workgroup.  They are given an lse of 0, so that p is
    e^x and the gradient g (1 - e^x), or 0 without a token."""
    import torch
    room(24)
    n = (1 << 29) + 37
    print(f"[gpu-rows] gradient {n} x 1", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.empty(n, 1, dtype=torch.float16, device=DEV).uniform_(-2.0, 1.0, generator=gen)
    g = torch.empty(n, device=DEV).uniform_(0.5, 2.0, generator=gen)
    tokens = torch.randint(-1, 1, (n,), generator=gen, device=DEV, dtype=torch.int32)
    lse = torch.zeros(n, device=DEV)
    d = torch.full((n, 1), 9.0, dtype=torch.float16, device=DEV)
    P.at_logprobs_grad(x, tokens, lse, None, g, d)
    for lo in range(0, n, 1 << 26):     # every row; the result's rounding is 2^-11
        s = slice(lo, lo + (1 << 26))
        want = torch.where(tokens[s] >= 0, g[s] * (1.0 - x[s, 0].float().exp()), torch.zeros_like(g[s]))
        assert torch.allclose(d[s, 0].float(), want, rtol=1e-3, atol=1e-5)


def test_log_probabilities_gradient_of_long_rows(P):
    """Rows of several workgroups in more than one launch: 16500 rows of 2^22 + 9 columns, 513
    workgroups each, 2^23 a launch."""
    import torch
    room(150)
    n, vocab = 16500, (1 << 22) + 9
    print(f"[gpu-rows] gradient {n} x {vocab}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(3)
    row = torch.randn(vocab, generator=gen, device=DEV).half()
    x = row.expand(n, vocab)            # one row, n times
    tokens = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    lse = torch.logsumexp(row.float(), 0).expand(n).contiguous()
    g = torch.arange(1, n + 1, device=DEV, dtype=torch.float32) * 2.0
    d = torch.empty(n, vocab, dtype=torch.float16, device=DEV)
    P.at_logprobs_grad(x, tokens, lse, None, g, d)
    p = (row.float() - lse[0]).exp()
    for r in rows_to_look_at(n, [(1 << 23) // 513], 20, torch.Generator().manual_seed(4)).tolist():
        want = -float(g[r]) * p
        want[tokens[r]] += float(g[r])
        assert torch.allclose(d[r].float(), want, rtol=1e-3, atol=2.0 ** -23), r


def test_embed(P):
    """2^26 + 9 rows of 520, a workgroup each with four rows a lane: the calls' last rows are in
    the third launch."""
    import torch
    room(80)
    n, vocab, dim = (1 << 26) + 9, 1000, 520
    print(f"[gpu-rows] lookup {n} x {dim}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(5)
    w = torch.randn(vocab, dim, generator=gen, device=DEV)
    tokens = torch.randint(-1, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    out = torch.full((n, dim), 9.0, dtype=torch.bfloat16, device=DEV)
    P.at_embed(w, tokens, out, scale=0.5)
    rows = rows_to_look_at(n, [k << 25 for k in (1, 2)] + [1 << 24], 4000, torch.Generator().manual_seed(6))
    t = tokens[rows].long()
    want = torch.where((t >= 0)[:, None], w[t.clamp(min=0)] * 0.5, torch.zeros(1, device=DEV)).to(torch.bfloat16)
    assert torch.equal(out[rows], want)
