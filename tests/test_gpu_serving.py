"""The serving operators together, as a program that proposes configurations calls them: a small causal
model of knob tokens, served from a paged cache token by token, against the same model computed whole in 64 bits."""
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


class Model:
    """One layer: token vectors, grouped attention with rotated normed heads, one product to the logits."""

    def __init__(self, vocab=200, width=64, heads=4, kv=2, dim=32, seed=0):
        import torch
        gen = torch.Generator().manual_seed(seed)
        new = lambda *s: (torch.randn(*s, generator=gen) / math.sqrt(s[-1])).to(DEV)  # noqa: E731
        self.vocab, self.heads, self.kv, self.dim = vocab, heads, kv, dim
        self.table, self.qkv, self.out = new(vocab, width), new((heads + 2 * kv) * dim, width), new(vocab, heads * dim) * 4
        self.weight = 1 + new(dim)
        self.freqs = 100.0 ** (-torch.arange(0, dim, 2, device=DEV, dtype=torch.float64) / dim)

    def whole(self, tokens, past, rep, allowed):
        """Log probabilities of every allowed next token after the sequence, in 64 bits."""
        import torch
        H, K, D = self.heads, self.kv, self.dim
        x = self.table.double()[tokens] * 8.0
        y = (x @ self.qkv.double().T).view(len(tokens), H + 2 * K, D)

        def turned(h):
            h = h / torch.sqrt(h.square().mean(2, keepdim=True) + 1e-6) * self.weight.double()
            t = torch.arange(len(tokens), device=DEV).double()[:, None, None] * self.freqs
            a, b = h[..., : D // 2], h[..., D // 2:]
            return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()], 2)

        q, k, v = turned(y[:, :H]), turned(y[:, H: H + K]), y[:, H + K:]
        o = []
        for h in range(H):
            s = (k[:, h // (H // K)] @ q[-1, h]) / math.sqrt(D)
            o.append(torch.softmax(s, 0) @ v[:, h // (H // K)])
        x = self.out.double() @ torch.cat(o)
        seen = torch.zeros(self.vocab, dtype=torch.bool, device=DEV)
        seen[past] = True
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        return torch.log_softmax(x.masked_fill(~allowed, -math.inf), 0)


def test_a_model_served_token_by_token(P):
    import torch
    m, B, page, width = Model(), 3, 4, 12
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, m.vocab, n).tolist() for n in (9, 1, 17)]
    caches = [torch.full((B * width + 1, page, m.kv, m.dim), math.nan, device=DEV) for _ in range(2)]
    table = torch.as_tensor(rng.permutation(B * width).reshape(B, width).astype(np.int32), device=DEV)
    allowed = torch.as_tensor(rng.random((2, m.vocab)) < 0.5, device=DEV)
    allowed[:, :3] = True
    words = np.packbits(np.pad(allowed.cpu().numpy(), ((0, 0), (0, -m.vocab % 32))), axis=1, bitorder="little").view(np.int32)
    mask = torch.as_tensor(words.copy(), device=DEV)
    rows = torch.tensor([0, 1, -1], dtype=torch.int32, device=DEV)
    rep = torch.tensor([1.3, 1.0, 2.0], device=DEV)
    history = torch.zeros(B, 40, dtype=torch.int64, device=DEV)
    said = [list(p) for p in prompts]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731

    def step(new):
        """One pass over the new tokens of each sequence: the log probabilities and likeliest tokens after them."""
        starts = ints([0] + np.cumsum([len(t) for t in new]).tolist())
        lengths = ints([len(s) for s in said])
        tokens = torch.tensor([t for s in new for t in s], device=DEV)
        n = len(tokens)
        x = torch.empty(n, m.table.shape[1], device=DEV)
        P.at_embed(m.table, tokens, x, scale=8.0)
        qkv = (x @ m.qkv.T).view(n, m.heads + 2 * m.kv, m.dim)
        q, k, v = qkv[:, : m.heads], qkv[:, m.heads: m.heads + m.kv], qkv[:, m.heads + m.kv:]
        P.at_paged_append(k, v, *caches, table, starts, lengths, q=q, q_out=q, freqs=m.freqs, k_weight=m.weight, q_weight=m.weight)
        o = torch.empty(n, m.heads, m.dim, device=DEV)
        P.at_paged_attention(q, *caches, table, starts, lengths, o)
        logits = o.view(n, -1)[starts[1:].long() - 1] @ m.out.T
        for b, s in enumerate(said):
            history[b, : len(s)] = torch.tensor(s, device=DEV)
        P.at_adjust_logits(logits, logits, tokens=history, lengths=lengths, repetition=rep, mask=mask, mask_rows=rows)
        best, index = torch.empty(B, 5, device=DEV), torch.empty(B, 5, dtype=torch.int32, device=DEV)
        lse = torch.empty(B, device=DEV)
        P.at_logprobs(logits, lse=lse, top_logp=best, top_idx=index)
        return logits - lse[:, None], best, index

    new = prompts
    for _ in range(20):
        got, best, index = step(new)
        for b in range(B):
            ok = allowed[int(rows[b])] if int(rows[b]) >= 0 else torch.ones(m.vocab, dtype=torch.bool, device=DEV)
            want = m.whole(torch.tensor(said[b], device=DEV), torch.tensor(said[b], device=DEV), float(rep[b]), ok)
            # fp32 products of 64 and 128 terms, logits of up to about 20: 2^-24 * 128 * 20 with room for their sums
            assert bool((torch.isfinite(got[b]) == ok).all())
            off = (got[b].double() - want)[ok].abs()
            assert float(off.max()) < 2.0 ** -24 * 128 * 64, float(off.max())
            top = int(index[b, 0])
            assert float(want[top]) >= float(want.max()) - 1e-3 and abs(float(best[b, 0]) - float(want[top])) < 1e-3
        new = [[int(index[b, rng.integers(0, 5)])] for b in range(B)]
        for b in range(B):
            said[b] += new[b]
