"""Batches over a paged cache, and the serving operators in plain 64-bit form, for tests.

Places of a cache that no sequence uses hold NaN, so that a read of one shows."""
import math

import numpy as np
import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def step(kind):
    """Half a step of a type, relative: what rounding to it is off by at most."""
    return torch.finfo(TYPES[kind]).eps / 2


class Batch:
    """new[b] new tokens of sequences that have ctx[b] positions already, in pages that lie anywhere."""

    def __init__(self, kind, new, ctx, heads, kv, dim, page=16, seed=0, behind=0, spread="tokens", extra=0, fill=True):
        rng = np.random.default_rng(seed)
        self.kind, self.kv, self.heads, self.dim, self.page = kind, kv, heads, dim, page
        self.new, self.len = np.asarray(new), np.asarray(new) + np.asarray(ctx)
        self.batch = len(self.new)
        starts = np.concatenate([[0], np.cumsum(self.new)])
        need = -(-self.len // page)
        self.pages, width = int(need.sum()) + 2 + extra, max(1, int(need.max(initial=0)))
        table = np.full((self.batch, width), -7, np.int64)
        table[np.arange(width)[None] < need[:, None]] = rng.permutation(self.pages)[: int(need.sum())]
        self.starts_h, self.table_h = starts, table
        put = lambda a: torch.as_tensor(a.astype(np.int32), device=DEV)  # noqa: E731
        self.starts, self.lengths, self.table = put(starts), put(self.len), put(table)
        self.n = int(starts[-1]) + behind
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.randn = lambda *sh: torch.randn(*sh, generator=gen, device=DEV).to(TYPES[kind])  # noqa: E731
        self.k_cache, self.v_cache = (self.cache(spread) for _ in range(2))
        if fill:
            for b in range(self.batch):
                for c in (self.k_cache, self.v_cache):
                    page_, off = self.where(b)
                    c[page_, off] = self.randn(len(page_), kv, dim)
        self.q = self.randn(self.n, heads, dim)
        self.out = torch.full((self.n, heads, dim), 77.0, device=DEV, dtype=TYPES[kind])
        self.lse = torch.full((self.n, heads), 77.0, device=DEV)

    def cache(self, spread):
        """[pages, page, kv, dim], heads inside places, or places inside heads, or with odd distances between all of them."""
        P, S, K, D, T = self.pages, self.page, self.kv, self.dim, TYPES[self.kind]
        if spread == "heads":
            return torch.full((P, K, S, D), math.nan, dtype=T, device=DEV).transpose(1, 2)
        if spread == "odd":
            return torch.full((P, S * (K * (D + 1) + 3) + 5), math.nan, dtype=T, device=DEV).as_strided(
                (P, S, K, D), (S * (K * (D + 1) + 3) + 5, K * (D + 1) + 3, D + 1, 1), 1)
        return torch.full((P, S, K, D), math.nan, dtype=T, device=DEV)

    def where(self, b, lo=0, hi=None):
        p = np.arange(lo, self.len[b] if hi is None else hi)
        return (torch.as_tensor(self.table_h[b, p // self.page], device=DEV), torch.as_tensor(p % self.page, device=DEV))

    def tokens(self, b):
        return slice(int(self.starts_h[b]), int(self.starts_h[b + 1]))

    def attend(self, P, **kw):
        P.at_paged_attention(self.q, self.k_cache, self.v_cache, self.table, self.starts, self.lengths, self.out, lse=self.lse, **kw)


def attention64(x, scale, window=0, gone=None):
    """(out, lse, tolerance of out, tolerance of lse) of a Batch in 64 bits; gone(b): positions that are not there.

    Tolerances, with u = 2^-24, A = sum p |v| and S the largest sum |q_d k_d| scale of a row:
      scores   off by (D + 4) u S, in their products and sums, and 4 u S in their scaling and the maximum's;
      weights  off by twice that relative, 4 u in 2^x, and half a step where they are rounded to the type (fp16: the largest
               is kept at 2^11 or more, and half a subnormal step, 2^-25, is 2^-36 of that);
      sums     over L keys, of weights and of weighted values: 2 (L + 8) u;
      joining  pieces: 8 u;  the result: half a step of the type, of its subnormals for fp16 2^-25.
    """
    u = 2.0 ** -24
    D, G, kind = x.dim, x.heads // x.kv, x.kind
    out, lse = x.out.double().clone(), x.lse.double().clone()
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(x.batch):
        t, L, m = x.tokens(b), int(x.len[b]), int(x.new[b])
        if m == 0:
            continue
        page, off = x.where(b)
        k, v = (c[page, off].double().repeat_interleave(G, 1).transpose(0, 1).contiguous() for c in (x.k_cache, x.v_cache))
        q = x.q[t].double().transpose(0, 1).contiguous()                       # [heads, m, D]
        pos = torch.arange(L - m, L, device=DEV)[:, None]
        j = torch.arange(L, device=DEV)[None]
        seen = j <= pos
        if window:
            seen = seen & (j > pos - window)
        if gone is not None and len(gone(b)):
            seen = seen & ~torch.isin(j, torch.as_tensor(gone(b), device=DEV))
        s = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
        big = torch.bmm(q.abs(), k.abs().transpose(1, 2).contiguous()) * scale
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        big = torch.where(seen, big, torch.zeros_like(big))
        S = big.amax(2, keepdim=True) if L else torch.zeros(x.heads, m, 1, device=DEV, dtype=torch.float64)
        l = torch.logsumexp(s, 2, keepdim=True)
        p = torch.where(seen, torch.exp(s - l), torch.zeros_like(s))
        out[t] = torch.bmm(p, torch.where(torch.isnan(v), torch.zeros_like(v), v)).transpose(0, 1)
        A = torch.bmm(p, torch.nan_to_num(v).abs())
        vmax = torch.nan_to_num(v).abs().amax(1, keepdim=True) if L else torch.zeros_like(A)
        score = (D + 8) * u * S
        rel = 2 * score + 2 * (L + 8) * u + 12 * u + (step(kind) if kind != "f32" else 0.0)
        extra = L * 2.0 ** -36 * vmax + 2.0 ** -25 if kind == "f16" else 0.0
        tol[t] = (A * rel + extra).transpose(0, 1) + out[t].abs() * step(kind) * (1 + 2 ** -6)
        lse[t] = l[..., 0].T
        tol_lse[t] = (score + (L + 16) * u)[..., 0].T + 4 * u * lse[t].abs().nan_to_num(posinf=0.0) + 2.0 ** -36 * L
    return out, lse, tol, tol_lse


def close(got, want, tol, what=""):
    got, want = got.double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(tol), (got - want).abs())
    bad = ~(off <= tol)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol.clamp(min=1e-300)).nan_to_num(nan=math.inf).max()):.3g} "
                                 f"of the tolerance, first at {torch.nonzero(bad)[0].tolist()}: {float(got[bad][0])} for {float(want[bad][0])}")
