"""Norms of heads whose squares, or the sums of them, fp32 does not hold."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,rot", [(1, 0), (31, 30), (80, 40), (128, 128), (255, 254), (256, 0)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_large_and_small_heads(kind, dim, rot, eps):
    """Heads of every size from 2^-130 to 2^120 side by side, zeros and infinities among them.

    Tolerance, with u = 2^-24: the norm is off by (D + 8) u relative, a pair's products and sum by 8 u of |a| + |b|, the
    result by half a step of the type.  Below 2^-126 steps have one size: six roundings in fp32 on the way, of 2^-150 and up to
    twice that by a sum, are below 2^-146 together, and the result's is 2^-134 in bf16, whose subnormals are 2^-133 apart."""
    import torch
    import paged_reference as R
    import paper_1805_08166_amd as P
    torch.cuda.set_device(0)
    from test_gpu_paged_append import turned
    u, small = 2.0 ** -24, 2.0 ** -146 + (2.0 ** -134 if kind == "bf16" else 0.0)
    for interleaved in (False, True):
        print(f"[gpu-append] norms {kind} dim {dim} rot {rot} eps {eps} interleaved {interleaved}", flush=True)
        x = R.Batch(kind, [40, 3], [0, 50], 6, 4, dim, page=16, seed=dim)
        sizes = torch.as_tensor(np.random.default_rng(1).permutation(np.linspace(-130, 120, x.n * 10)).reshape(x.n, 10, 1), device=DEV)
        both = (x.randn(x.n, 10, dim).double() * 2.0 ** sizes).to(x.q.dtype)
        both[5, 3], both[7, 8] = 0.0, 0.0
        both[9, 2, 0], both[9, 7, dim - 1] = math.inf, -math.inf
        q, k, v = both[:, :6], both[:, 6:], x.randn(x.n, 4, dim)
        qw, kw = ((1 + 0.2 * x.randn(dim).float()).to(x.q.dtype) for _ in range(2))
        freqs = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1))
        pos = torch.cat([torch.arange(0, 40), torch.arange(50, 53)]).to(DEV)
        P.at_paged_append(k, v, x.k_cache, x.v_cache, x.table, x.starts, x.lengths, q=q, q_out=x.out, freqs=freqs if rot else None,
                          interleaved=interleaved, q_weight=qw, k_weight=kw, eps=eps)
        torch.cuda.synchronize()
        keys = torch.cat([x.k_cache[x.where(b, int(x.len[b] - x.new[b]))] for b in range(2)])
        for got, h, w in ((x.out, q, qw), (keys, k, kw)):
            y, big = turned(h, pos, freqs, interleaved, 1.0, w, eps)
            # an infinity's head: NaN in its place and in its pair, the others 0 times what is finite
            R.close(got, y, (big * (8 + dim + 8) * u + y.abs() * R.step(kind) * (1 + 2 ** -6)).nan_to_num(0.0) + small, "heads")
