"""The learned-proposals example: the sequence-model operators together, after
a search.  Its gradients are compared with differences of its own loss in 64
bits (a plain torch model of the same parameters), its training with where it
started."""
import math
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    import torch
    torch.cuda.set_device(0)
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import learned_proposals
    return learned_proposals


def plain_loss(m, table, hidden, out, values, bonus):
    """The loss in 64 bits on the CPU."""
    import torch
    n = len(values)
    value = table[values + m.offsets.cpu()] * m.scale
    x = table[m.positions.cpu()] * m.scale + value.cumsum(1) - value
    logits = torch.tanh(x.reshape(n * m.knobs, m.width) @ hidden.T) @ out.T
    valid = m.valid.cpu().repeat(n)
    logits = logits.masked_fill(torch.arange(m.most)[None] >= valid[:, None], -math.inf)
    lp = torch.log_softmax(logits, 1)
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    return float(-(lp[torch.arange(len(lp)), values.reshape(-1)].mean() + bonus * entropy.mean()))


def test_gradients_against_differences(E):
    """Central differences along random directions.  Step 1e-4 of a direction of
    norm 1: truncation below 1e-7, fp32 gradients within 1e-5 of their norm."""
    import torch
    m = E.Proposals([11, 7, 3, 2], width=32, seed=3)
    gen = torch.Generator().manual_seed(1)
    values = torch.stack([torch.randint(0, s, (25,), generator=gen) for s in m.sizes], 1)
    _, grads = m.gradients(values.to("cuda"), 0.3)
    base = {k: getattr(m, k).cpu().double() for k in ("table", "hidden", "out")}
    for name in base:
        for _ in range(3):
            v = torch.randn(base[name].shape, generator=gen).double()
            v /= v.norm()
            up, down = ({**base, name: base[name] + s * 1e-4 * v} for s in (1, -1))
            slope = (plain_loss(m, **up, values=values, bonus=0.3) - plain_loss(m, **down, values=values, bonus=0.3)) / 2e-4
            got = float((grads[name].cpu().double() * v).sum())
            assert abs(slope - got) < 1e-6 + 1e-5 * float(grads[name].norm()), (name, slope, got)


def test_knob_values_round_trip(E):
    m = E.Proposals([220, 220, 10, 3, 2], width=16)
    cfgs = np.array([0, 1, 5, 12345, 220 * 220 * 60 - 1], np.uint64)
    assert np.array_equal(m.indices(m.values(cfgs)), cfgs)


def test_trains_and_proposes(E):
    got = E.run(steps=60, chains=32, anneal=60, proposals=4, say=lambda s: print("[gpu-proposals]", s, flush=True))
    assert all(math.isfinite(x) for x in got["losses"])
    assert got["losses"][-1] < got["losses"][0] - 0.1
    assert got["logp"] > got["uniform"] + 1.0
    sizes = np.array([220, 220, 10, 3, 2])
    v = got["proposals"].cpu().numpy()
    assert v.shape == (4, 5) and (v >= 0).all() and (v < sizes).all()
