"""Proposals learned from what a search kept.

The annealing search of Algorithm 1 mutates one knob at a time, uniformly.
Its chains end in lists of good configurations, and a configuration is a short
sequence of tokens, one knob value each.  This example trains a small model on
those sequences, knob by knob: the value of knob j given the values of the knobs
before it, under a softmax over that knob's own number of values.  Trained, the
model proposes configurations, and says how likely any configuration is.

    python examples/learned_proposals.py [--steps 200]

One training step uses the sequence-model operators as a program would:

  at_embed           token vectors, times sqrt(width), summed over the knobs before
  (torch products)   hidden = tanh(x W^T), logits = hidden V^T
  at_logprobs        log probabilities of the kept values and entropies; rows
                     are ragged: knob j has knob_sizes[j] values
  at_logprobs_grad   gradient of -(log probability) - bonus * entropy
  at_embed_grad      gradient of the token table
  at_orthogonalize   the update of the hidden matrix from its momentum

and a proposal is made one row at a time: the top values of a knob, their log
probabilities, one of them drawn.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_1805_08166_amd as P  # noqa: E402
import workloads as W  # noqa: E402

DEV = "cuda"


class Proposals:
    """A model of a space's configurations as sequences of knob values."""

    def __init__(self, knob_sizes, width: int = 128, seed: int = 0):
        self.sizes = [int(s) for s in knob_sizes]
        self.width, self.knobs, self.most = width, len(self.sizes), max(self.sizes)
        # one table for every value of every knob, then one token a position
        self.first = np.concatenate([[0], np.cumsum(self.sizes)]).astype(np.int64)
        vocab = int(self.first[-1]) + self.knobs
        gen = torch.Generator(device=DEV).manual_seed(seed)
        new = lambda *shape: torch.randn(*shape, generator=gen, device=DEV) / width  # noqa: E731
        self.table, self.hidden, self.out = new(vocab, width), new(width, width) * math.sqrt(width), new(self.most, width)
        self.momentum = {name: torch.zeros_like(getattr(self, name)) for name in ("table", "hidden", "out")}
        self.scale = math.sqrt(width)
        self.offsets = torch.as_tensor(self.first[:-1], device=DEV)
        self.positions = torch.arange(self.knobs, device=DEV) + int(self.first[-1])
        self.valid = torch.tensor(self.sizes, dtype=torch.int32, device=DEV)

    def values(self, cfgs: np.ndarray) -> torch.Tensor:
        """Knob values [n, knobs] of configuration indices (knob 0 most significant)."""
        rest, cols = cfgs.astype(np.uint64), []
        for size in reversed(self.sizes):
            cols.append((rest % np.uint64(size)).astype(np.int64))
            rest = rest // np.uint64(size)
        return torch.as_tensor(np.stack(cols[::-1], 1), device=DEV)

    def indices(self, values: torch.Tensor) -> np.ndarray:
        out = np.zeros(len(values), np.uint64)
        for j, col in enumerate(values.cpu().numpy().T):
            out = out * np.uint64(self.sizes[j]) + col.astype(np.uint64)
        return out

    def _states(self, values):
        """Hidden vectors of every knob's position, from the values before it."""
        n = len(values)
        # a sequence's tokens: its values, then its positions
        tokens = torch.cat([values + self.offsets, self.positions.expand(n, -1)], 1).contiguous()
        rows = torch.empty(n * 2 * self.knobs, self.width, device=DEV)
        P.at_embed(self.table, tokens.view(-1), rows, scale=self.scale)
        rows = rows.view(n, 2, self.knobs, self.width)
        x = rows[:, 1] + torch.cumsum(rows[:, 0], 1) - rows[:, 0]
        x = x.reshape(n * self.knobs, self.width)
        return tokens, x, torch.tanh(x @ self.hidden.T)

    def log_probabilities(self, values):
        """(log probability of each knob's value, entropy, and what the gradient needs)."""
        n = len(values) * self.knobs
        tokens, x, h = self._states(values)
        logits = h @ self.out.T
        logp, entropy, lse = (torch.empty(n, device=DEV) for _ in range(3))
        valid = self.valid.repeat(len(values))
        P.at_logprobs(logits, values.reshape(-1), logp, entropy, lse, valid=valid)
        return logp, entropy, (tokens, x, h, logits, lse, valid)

    def gradients(self, values, bonus: float):
        """Loss and gradients of -mean(log probability) - bonus * mean(entropy)."""
        logp, entropy, (tokens, x, h, logits, lse, valid) = self.log_probabilities(values)
        n = len(logp)
        dlogits = torch.empty_like(logits)
        P.at_logprobs_grad(logits, values.reshape(-1), lse, entropy, torch.full_like(logp, -1.0 / n), dlogits,
                           dentropy=torch.full_like(logp, -bonus / n), valid=valid)
        dx = ((dlogits @ self.out) * (1.0 - h * h))
        grads = {"out": dlogits.T @ h, "hidden": dx.T @ x}
        dx = (dx @ self.hidden).view(len(values), self.knobs, self.width)
        # a value's vector is in the sums of all later knobs
        later = dx.flip(1).cumsum(1).flip(1) - dx
        dtable = torch.empty_like(self.table)
        P.at_embed_grad(torch.stack([later, dx], 1).view(-1, self.width), tokens.view(-1), dtable, scale=self.scale)
        grads["table"] = dtable
        return float(-(logp.mean() + bonus * entropy.mean())), grads

    def step(self, values, rate: float = 0.5, bonus: float = 0.01) -> float:
        loss, grads = self.gradients(values, bonus)
        for name, g in grads.items():
            self.momentum[name].mul_(0.9).add_(g)
        self.table.add_(self.momentum["table"], alpha=-rate * 0.02)
        self.out.add_(self.momentum["out"], alpha=-rate)
        update = torch.empty(self.hidden.shape, dtype=torch.bfloat16, device=DEV)
        P.at_orthogonalize(self.momentum["hidden"], update)
        self.hidden.add_(update, alpha=-rate * 0.02)
        return loss

    def propose(self, n: int, top: int = 8, seed: int = 0) -> torch.Tensor:
        """n configurations, each knob's value drawn from its `top` likeliest, one row at a time."""
        rng = np.random.default_rng(seed)
        out = torch.zeros(n, self.knobs, dtype=torch.int64, device=DEV)
        best, index = torch.empty(1, top, device=DEV), torch.empty(1, top, dtype=torch.int32, device=DEV)
        for i in range(n):
            for j in range(self.knobs):
                _, _, h = self._states(out[i: i + 1])
                logits = h[j: j + 1] @ self.out.T
                P.at_logprobs(logits, top_logp=best, top_idx=index, valid=self.valid[j: j + 1])
                p = np.exp(best[0].cpu().numpy().astype(np.float64))
                out[i, j] = int(index[0, rng.choice(top, p=p / p.sum())])
        return out


def kept_by_a_search(space, ensemble, chains: int, steps: int, topk: int, seed: int) -> np.ndarray:
    """Distinct configurations of the chains' best lists after an annealing run."""
    ch = P.at_chains_create(space, 0, chains, topk, seed)
    thr = torch.from_numpy(P.at_sa_thresholds(seed, 0, chains, 0, steps)).to(DEV)
    best = torch.zeros((chains, topk, 4), dtype=torch.int32, device=DEV)
    P.at_sa_run(space, ensemble, ch, steps, thr, best)
    e = P.entries(best).reshape(-1)
    return np.unique(e["cfg"][e["flag"] == 1])


def scores(space, ensemble, cfgs: np.ndarray) -> np.ndarray:
    d = torch.from_numpy(cfgs.view(np.int64)).to(DEV)
    feats = torch.empty((len(cfgs), space.n_features), dtype=torch.int32, device=DEV)
    out = torch.empty(len(cfgs), dtype=torch.float32, device=DEV)
    P.at_extract_features(space, d, feats)
    P.at_gbt_predict(ensemble, feats, out)
    return out.cpu().numpy()


def run(steps: int = 200, chains: int = 64, anneal: int = 200, proposals: int = 16, say=print) -> dict:
    space = P.at_space_create(W.GEMM, W.GEMM_512)
    fid, thr, leaf = W.make_ensemble(100, 6, 110, 1000)
    ensemble = P.at_ensemble_create(fid, thr, leaf, 110)
    kept = kept_by_a_search(space, ensemble, chains, anneal, 8, 2000)
    model = Proposals(space.knob_sizes)
    values = model.values(kept)
    losses = [model.step(values) for _ in range(steps)]
    logp = float(model.log_probabilities(values)[0].view(len(kept), -1).sum(1).mean())
    drawn = model.propose(proposals)
    got = {"kept": len(kept), "losses": losses, "logp": logp, "uniform": -math.log(space.n_configs), "proposals": drawn,
           "score_kept": float(scores(space, ensemble, kept).mean()),
           "score_proposed": float(scores(space, ensemble, model.indices(drawn)).mean()),
           "score_random": float(scores(space, ensemble, W.make_configs(4096, space.n_configs, 5)).mean())}
    say(f"{got['kept']} configurations kept by the search, mean model score {got['score_kept']:.3f}")
    say(f"loss a knob {losses[0]:.3f} -> {losses[-1]:.3f}; log probability of a kept configuration {logp:.2f} "
        f"(uniform: {got['uniform']:.2f})")
    say(f"mean model score of {proposals} proposals {got['score_proposed']:.3f}, of random configurations "
        f"{got['score_random']:.3f}")
    return got


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    run(ap.parse_args().steps)
