"""Changes to logits against a plain 64-bit form, row by row."""
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


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def reference(x, past, lengths, prompt, rep, freq, pres, bt, bias, mask, rows, valid):
    """(values, tolerance, touched, written) in 64 bits.  Each of the four steps is off by half a step of fp32 of its result, or of its
    operands where they cancel; the last rounding by half a step of the type."""
    n, V = x.shape
    y, tol = x.astype(np.float64).copy(), np.zeros((n, V))
    touched, written = np.zeros((n, V), bool), np.zeros((n, V), bool)
    u = 2.0 ** -24
    for i in range(n):
        r = y[i]
        ruled = np.isneginf(r)
        if past is not None:
            L = past.shape[1] if lengths is None else min(max(int(lengths[i]), 0), past.shape[1])
            h = past[i, :L].astype(np.int64)
            m = 0 if prompt is None else max(int(prompt[i]), 0)
            inside = lambda a: a[(a >= 0) & (a < V)]  # noqa: E731
            seen = np.unique(inside(h))
            count = np.bincount(inside(h[m:]), minlength=V)
            touched[i, seen] = True
            if rep is not None:
                r[seen] = np.where(r[seen] > 0, r[seen] / rep[i], r[seen] * rep[i])
                tol[i, seen] += u * np.abs(r[seen])
            for f, c in ((freq, count), (pres, count > 0)):
                if f is not None:
                    r -= float(f[i]) * c
                    tol[i] += np.where(count > 0, 2 * u * (np.abs(r) + float(abs(f[i])) * c), 0)
        if bt is not None:
            for t, v in zip(bt[i], bias[i]):
                if 0 <= t < V:
                    touched[i, t] = True
            for t, v in {int(t): float(v) for t, v in zip(bt[i], bias[i]) if 0 <= t < V}.items():
                r[t] += v
                tol[i, t] += u * (abs(r[t]) + abs(v))
        r[ruled] = -np.inf
        if mask is not None:
            m = i if rows is None else int(rows[i])
            if 0 <= m < len(mask):
                bits = np.unpackbits(mask[m].view(np.uint8), bitorder="little")[:V]
                r[bits == 0] = -np.inf
        written[i, : V if valid is None else min(max(int(valid[i]), 0), V)] = True
    return y, np.nan_to_num(tol, nan=0, posinf=0, neginf=0), touched, written


class Case:
    def __init__(self, kind, n, V, past=0, biases=0, masks=0, index="int64", seed=0, pad=0, valid=False, lengths=True, prompt=True,
                 penalties=("rep", "freq", "pres")):
        import torch
        rng = np.random.default_rng(seed)
        self.kind, self.n, self.V = kind, n, V
        t = types()[kind]
        full = torch.as_tensor(rng.normal(size=(n, V + pad)) * 3, dtype=t, device=DEV)
        full[torch.as_tensor(rng.random((n, V + pad)) < 0.03, device=DEV)] = -math.inf
        self.x = full[:, :V]
        self.out = torch.full((n, V + pad), 55.0, dtype=t, device=DEV)[:, :V]
        self.a = dict.fromkeys(("past", "lengths", "prompt", "rep", "freq", "pres", "bt", "bias", "mask", "rows", "valid"))
        if past:
            self.a["past"] = rng.integers(-2, V + 2, (n, past)).astype(index)
            self.a["past"][:, ::2] = rng.integers(0, min(V, 5), self.a["past"][:, ::2].shape)
            if lengths:
                self.a["lengths"] = rng.integers(-1, past + 3, n).astype(np.int32)
                self.a["lengths"][0] = past
            if prompt:
                self.a["prompt"] = rng.integers(-1, past + 2, n).astype(np.int32)
        for name in penalties:
            self.a[name] = (rng.random(n) + (1 if name == "rep" else 0)).astype(np.float32)
        if biases:
            self.a["bt"] = rng.integers(-1, V + 1, (n, biases)).astype(index)
            self.a["bias"] = rng.normal(size=(n, biases)).astype(np.float32)
        if masks:
            self.a["mask"] = rng.integers(-2 ** 31, 2 ** 31, (masks, (V + 31) // 32)).astype(np.int32)
            self.a["mask"][0] = 0            # leaves nothing
            if masks != n:
                self.a["rows"] = rng.integers(-1, masks + 1, n).astype(np.int32)
        if valid:
            self.a["valid"] = rng.integers(-1, V + 2, n).astype(np.int32)

    def call(self, P, out=None, **kw):
        import torch
        put = {k: None if v is None else torch.as_tensor(v, device=DEV) for k, v in self.a.items()}
        P.at_adjust_logits(self.x, self.out if out is None else out, tokens=put["past"], lengths=put["lengths"],
                           prompt_lengths=put["prompt"], repetition=put["rep"], presence=put["pres"], frequency=put["freq"],
                           bias_tokens=put["bt"], bias=put["bias"], mask=put["mask"], mask_rows=put["rows"], valid=put["valid"], **kw)
        torch.cuda.synchronize()

    def check(self, P):
        import torch
        print(f"[gpu-adjust] {self.kind} {self.n} x {self.V} " + " ".join(k for k, v in self.a.items() if v is not None), flush=True)
        x = self.x.double().cpu().numpy()
        want, tol, touched, written = reference(x, *(self.a[k] for k in ("past", "lengths", "prompt", "rep", "freq", "pres", "bt",
                                                                         "bias", "mask", "rows", "valid")))
        self.call(P)
        got = self.out.double().cpu().numpy()
        assert (got[~written] == 55).all()
        ok = np.isfinite(want) & written
        assert (got[written & ~ok] == want[written & ~ok]).all()
        tol = tol + np.where(touched, np.abs(np.nan_to_num(want)) * torch.finfo(self.out.dtype).eps / 2 * (1 + 2 ** -6), 0)
        if self.kind == "f16":
            tol += np.where(touched, 2.0 ** -25, 0)
        with np.errstate(invalid="ignore"):
            off = np.abs(got - want)
        assert (off[ok] <= tol[ok]).all(), (np.nanmax((off - tol)[ok]), np.argwhere(ok & (off > tol))[0])
        # in place: the same values
        base = torch.full((self.n, self.V), 0.0, dtype=self.x.dtype, device=DEV)
        base.copy_(self.x)
        first = self.out.clone()
        keep, self.x = self.x, base
        self.call(P, out=base)
        self.x = keep
        w = torch.as_tensor(written, device=DEV)
        assert torch.equal(base[w].view(torch.int16 if self.kind != "f32" else torch.int32),
                           first[w].view(torch.int16 if self.kind != "f32" else torch.int32))
        assert torch.equal(base[~w], self.x[~w])


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 220, 1000, 8191, 8192, 8193, 50001])
def test_vocabularies(P, kind, V):
    Case(kind, 3, V, past=50, biases=7, masks=2, seed=V, pad=V % 3).check(P)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_rows(P, kind):
    """Many rows of few values, as knobs have them, and every way of leaving something out."""
    Case(kind, 3000, 220, past=7, masks=7, valid=True, seed=1).check(P)
    Case(kind, 1, 131072, past=3000, biases=300, masks=1, seed=2).check(P)
    Case(kind, 5, 700, seed=3, penalties=()).check(P)
    Case(kind, 5, 700, masks=5, seed=4, penalties=()).check(P)
    Case(kind, 5, 700, biases=40, seed=5, index="int32", valid=True, penalties=()).check(P)
    Case(kind, 5, 700, past=40, seed=6, index="int32", penalties=("rep",)).check(P)
    Case(kind, 5, 700, past=40, seed=7, penalties=("freq",), prompt=False).check(P)
    Case(kind, 5, 700, past=40, seed=8, penalties=("pres",), lengths=False).check(P)
    Case(kind, 70, 30000, past=9000, biases=3, masks=3, seed=9, index="int32").check(P)
    Case(kind, 300, 30001, past=33, biases=9, masks=3, seed=12, valid=True, pad=5).check(P)
    # long rows: tables, more of the past than a table holds, pieces of a row
    Case(kind, 130, 70001, past=3000, biases=256, masks=3, seed=13, valid=True).check(P)
    Case(kind, 130, 40000, past=100, biases=257, seed=14).check(P)
    Case(kind, 130, 40000, masks=2, seed=15, penalties=()).check(P)


def test_long_rows(P):
    """A table that is three quarters full, and a past that no table holds, of all different tokens and of few."""
    import torch
    for past in (12288, 12290):
        for few in (False, True):
            c = Case("bf16", 33, 131072, past=past, masks=2, seed=16, index="int32", lengths=False)
            if not few:
                c.a["past"][:] = np.random.default_rng(1).permutation(131072)[:past]
            c.check(P)
    Case("f32", 9, 300001, past=500, biases=30, masks=2, seed=17).check(P)
    Case("bf16", 5, 1100003, past=500, biases=30, masks=2, seed=18, valid=True).check(P)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_tables(P, kind):
    """Many long rows: tables of every filling, none, and a past that no table holds."""
    V = 16387 if kind == "f32" else 32771
    Case(kind, 830, V, past=600, biases=256, masks=3, seed=19, valid=True, pad=1).check(P)
    Case(kind, 830, V, biases=1, seed=20, penalties=()).check(P)
    c = Case(kind, 830, V, past=12288 + (kind == "f16"), masks=2, seed=21, index="int32", lengths=False)
    c.a["past"][:] = np.random.default_rng(1).permutation(V)[:c.a["past"].shape[1]]
    c.check(P)


def test_tables_of_pieces(P):
    """Half a million columns and more: several pieces of the largest size."""
    Case("f32", 17, 1000001, past=500, biases=30, masks=2, seed=17).check(P)
    Case("bf16", 31, 1100003, past=500, biases=30, masks=2, seed=18, valid=True).check(P)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("biases", [255, 256, 257, 3000])
def test_many_biases(P, kind, biases):
    """More biases of one segment than its list in LDS holds, many of them for the same tokens."""
    for V in (100, 600):
        Case(kind, 3, V, past=5, biases=biases, seed=biases).check(P)


def test_one_token_many_times(P):
    """Counts of tens of thousands, in the prompt and the answer."""
    c = Case("f32", 2, 100, past=70000, seed=10, penalties=("freq", "pres"))
    c.a["past"][:] = 3
    c.a["lengths"][:] = 70000
    c.a["prompt"][:] = [0, 69999]
    c.a["freq"][:] = 0.5
    c.check(P)
    assert float(c.out[0, 3]) < -30000 and abs(float(c.out[1, 3] - c.x[1, 3])) < 3


def test_ruled_out_and_not_finite(P):
    """-inf stays, NaN and +inf take part like numbers and are masked like them; a mask may leave nothing."""
    import torch
    x = torch.zeros(4, 64, device=DEV)
    x[:, 0], x[:, 1], x[:, 2], x[:, 3] = -math.inf, math.nan, math.inf, 2.0
    past = torch.tensor([[0, 1, 2, 3]] * 4, device=DEV)
    out = torch.empty_like(x)
    bias = torch.full((4, 1), math.inf, device=DEV)
    mask = torch.tensor([[-1, -1], [0, 0], [~0b110, -1]], dtype=torch.int32, device=DEV)
    rows = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV)
    P.at_adjust_logits(x, out, tokens=past, repetition=torch.full((4,), 2.0, device=DEV), bias_tokens=past[:, :1].contiguous(),
                       bias=bias, mask=mask, mask_rows=rows)
    got = out.cpu().numpy()
    assert np.isneginf(got[:, 0]).all() and np.isneginf(got[1]).all()
    assert np.isnan(got[[0, 3], 1]).all() and np.isposinf(got[[0, 3], 2]).all() and (got[[0, 2, 3], 3] == 1.0).all()
    assert np.isneginf(got[2, 1:3]).all()
    # what at_logprobs makes of a row that has nothing left
    lse, top = torch.empty(4, device=DEV), torch.empty(4, 2, dtype=torch.int32, device=DEV)
    P.at_logprobs(out, lse=lse, top_idx=top)
    assert float(lse[1]) == -math.inf and top[1].tolist() == [-1, -1]


def test_untouched_bits_and_repeated_biases(P):
    """NaNs that nothing applies to keep their bits; of a token's biases the last one counts, however many there are."""
    import torch
    x = torch.full((2, 40), 0x7FC1, dtype=torch.int16, device=DEV).view(torch.bfloat16)
    out = torch.zeros_like(x)
    P.at_adjust_logits(x, out)
    assert torch.equal(out.view(torch.int16), x.view(torch.int16))
    z = torch.zeros(1, 40, device=DEV)
    tokens = torch.full((1, 5000), 7, dtype=torch.int64, device=DEV)
    bias = torch.arange(5000, device=DEV, dtype=torch.float32)[None].contiguous()
    for _ in range(3):
        P.at_adjust_logits(z, z, bias_tokens=tokens, bias=bias)
    assert float(z[0, 7]) == 3 * 4999.0 and int((z != 0).sum()) == 1


def test_strides_streams_and_graphs(P):
    import torch
    c = Case("bf16", 6, 3001, past=64, biases=4, masks=2, seed=11)
    c.call(P)
    want = c.out.clone()
    # rows of the past and the biases inside larger ones, one past for all rows
    big = torch.zeros(6, 200, dtype=torch.int64, device=DEV)
    put = {k: None if v is None else torch.as_tensor(v, device=DEV) for k, v in c.a.items()}
    big[:, 9: 73] = put["past"]
    bt, b = torch.zeros(6, 9, dtype=torch.int64, device=DEV), torch.zeros(6, 9, device=DEV)
    bt[:, 2:6], b[:, 2:6] = put["bt"], put["bias"]
    c.out.fill_(55)

    def run(**kw):
        P.at_adjust_logits(c.x, c.out, tokens=big[:, 9: 73], lengths=put["lengths"], prompt_lengths=put["prompt"], repetition=put["rep"],
                           presence=put["pres"], frequency=put["freq"], bias_tokens=bt[:, 2:6], bias=b[:, 2:6], mask=put["mask"],
                           mask_rows=put["rows"], **kw)

    run()
    assert torch.equal(c.out, want)
    s = torch.cuda.Stream()
    c.out.fill_(55)
    torch.cuda.synchronize()
    run(stream=s)
    s.synchronize()
    assert torch.equal(c.out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        c.out.fill_(55)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)
    shared = put["past"][:1].expand(6, 64)
    P.at_adjust_logits(c.x, c.out, tokens=shared, repetition=put["rep"])
    for i in range(6):
        P.at_adjust_logits(c.x[i: i + 1], want[i: i + 1], tokens=put["past"][:1], repetition=put["rep"][i: i + 1])
    assert torch.equal(c.out, want)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_bias_for_every_column(P, kind):
    """And more: of several for a token the last counts.  The time goes with their number, not with the square, which took 8 ms here
    for fp32."""
    import torch
    c = Case(kind, 8, 32768, past=20, biases=32768 + 500, masks=2, seed=22)
    rng = np.random.default_rng(0)
    for i in range(8):
        c.a["bt"][i, 500:] = rng.permutation(32768)
    c.check(P)
    for n, V in ((3, 5000), (40, 70001)):
        c = Case(kind, n, V, past=9, biases=2 * V, seed=23)
        c.check(P)
    x, out = (torch.zeros(8, 32768, device=DEV, dtype=types()[kind]) for _ in range(2))
    tokens = torch.stack([torch.randperm(32768, device=DEV) for _ in range(8)])
    bias = torch.randn(8, 32768, device=DEV)
    call = lambda: P.at_adjust_logits(x, out, bias_tokens=tokens, bias=bias)  # noqa: E731
    call()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    call()
    end.record()
    torch.cuda.synchronize()
    print(f"[gpu-adjust] {begin.elapsed_time(end):.3f} ms", flush=True)
    assert begin.elapsed_time(end) < 3.0
    assert torch.equal(out, torch.zeros_like(bias).scatter_(1, tokens, bias).to(out.dtype))
