"""Refusals of the sequence-model operators: every bad argument is turned into
a status before the device is touched, and the binding's own checks raise
ValueError.  No GPU is needed."""
import ctypes

import pytest

INVALID, UNSUPPORTED = -1, -2
F32, BF16, F16 = 0, 1, 2
I32, I64 = 0, 1
P16 = 1 << 20      # never dereferenced: the calls below are refused, or have nothing to do
ODD = P16 + 1


@pytest.fixture(scope="module")
def P():
    from paper_1805_08166_amd import build as B
    if B.stale():
        B.build()
    import paper_1805_08166_amd
    return paper_1805_08166_amd


def embed(P, weight=P16, wtype=F32, ldw=8, vocab=10, dim=8, tokens=P16, itype=I64, n=4, scale=1.0, out=P16, otype=F32,
          ldo=8):
    return P.lib().at_embed(weight, wtype, ldw, vocab, dim, tokens, itype, n, scale, out, otype, ldo, None)


def embed_grad(P, dout=P16, dtype=F32, ldd=8, tokens=P16, itype=I32, n=4, scale=1.0, accumulate=0, dweight=P16, gtype=F32,
               ldg=8, vocab=10, dim=8, ws=P16, wb=1 << 30):
    return P.lib().at_embed_grad(dout, dtype, ldd, tokens, itype, n, scale, accumulate, dweight, gtype, ldg, vocab, dim,
                                 ws, wb, None)


def logprobs(P, logits=P16, type=F32, ld=8, n=4, vocab=8, valid=None, tokens=P16, itype=I64, scale=1.0, k=0, logp=P16,
             top=P16, ws=P16, wb=1 << 30):
    return P.lib().at_logprobs(logits, type, ld, n, vocab, valid, tokens, itype, scale, k, logp, None, None, top, top, ws,
                               wb, None)


def logprobs_grad(P, logits=P16, type=F32, ld=8, n=4, vocab=8, valid=None, tokens=P16, itype=I64, scale=1.0, lse=P16,
                  entropy=P16, dlogp=P16, dentropy=P16, dlogits=P16, ldd=8):
    return P.lib().at_logprobs_grad(logits, type, ld, n, vocab, valid, tokens, itype, scale, lse, entropy, dlogp, dentropy,
                                    dlogits, ldd, None)


def ortho(P, x=P16, xtype=F32, xbatch=64, ldx=8, batch=2, rows=8, cols=8, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7,
          scale=1.0, out=P16, otype=BF16, obatch=64, ldo=8, ws=P16, wb=1 << 40):
    return P.lib().at_orthogonalize(x, xtype, xbatch, ldx, batch, rows, cols, steps, a, b, c, eps, scale, out, otype,
                                    obatch, ldo, ws, wb, None)


NAN, INF = float("nan"), float("inf")
REFUSED = [
    (embed, dict(wtype=3), INVALID), (embed, dict(otype=-1), INVALID), (embed, dict(itype=2), INVALID),
    (embed, dict(n=-1), INVALID), (embed, dict(vocab=0), INVALID), (embed, dict(dim=-1), INVALID),
    (embed, dict(ldw=-1), INVALID), (embed, dict(ldo=7), INVALID), (embed, dict(scale=INF), INVALID),
    (embed, dict(scale=NAN), INVALID), (embed, dict(weight=None), INVALID), (embed, dict(tokens=None), INVALID),
    (embed, dict(out=None), INVALID), (embed, dict(weight=ODD), INVALID), (embed, dict(tokens=P16 + 4), INVALID),
    (embed, dict(n=1 << 31), UNSUPPORTED), (embed, dict(vocab=1 << 31), UNSUPPORTED),
    (embed_grad, dict(dtype=9), INVALID), (embed_grad, dict(ldg=3), INVALID), (embed_grad, dict(ldd=-8), INVALID),
    (embed_grad, dict(dweight=None), INVALID), (embed_grad, dict(dout=None), INVALID),
    (embed_grad, dict(ws=None), INVALID), (embed_grad, dict(wb=16), INVALID), (embed_grad, dict(ws=P16 + 8), INVALID),
    (embed_grad, dict(dweight=ODD, gtype=BF16), INVALID), (embed_grad, dict(n=1 << 31), UNSUPPORTED),
    (logprobs, dict(type=5), INVALID), (logprobs, dict(itype=7), INVALID), (logprobs, dict(ld=-1), INVALID),
    (logprobs, dict(scale=0.0), INVALID), (logprobs, dict(scale=-1.0), INVALID), (logprobs, dict(scale=NAN), INVALID),
    (logprobs, dict(k=65), INVALID), (logprobs, dict(k=-1), INVALID), (logprobs, dict(logits=None), INVALID),
    (logprobs, dict(logits=ODD, type=F16), INVALID), (logprobs, dict(logp=P16 + 2), INVALID),
    (logprobs, dict(n=-3), INVALID), (logprobs, dict(vocab=1 << 31, ld=1 << 31), UNSUPPORTED),
    (logprobs, dict(n=1, vocab=100000, ws=None), INVALID), (logprobs, dict(n=1, vocab=100000, wb=8), INVALID),
    (logprobs_grad, dict(type=4), INVALID), (logprobs_grad, dict(ldd=7), INVALID), (logprobs_grad, dict(lse=None), INVALID),
    (logprobs_grad, dict(entropy=None), INVALID), (logprobs_grad, dict(dlogits=None), INVALID),
    (logprobs_grad, dict(scale=0.0), INVALID), (logprobs_grad, dict(dlogits=ODD, type=BF16, logits=P16), INVALID),
    (logprobs_grad, dict(n=1 << 30, vocab=1 << 20, ldd=1 << 20), UNSUPPORTED),
    (ortho, dict(xtype=8), INVALID), (ortho, dict(otype=F16), UNSUPPORTED), (ortho, dict(steps=0), INVALID),
    (ortho, dict(steps=65), INVALID), (ortho, dict(a=NAN), INVALID), (ortho, dict(eps=-1.0), INVALID),
    (ortho, dict(scale=INF), INVALID), (ortho, dict(ldo=7), INVALID), (ortho, dict(obatch=63), INVALID),
    (ortho, dict(ldx=-1), INVALID), (ortho, dict(x=None), INVALID), (ortho, dict(out=ODD), INVALID),
    # both sides up to 128 take no workspace
    (ortho, dict(rows=200, obatch=1600, ws=None), INVALID), (ortho, dict(rows=200, obatch=1600, wb=100), INVALID),
    (ortho, dict(batch=65536), UNSUPPORTED),
    (ortho, dict(rows=65537), UNSUPPORTED), (ortho, dict(rows=-1), INVALID),
]


@pytest.mark.parametrize("call,args,status", REFUSED, ids=lambda v: getattr(v, "__name__", None) or str(v))
def test_refused(P, call, args, status):
    assert call(P, **args) == status
    assert "at_" in P.lib().at_last_error().decode()


def test_nothing_to_do(P):
    """Empty calls succeed without a device, and take NULL buffers."""
    assert embed(P, n=0, weight=None, tokens=None, out=None) == 0
    assert embed(P, dim=0, ldo=0, weight=None, tokens=None, out=None) == 0
    assert embed_grad(P, n=0, accumulate=1, dweight=None, ws=None) == 0
    assert embed_grad(P, dim=0, ldg=0, dweight=None, ws=None) == 0
    assert logprobs(P, n=0, logits=None) == 0
    assert logprobs_grad(P, vocab=0, ldd=0) == 0
    assert ortho(P, rows=0, x=None, out=None, ws=None) == 0
    assert ortho(P, batch=0, x=None, out=None, ws=None) == 0


def test_workspace_sizes(P):
    assert P.at_embed_grad_workspace(100, 50, 64) > 100 * 8
    assert P.at_logprobs_workspace(4096, 220, 8) == 0          # a wave a row
    assert P.at_logprobs_workspace(1, 131072, 20) > 0          # one row over many workgroups
    assert P.at_orthogonalize_workspace(2, 100, 300) > 2 * 100 * 300 * 4
    for fn, args in [(P.at_embed_grad_workspace, (-1, 5, 5)), (P.at_logprobs_workspace, (1, 5, 65)),
                     (P.at_orthogonalize_workspace, (1, -1, 5))]:
        with pytest.raises(P.ATError):
            fn(*args)
    v = ctypes.c_int64()
    assert P.lib().at_embed_grad_workspace(4, 4, 4, None) == INVALID
    assert P.lib().at_logprobs_workspace(1 << 31, 4, 4, ctypes.byref(v)) == UNSUPPORTED


def test_binding_checks(P):
    import torch
    w, t, o = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device"):
        P.at_embed(w, t, o)
    with pytest.raises(ValueError, match="int32 or int64"):
        P.at_embed(w, t.float(), o)
    with pytest.raises(ValueError, match="device"):
        P.at_embed_grad(o, t, w)
    with pytest.raises(ValueError, match="device"):
        P.at_logprobs(w)
    with pytest.raises(ValueError, match="device"):
        P.at_logprobs_grad(w, None, None, None, None, w)
    with pytest.raises(ValueError, match="shape"):
        P.at_orthogonalize(w, o)
    with pytest.raises(ValueError, match="device"):
        P.at_orthogonalize(w, w)


def test_fp16_products_flag(P):
    """The flag goes with an output type, of the same ones, and needs less workspace."""
    for base in (F32, BF16):
        assert ortho(P, rows=0, x=None, out=None, otype=base | P.AT_FP16_PRODUCTS) == 0
        assert ortho(P, steps=0, otype=base | P.AT_FP16_PRODUCTS) == INVALID
    assert ortho(P, otype=F16 | P.AT_FP16_PRODUCTS) == UNSUPPORTED
    assert ortho(P, otype=32) == UNSUPPORTED
    for base in (F32, BF16):
        whole = P.at_orthogonalize_workspace(2, 700, 900, base)
        assert whole == P.at_orthogonalize_workspace(2, 700, 900, F32) > 2 * 700 * 900 * 12
        assert P.at_orthogonalize_workspace(2, 700, 900, base | P.AT_FP16_PRODUCTS) < whole


def test_embed_grad_past_a_launch(P):
    """2^30 tokens of one row, repeated, of 8192 columns: 2^24 workgroups of 256 threads are
    more than a launch holds.  One column tile fewer is not."""
    many = dict(ldd=0, n=1 << 30, vocab=10, dtype=BF16, wb=1 << 42)
    assert embed_grad(P, dim=8192, ldg=8192, **many) == UNSUPPORTED
    assert "at_embed_grad" in P.lib().at_last_error().decode()
    assert embed_grad(P, dim=8192 - 512, ldg=8192, ws=None, **many) == INVALID    # its workspace is looked at
