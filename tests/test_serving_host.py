"""Refusals of the serving operators: every bad argument is turned into a
status before the device is touched, and the binding's own checks raise
ValueError.  No GPU is needed."""
import ctypes
import struct

import pytest

INVALID, UNSUPPORTED = -1, -2
F32, BF16, F16 = 0, 1, 2
I32, I64 = 0, 1
P16 = 1 << 20      # never dereferenced: the calls below are refused, or have nothing to do
ODD = P16 + 1
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def P():
    from paper_1805_08166_amd import build as B
    if B.stale():
        B.build()
    import paper_1805_08166_amd
    return paper_1805_08166_amd


CACHE = dict(k=P16, v=P16, k_page=16 * 2 * 8, k_token=2 * 8, k_head=8, v_page=16 * 2 * 8, v_token=2 * 8, v_head=8, type=BF16, pages=10,
             page_size=16, heads=2, dim=8, table=P16, table_ld=4, width=4, starts=P16, lengths=P16, batch=3)


def cache(args):
    """The struct, with those of args that are its fields."""
    c = {**CACHE, **{k[2:]: args.pop(k) for k in list(args) if k.startswith("c_")}}
    return struct.pack("=19q", *((v or 0) for v in c.values()))


def append(P, k=P16, k_token=16, k_head=8, v=P16, v_token=16, v_head=8, n=5, q=P16, q_token=32, q_head=8, q_heads=4, q_out=P16,
           o_token=32, o_head=8, kw=None, qw=None, eps=1e-6, freqs=P16, rot=8, interleaved=0, rot_scale=1.0, whole=True, **c):
    return P.lib().at_paged_append(cache(c) if whole else None, k, k_token, k_head, v, v_token, v_head, n, q, q_token, q_head, q_heads,
                                   q_out, o_token, o_head, kw, qw, eps, freqs, rot, interleaved, rot_scale, None)


def attend(P, q=P16, q_token=32, q_head=8, n=5, q_heads=4, scale=0.3, window=0, out=P16, o_token=32, o_head=8, lse=None, ws=P16,
           wb=1 << 40, whole=True, **c):
    return P.lib().at_paged_attention(cache(c) if whole else None, q, q_token, q_head, n, q_heads, scale, window, out, o_token, o_head,
                                      lse, ws, wb, None)


def adjust(P, logits=P16, type=F32, ld=70, n=4, vocab=70, out=P16 * 2, ldo=70, itype=I64, past=P16, ldp=5, past_len=5, lengths=None,
           prompt=None, rep=None, freq=None, pres=None, bt=None, bias=None, n_bias=0, bias_ld=0, mask=None, mask_ld=3, masks=1,
           rows=None, valid=None):
    return P.lib().at_adjust_logits(logits, type, ld, n, vocab, out, ldo, itype, past, ldp, past_len, lengths, prompt, rep, freq, pres,
                                    bt, bias, n_bias, bias_ld, mask, mask_ld, masks, rows, valid, None)


CACHE_REFUSED = [
    (dict(whole=False), INVALID), (dict(c_type=3), INVALID), (dict(c_type=1 << 32), INVALID), (dict(c_pages=-1), INVALID),
    (dict(c_page_size=0), INVALID), (dict(c_heads=0), INVALID), (dict(c_dim=0), INVALID), (dict(c_dim=257), UNSUPPORTED),
    (dict(c_heads=65536), UNSUPPORTED), (dict(c_batch=-1), INVALID), (dict(c_batch=1 << 24), UNSUPPORTED),
    (dict(c_width=-1), INVALID), (dict(c_width=1 << 31), UNSUPPORTED), (dict(c_pages=1 << 31), UNSUPPORTED),
    (dict(c_page_size=1 << 31), UNSUPPORTED), (dict(c_k_page=-1), INVALID), (dict(c_v_head=-8), INVALID), (dict(c_table_ld=-4), INVALID),
    (dict(c_k=None), INVALID), (dict(c_v=None), INVALID), (dict(c_table=None), INVALID), (dict(c_starts=None), INVALID),
    (dict(c_lengths=None), INVALID), (dict(c_k=ODD), INVALID), (dict(c_starts=P16 + 2), INVALID), (dict(n=-1), INVALID),
    (dict(n=1 << 31), UNSUPPORTED),
]
REFUSED = [(f, dict(a), s) for f in (append, attend) for a, s in CACHE_REFUSED] + [
    (append, dict(rot=3), INVALID), (append, dict(rot=10), INVALID), (append, dict(rot=-2), INVALID), (append, dict(freqs=None), INVALID),
    (append, dict(freqs=P16 + 4), INVALID), (append, dict(rot_scale=INF), INVALID), (append, dict(eps=-1.0), INVALID),
    (append, dict(eps=NAN), INVALID), (append, dict(k=None), INVALID), (append, dict(v=None), INVALID), (append, dict(q_out=None), INVALID),
    (append, dict(k_token=-1), INVALID), (append, dict(q_head=-1), INVALID), (append, dict(o_head=7), INVALID),
    (append, dict(o_token=31), INVALID), (append, dict(kw=ODD), INVALID), (append, dict(q_heads=65536), UNSUPPORTED),
    (append, dict(c_k_head=7), INVALID), (append, dict(c_v_token=15), INVALID), (append, dict(c_k_page=255), INVALID),
    (append, dict(c_v_page=0), INVALID),
    (attend, dict(q_heads=3), INVALID), (attend, dict(q_heads=0), INVALID), (attend, dict(q_heads=65538), UNSUPPORTED),
    (attend, dict(scale=0.0), INVALID), (attend, dict(scale=-1.0), INVALID), (attend, dict(scale=NAN), INVALID),
    (attend, dict(window=-1), INVALID), (attend, dict(q=None), INVALID), (attend, dict(out=None), INVALID), (attend, dict(out=ODD), INVALID),
    (attend, dict(lse=P16 + 2), INVALID), (attend, dict(o_token=31), INVALID), (attend, dict(o_head=4), INVALID),
    (attend, dict(q_token=-1), INVALID),
    # heads above 128 values, whose rows are not whole 16 bytes or do not lie at such addresses
    (attend, dict(c_dim=132, c_k_head=132, c_k_token=264, c_v_head=132, c_v_token=264, q_head=132, q_token=528, o_head=132, o_token=528), UNSUPPORTED),
    (attend, dict(c_dim=136, c_k_head=136, c_k_token=273, c_v_head=136, c_v_token=272, q_head=136, q_token=544, o_head=136, o_token=544), UNSUPPORTED),
    (attend, dict(c_dim=136, c_k=P16 + 2, c_k_head=136, c_k_token=272, c_v_head=136, c_v_token=272, q_head=136, q_token=544, o_head=136, o_token=544), UNSUPPORTED),
    # long tables of few rows take a workspace
    (attend, dict(c_width=4096, c_table_ld=4096, ws=None), INVALID), (attend, dict(c_width=4096, c_table_ld=4096, wb=64), INVALID),
    (attend, dict(c_width=4096, c_table_ld=4096, ws=P16 + 8), INVALID),
    (adjust, dict(type=3), INVALID), (adjust, dict(itype=2), INVALID), (adjust, dict(n=-1), INVALID), (adjust, dict(ld=-1), INVALID),
    (adjust, dict(ldo=69), INVALID), (adjust, dict(out=P16, ldo=71), INVALID), (adjust, dict(past_len=-1), INVALID),
    (adjust, dict(past_len=1 << 30), UNSUPPORTED), (adjust, dict(n_bias=1 << 31), UNSUPPORTED), (adjust, dict(vocab=1 << 31, ldo=1 << 31), UNSUPPORTED),
    (adjust, dict(ldp=-1), INVALID), (adjust, dict(logits=None), INVALID), (adjust, dict(out=None), INVALID),
    (adjust, dict(bt=P16, n_bias=3), INVALID), (adjust, dict(bias=P16, n_bias=3), INVALID), (adjust, dict(past=P16 + 4), INVALID),
    (adjust, dict(out=ODD), INVALID), (adjust, dict(mask=P16 + 2), INVALID), (adjust, dict(valid=ODD), INVALID),
    (adjust, dict(mask=P16, masks=-1), INVALID), (adjust, dict(mask=P16, mask_ld=-3), INVALID),
]


@pytest.mark.parametrize("call,args,status", REFUSED, ids=lambda v: getattr(v, "__name__", None) or str(v))
def test_refused(P, call, args, status):
    assert call(P, **args) == status
    assert "at_" in P.lib().at_last_error().decode()


def test_nothing_to_do(P):
    """Empty calls succeed without a device, and take NULL buffers."""
    assert append(P, n=0, k=None, v=None, q=None) == 0
    assert append(P, c_batch=0, c_table=None, c_starts=None, c_lengths=None, k=None, v=None, q=None) == 0
    assert attend(P, n=0, q=None, out=None, ws=None, wb=0) == 0
    assert attend(P, c_batch=0, c_starts=None, c_lengths=None, ws=None, wb=0) == 0
    assert adjust(P, n=0, logits=None, out=None) == 0
    assert adjust(P, vocab=0, ldo=0, logits=None, out=None) == 0


def test_layouts_that_do_not_overlap(P):
    """Heads outside or inside the places of a page, keys and values in one buffer: taken.  Axes of one entry may have any distance."""
    none = dict(n=0)
    assert append(P, c_k_page=256, c_k_token=8, c_k_head=128, **none) == 0
    assert append(P, c_k_page=512, c_v_page=512, c_v=P16 + 512, **none) == 0
    assert append(P, c_heads=1, c_k_head=0, c_v_head=0, c_k_token=8, c_v_token=8, **none) == 0
    assert append(P, c_pages=1, c_k_page=0, c_v_page=0, **none) == 0
    assert append(P, q_heads=1, o_head=0, n=0) == 0


def test_workspace_sizes(P):
    W = P.at_paged_attention_workspace
    assert W(0, 4, 1000, 8, 2, 64) == 0 and W(4, 0, 1000, 8, 2, 64) == 0
    assert W(1, 1, 64, 8, 2, 64) == 0                       # one tile of keys
    assert W(1, 1, 100000, 8, 2, 64) > 0
    assert W(100000, 1, 100000, 32, 8, 64) == 0             # rows enough
    for bad in ((-1, 1, 1, 2, 1, 8), (1, 1, 1, 3, 2, 8), (1, 1, 1, 2, 0, 8), (1, 1, 1, 2, 1, 300), (1, 1, -1, 2, 1, 8), (1, 1, 1, 2, 1, 8, 5)):
        with pytest.raises(P.ATError):
            W(*bad)
    assert P.lib().at_paged_attention_workspace(1, 1, 1, 1, 1, 8, F32, None) == INVALID
    v = ctypes.c_int64()
    assert P.lib().at_paged_attention_workspace(1 << 31, 1, 1, 1, 1, 8, F32, ctypes.byref(v)) == UNSUPPORTED


def test_binding_checks(P):
    import torch
    k, c = torch.zeros(3, 2, 8), torch.zeros(4, 16, 2, 8)
    table, starts, lengths = (torch.zeros(*s, dtype=torch.int32) for s in ((1, 4), (2,), (1,)))
    with pytest.raises(ValueError, match="device"):
        P.at_paged_append(k, k, c, c, table, starts, lengths)
    with pytest.raises(ValueError, match="device"):
        P.at_paged_attention(k, c, c, table, starts, lengths, k)
    with pytest.raises(ValueError, match="device"):
        P.at_adjust_logits(torch.zeros(2, 5), torch.zeros(2, 5))


@pytest.mark.parametrize("call,args", [(append, dict(o_token=40)), (append, dict(o_token=8, o_head=40)), (append, dict(n=1, o_head=16)),
                                       (attend, dict(o_token=40)), (attend, dict(o_token=8, o_head=40)), (attend, dict(n=1, o_head=16))])
def test_in_place_with_other_strides_is_refused(P, call, args):
    """Outputs that start where the queries do and lie apart otherwise would replace other tokens' queries."""
    assert call(P, **args) == INVALID
    assert "stride" in P.lib().at_last_error().decode()


def test_rows_of_one_entry_are_whole_whatever_the_stride(P):
    """Distances along axes of one head, page or place do not count for whole 16 bytes: such a call goes on to its workspace."""
    wide = dict(c_dim=136, c_k_token=136, c_v_token=136, c_k_page=2176, c_v_page=2176, q_head=136, q_token=544, o_head=136, o_token=544,
                c_width=4096, c_table_ld=4096, ws=None)
    one = dict(wide, c_heads=1, c_k_head=7, c_v_head=7)
    assert attend(P, **one) == INVALID and "workspace" in P.lib().at_last_error().decode()
    assert attend(P, **{**one, "c_pages": 1, "c_k_page": 3}) == INVALID
    assert attend(P, **{**one, "c_page_size": 1, "c_width": 65536, "c_table_ld": 65536, "c_k_token": 5, "c_v_token": 5}) == INVALID
    assert attend(P, **{**one, "c_page_size": 1, "c_width": 65536, "c_table_ld": 65536, "c_k_token": 1 << 26}) == INVALID
    assert attend(P, **{**one, "c_k_token": 1 << 26}) == UNSUPPORTED
    assert attend(P, **dict(wide, c_heads=2, c_k_head=7, c_v_head=136)) == UNSUPPORTED
