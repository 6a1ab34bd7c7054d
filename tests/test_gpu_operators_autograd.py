"""The operators write their outputs behind autograd's back, and say so: a graph that
saved what they overwrote refuses to go backwards."""
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import torch
    torch.cuda.set_device(0)
    import paper_1805_08166_amd
    return paper_1805_08166_amd


def test_outputs_are_marked_as_written(P):
    import torch
    n, vocab, dim = 6, 40, 16
    new = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
    w, out, t = new(vocab, dim), new(n, dim), torch.zeros(n, dtype=torch.int64, device=DEV)
    x, d, logp, H, lse = new(n, vocab), new(n, vocab), new(n), new(n), new(n)
    top, idx = new(n, 3), torch.zeros(n, 3, dtype=torch.int32, device=DEV)
    m, u = torch.randn(8, 8, device=DEV), new(8, 8)

    def bumped(call, outs, ins):
        before = [t._version for t in outs], [t._version for t in ins]
        call()
        assert all(t._version > v for t, v in zip(outs, before[0]))
        assert [t._version for t in ins] == before[1]

    bumped(lambda: P.at_embed(w, t, out), [out], [w, t])
    bumped(lambda: P.at_embed_grad(out, t, w, accumulate=True), [w], [out, t])
    bumped(lambda: P.at_logprobs(x, t, logp, H, lse, top, idx), [logp, H, lse, top, idx], [x, t])
    bumped(lambda: P.at_logprobs(x, entropy=H), [H], [x, logp])
    bumped(lambda: P.at_logprobs_grad(x, t, lse, H, logp, d), [d], [x, t, lse, H, logp])
    bumped(lambda: P.at_orthogonalize(m, u), [u], [m])


def test_backward_through_an_overwritten_tensor_is_refused(P):
    import torch
    w, t = torch.randn(9, 4, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    rows, scale = torch.ones(3, 4, device=DEV), torch.ones(4, device=DEV, requires_grad=True)
    loss = (rows * scale).sum()
    P.at_embed(w, t, rows)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        out = torch.empty(3, 4, device=DEV)
        P.at_embed(w, t, out)
        assert torch.equal(out, w[t])
