"""Tensors that the language-model operators write count as changed in place: a
backward pass that needs what was there refuses, as with torch's own operations."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def put(a, dt=torch.int32):
    return torch.tensor(a, dtype=dt, device="cuda")


def test_written_tensors_count_as_changed(lm):
    table, free, offsets = put([[0, 0]]), put([2, 0, 1]), put([0, 0])
    slots, status = put([0] * 4, torch.int64), put([0] * 4)
    written = [table, free, offsets, slots, status]
    old = [t._version for t in written]
    lm.mca_block_tables(put([0]), put([3]), table, free, 2, offsets, slots, status)
    assert all(t._version > v for t, v in zip(written, old))
    k = torch.randn(4, 1, 32, device="cuda")
    caches = [torch.zeros(3, 1, 2, 32, device="cuda") for _ in range(2)]
    out, lse = torch.zeros(4, 1, 32, device="cuda"), torch.zeros(4, 1, device="cuda")
    written = [*caches, out, lse]
    old = [t._version for t in written]
    lm.mca_cache_append(k, k, *caches, slots)
    kept = caches[0]._version
    lm.mca_tree_attention(k, k, k, *caches, table, put([3]), put([0, 4]), put([-1] * 4), 4, out=out, lse=lse)
    assert all(t._version > v for t, v in zip(written, old)) and caches[0]._version == kept


@pytest.mark.parametrize("place", ["logits", "new"])
def test_a_backward_pass_notices_a_gradient_in_place_of_the_logits(lm, place):
    x = torch.randn(3, 40, device="cuda", requires_grad=True)
    tok = put([1, 2, 3])
    z = x * 2
    y = (z * z).sum()  # its gradient needs z
    with torch.no_grad():
        r = lm.mca_token_logprobs(z, tok)
        lm.mca_token_logprobs_grad(z, tok, r.lse, r.entropy, torch.ones_like(r.lse), out=z if place == "logits" else None)
    if place == "logits":
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    else:
        y.backward()
        assert torch.equal(x.grad, 8 * x.detach())


def test_a_function_of_autograd_around_the_calls(lm):
    """Forward and backward in an autograd function, where gradients are not recorded."""

    class LogProbs(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z, tok):
            r = lm.mca_token_logprobs(z, tok)
            ctx.save_for_backward(z, tok, r.lse, r.entropy)
            return r.logprob, r.entropy

        @staticmethod
        def backward(ctx, g, ge):
            return lm.mca_token_logprobs_grad(*ctx.saved_tensors, g.contiguous(), ge.contiguous()), None

    x = torch.randn(5, 90, device="cuda", requires_grad=True)
    tok = put([1, 2, 3, 4, 5])
    logprob, entropy = LogProbs.apply(x, tok)
    (logprob.sum() + entropy.sum()).backward()
    y = x.detach().double().requires_grad_()
    lp = torch.log_softmax(y, 1)
    (lp.gather(1, tok.long()[:, None]).sum() - (lp.exp() * lp).sum()).backward()
    # 32-bit sums of 90 terms of at most 20
    assert (x.grad.double() - y.grad).abs().max() <= 2.0 ** -18
