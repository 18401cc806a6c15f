"""Numbers beyond 32 bits that a program gives as "no limit" are refused, not cut; and what may be left out."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_calls_refuse_numbers_beyond_32_bits():
    from paper_2607_08406_amd import lm
    from paper_2607_08406_amd.mca import MCAError
    put = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.zeros(1, 1, 32, device="cuda")
    cache = torch.zeros(2, 1, 16, 32, device="cuda")
    tail = put([[1]]), put([5]), put([0, 1]), put([-1])
    lm.mca_tree_attention(k, k, k, cache, cache, *tail, 1, max_len=16)
    slots, status = torch.zeros(9, dtype=torch.int64, device="cuda"), put([0] * 4)
    for bad in (lambda: lm.mca_tree_attention(k, k, k, cache, cache, *tail, 1, max_len=2 ** 32),
                lambda: lm.mca_tree_attention(k, k, k, cache, cache, *tail, 2 ** 32 + 1),
                lambda: lm.mca_token_logprobs(k[0], put([0]), 2 ** 32 + 1),
                lambda: lm.mca_block_tables(put([0]), put([3]), put([[0]]), put([0]), 2 ** 32 + 16, put([0, 0]), slots, status)):
        with pytest.raises(MCAError, match="2.31"):
            bad()


def test_the_entropy_may_be_left_out_without_its_gradient():
    from paper_2607_08406_amd import lm
    from paper_2607_08406_amd.mca import MCAError
    z, tok = torch.randn(3, 50, device="cuda"), torch.tensor([1, 2, 3], device="cuda")
    r = lm.mca_token_logprobs(z, tok)
    g = torch.randn(3, device="cuda")
    assert torch.equal(lm.mca_token_logprobs_grad(z, tok, r.lse, None, g), lm.mca_token_logprobs_grad(z, tok, r.lse, r.entropy, g))
    with pytest.raises(MCAError, match="entropy"):
        lm.mca_token_logprobs_grad(z, tok, r.lse, None, g, g)
