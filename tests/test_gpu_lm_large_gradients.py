"""Gradients of log probabilities and entropies next to the end of 32-bit floats."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("vocab", [70, 5001])
@pytest.mark.parametrize("typ", list(TYPES))
def test_gradients_of_the_entropy_up_to_the_largest(lm, typ, vocab):
    """Symbols of probability 0 get 0 for every finite gradient of the entropy; of one symbol with all the probability
    the entropy does not move."""
    z = torch.full((4, vocab), -float("inf"))
    z[:, 5] = 1.0
    z[1, 6:9] = torch.tensor([-30000.0, -20000.0, -200.0])
    z[2:, 9] = 1.0
    z = z.to(TYPES[typ]).cuda()
    tok = torch.full((4,), 5, device="cuda")
    res = lm.mca_token_logprobs(z, tok)
    ge = torch.tensor([3.4e38, -3.4e38, 3.4e38, 1e36], device="cuda")
    got = lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, torch.ones(4, device="cuda"), ge)
    p = torch.softmax(z.double(), 1)
    off = (p == 0) | (p < 1e-60)
    assert (got[off] == 0).all()
    assert (got[:2, 5] == 0).all()
