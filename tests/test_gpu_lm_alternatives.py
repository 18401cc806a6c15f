"""Alternatives of rows that NaN leaves without an order."""
import pytest
import torch

from oracle import lm as olm

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("vocab,rows", [(40, 6), (900, 6), (5000, 6), (40000, 700), (40000, 6), (300000, 6)])
def test_alternatives_of_rows_without_order(lm, typ, vocab, rows):
    """Rows of NaN of either sign, some NaN, +inf: their alternatives are symbols of the vocabulary."""
    z = torch.randn(rows, vocab, device="cuda").to(TYPES[typ])
    nan = torch.full((vocab,), float("nan"), device="cuda").to(z.dtype)
    wide = torch.int32 if typ == "f32" else torch.int16
    minus = (nan.view(wide) | torch.iinfo(wide).min).view(z.dtype)
    z[0], z[1] = nan, minus
    z[2, ::2], z[2, 1::2] = nan[::2], minus[1::2]
    z[3, vocab // 2:] = minus[vocab // 2:]
    z[4, ::3] = float("inf")
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for n in (1, 32):
        r = lm.mca_token_logprobs(z, tok, n)
        assert ((r.top_id >= 0) & (r.top_id < vocab)).all()
        assert torch.isnan(r.top_logprob[:5]).all()
        for x in (r.logprob, r.entropy, r.lse):
            assert torch.isnan(x[:5]).all() and torch.isfinite(x[5:]).all()
        assert (r.top_id[5].cpu().numpy() == olm.top(z[5:6].double().cpu().numpy(), n)[0]).all()
