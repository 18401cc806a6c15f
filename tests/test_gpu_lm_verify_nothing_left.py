"""mca_verify_drafts where rejections leave nothing: every token is the one that the target's own probabilities give.

Draft and target agree and accept is 1, so max(p - c q, 0) is 0 at every symbol.  The draw's sums of V
exponentials are off by 2^-47 each at most, the fp64 reference's by V 2^-53: a sample further than 2^-40 of the sum from a
border gives one token only.
"""
import numpy as np
import pytest
import torch

from lm8_util import TYPES, host, put

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("kids", [1, 2, 4])
@pytest.mark.parametrize("vocab,requests", [(3000, 30), (150, 30), (8192, 12), (20011, 30), (40000, 30)])
def test_every_token(lm, vocab, requests, kids, typ):
    rng = np.random.default_rng(vocab + kids)
    n = kids + 1
    z = torch.from_numpy(rng.normal(size=(requests * n, vocab)) * 3).to(TYPES[typ]).cuda()
    parents = np.tile([-1] + [0] * kids, requests)
    sample = rng.random(requests).astype(np.float32)
    tokens = rng.integers(0, vocab, requests * n)
    got = lm.mca_verify_drafts(z, z.clone(), put(tokens), put(parents), put(np.arange(requests + 1) * n), put([7] * requests), n,
                               put(np.ones(requests * n), np.float32), put(sample, np.float32))
    x = host(z)[::n].astype(np.float64)
    p = np.exp(x - x.max(1, keepdims=True))
    ends = np.cumsum(p, 1)
    goal = sample.astype(np.float64)[:, None] * ends[:, -1:]
    assert (np.abs(ends - goal).min(1) > 2.0 ** -40 * ends[:, -1]).all()
    np.testing.assert_array_equal(host(got.new_len), 8)
    np.testing.assert_array_equal(host(got.token), (ends <= goal).sum(1))
