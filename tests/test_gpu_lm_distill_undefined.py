"""mca_distill_grad: a row whose loss is NaN has a gradient of NaN at every symbol, masked ones among them."""
import numpy as np
import pytest
import torch

from lm8_util import TYPES, host, put
from oracle import lm as olm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("vocab", [70, 767, 2000, 70000])
@pytest.mark.parametrize("rest", [False, True])
def test_a_loss_of_nan(lm, rest, vocab, typ, pad):
    """NaN and +inf of the teacher and at the student's logits, where all others, or all, are masked."""
    nan, inf = float("nan"), float("inf")
    z = torch.full((10, vocab), -inf, device="cuda", dtype=TYPES[typ])
    ids = np.tile([3, vocab // 2, vocab - 1], (10, 1))
    logp = np.full(ids.shape, np.log(0.3), np.float32)
    z[:6, put(ids[0]).long()] = 1.0
    z[0, 3], z[1, vocab - 1] = nan, inf
    logp[2, 1], logp[3, 0] = np.nan, np.inf
    # 4: others masked, nothing undefined.  5: a NaN and no valid entry.  6, 7: everything masked, the teacher NaN and +inf
    z[5, 3], ids[5] = nan, -1
    logp[6, 1], logp[7, 2] = np.nan, np.inf
    # 8: everything masked.  9: a NaN at another symbol, all the teacher's masked
    z[9, 5] = nan
    g = torch.linspace(-1.0, 2.0, 10, device="cuda")
    logp_d, ids_d = put(logp, np.float32), put(ids)
    got = lm.mca_distill(z, logp_d, ids_d, rest)
    out = torch.zeros(10, vocab + pad, device="cuda", dtype=z.dtype)[:, :vocab]
    grad = host(lm.mca_distill_grad(z, logp_d, ids_d, got.lse, got.lse_rest, g, rest, out=out)).astype(np.float64)
    loss, _, _, d = olm.distill(host(z), logp, ids, 1.0, rest)
    np.testing.assert_array_equal(np.isnan(host(got.loss)), np.isnan(loss))
    assert list(np.nonzero(np.isnan(loss))[0]) == [0, 1, 2, 3, 6, 7, 9]
    np.testing.assert_array_equal(np.isnan(grad), np.isnan(loss)[:, None] & np.ones(vocab, bool))
    assert (grad[[5, 8]] == 0).all()
    want = d[4] * float(g[4])  # probabilities of a third and 0.3, with rest 0.1 of others that have none
    assert (np.abs(grad[4] - want) <= torch.finfo(z.dtype).eps / 2 * np.abs(want) + 2.0 ** -20).all()
