"""mca_cache8_append into blocks whose kept tokens have larger scales than the source type would give them: what is
written reads back as numbers that the type holds."""
import numpy as np
import pytest
import torch

from lm8_util import TYPES, cache, codes, host, put
from oracle import lm as olm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("typ,exps", [("f16", [7, 8, 9, 10, 12, 15, 20, 21, 22, 23, 24, 25, 26, 40, 127]),
                                      ("bf16", [119, 120, 121, 122, 125, 127]), ("f32", [119, 120, 121, 122, 125, 127])])
def test_largest_values_behind_larger_ones(lm, typ, exps):
    dim, n, big = 32, len(exps), torch.finfo(TYPES[typ]).max
    # every request has one token and takes three: values about the type's largest, of both signs
    top = torch.linspace(0.85, 1.0, 3 * dim, device="cuda", dtype=torch.float64).view(3, 1, dim) * big
    k = top.repeat(n, 1, 1).to(TYPES[typ])
    v = -k
    (kc, _), (vc, _) = cache(np.random.default_rng(1), n, 1, 8, dim)
    scales = np.array(exps)[:, None] + 127
    got = [codes(kc), codes(vc), put(scales, np.uint8), put(scales, np.uint8)]
    table, lengths, offsets = put(np.arange(n)[:, None]), put([1] * n), put(np.arange(n + 1) * 3)
    lm.mca_cache8_append(k, v, *got, table, lengths, offsets)
    want = olm.cache8_append(host(k), host(v), kc, vc, scales.astype(np.uint8), scales.astype(np.uint8), host(table), [1] * n,
                             np.arange(n + 1) * 3, None, typ)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(host(g), w)
    back = lm.mca_cache8_read(torch.zeros_like(k), torch.zeros_like(v), *got, table, lengths, offsets)
    every = olm.e4m3_value(np.arange(127, dtype=np.uint8))
    for x, y in zip(back, (k, v)):
        assert torch.isfinite(x).all()
        x, y = x.double().cpu().numpy().reshape(n, -1), y.double().cpu().numpy().reshape(n, -1)
        for r, e in enumerate(exps):
            # the nearest of what the type holds of the codes' values (both at a tie)
            held = every * 2.0 ** max(e, 8 if typ == "f16" else 120)
            held = held[held <= big]
            off = np.abs(np.abs(y[r])[:, None] - held).min(1)
            assert (np.abs(x[r] - y[r]) == off).all(), (e, x[r][:3], y[r][:3])
