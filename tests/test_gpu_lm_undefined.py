"""Results that the definitions leave without a value, and values next to the types' ends."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("length", [0, 40, 700])
@pytest.mark.parametrize("nodes,max_len", [(2, 40), (2, 1000), (2, 1 << 17), (80, 1 << 17), (240, 1 << 17)])
def test_rows_of_nothing_but_minus_infinity(lm, typ, dim, length, nodes, max_len):
    """Every score that a row sees is -inf: softmax and its sum have no value, whichever way the work is cut.  Request
    1 has the same keys but for one cached token; its rows see that alone."""
    if length > max_len:
        length = max_len
    dt, block = TYPES[typ], 16
    n = min(nodes, 80)
    group = nodes // n
    width = max(1, -(-length // block))
    g = torch.Generator().manual_seed(nodes + length)
    q, k, v = torch.zeros(2 * n, group, dim), torch.zeros(2 * n, 1, dim), torch.randn(2 * n, 1, dim, generator=g)
    q[:, :, 3], k[:, 0, 3] = 1.0, -float("inf")
    kc, vc = torch.zeros(2 * width, 1, block, dim), torch.randn(2 * width, 1, block, dim, generator=g)
    kc[..., 3] = -float("inf")
    at = length // 2
    kc[width + at // block, 0, at % block, 3] = 0.5
    put = lambda a: torch.tensor(a, dtype=torch.int32).cuda()  # noqa: E731
    q, k, v, kc, vc = (x.to(dt).cuda() for x in (q, k, v, kc, vc))
    out, lse = lm.mca_tree_attention(q, k, v, kc, vc, put(np.arange(2 * width).reshape(2, width)), put([length] * 2),
                                     put([0, n, 2 * n]), put(np.tile(np.arange(n) - 1, 2)), n, max_len=max_len, scale=1.0)
    assert torch.isnan(out[:n]).all() and torch.isnan(lse[:n]).all()
    if length:
        assert (out[n:] == vc[width + at // block, 0, at % block]).all()
        assert torch.allclose(lse[n:], torch.full_like(lse[n:], 0.5), atol=1e-6, rtol=0)
