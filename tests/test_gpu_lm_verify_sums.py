"""mca_verify_drafts: what a child's acceptance is held to over long rows.

Rows of 1 and w = exp(-c) in turn, whose sum a softmax divides by.  Added one by one in 32 bits a lane's
sum would drift: each addition of w to a sum of 2^7 and more loses the same part of a step, w's bits
below that being about half of one.  Bounds, u = 2^-24: w is off by one step of an exponential between
0.5 and 1 (2 u relative) and by the roundings of its argument (c < 0.11, two roundings); up to 8 of them are added in 32 bits
(7 u), then in 64.  So p is off by less than 10 u, accept by 1 u for its type: at 12 u on either side of the
border the decision is certain.
"""
import math

import numpy as np
import pytest
import torch

from lm8_util import TYPES, host, put

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("bits,part", [(17, 0.49), (17, 0.51), (16, 0.49), (16, 0.51)])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("vocab,requests,nodes", [(8192, 8, 3), (16380, 8, 2), (70000, 1024, 2)])
def test_children_next_to_their_border(lm, typ, vocab, requests, nodes, drawn, bits, part):
    """Small vocabularies in one workgroup, a row in one part, and rows so many that long ones are in one part."""
    w = math.floor(0.9 * 2 ** bits) / 2 ** bits + part * 2.0 ** -bits
    c = -math.log(w)
    z = torch.full((vocab,), -1.0, device="cuda")
    z[::4] = 0.0
    rows = requests * nodes
    target = z.to(TYPES[typ]).expand(rows, vocab).contiguous()
    draft = torch.zeros_like(target) if drawn else None
    ones = -(-vocab // 4)
    p = math.exp(-c) / (ones + (vocab - ones) * math.exp(-c))
    border = p * vocab if drawn else p  # u q < p, q = 1 / vocab or 1
    sign = np.where(np.arange(requests) % 2 == 0, 1, -1)
    accept = np.full((requests, nodes), 0.5)
    accept[:, 1] = border * (1 + sign * 12 * U)
    tokens = np.ones((requests, nodes), int)
    parents = np.full((requests, nodes), -1)
    parents[:, 1] = 0
    lengths = np.arange(requests)
    got = lm.mca_verify_drafts(target, draft, put(tokens.reshape(-1)), put(parents.reshape(-1)), put(np.arange(requests + 1) * nodes),
                               put(lengths), nodes, put(accept.reshape(-1), np.float32), put(np.full(requests, 0.5), np.float32),
                               scale=c)
    np.testing.assert_array_equal(host(got.new_len) - lengths, np.where(sign > 0, 1, 2))
