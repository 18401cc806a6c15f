"""mca_distill with `rest`, teacher's symbols at the ends of rows and of their parts.

The others' sum is relative to the largest of the others, wherever the teacher's symbols stand and
however far above the rest they lie.  Bounds, u = 2^-24: the others' logits lie within 12 of each
other, so an exponential is off by at most (2 + 3 * 12) u (its argument is the product of a
difference and scale log2 e, each rounded), and a sum of V of them by as much and u for each of
a lane's terms and of the joins, (V / 64 + 186) u in all as a bound on both.  lse_rest is off by that and half a
step of its own; the loss, whose logarithms are of 64 bits, by that of both sums and half a step of
its own.  No term grows with the distance to the teacher's symbols.
"""
import numpy as np
import pytest
import torch

from lm8_util import TYPES, host, put
from oracle import lm as olm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def ends(vocab, head, per_vector, splits):
    """Symbols at both ends of a row that has `head` symbols in front of its first vector, of its vectors, and of the
    first and last vectors of its parts."""
    nvec = (vocab - head) // per_vector
    per = -(-nvec // splits)
    at = {0, vocab - 1, head, head + nvec * per_vector - 1}
    for i in range(splits):
        a, b = min(i * per, nvec), min((i + 1) * per, nvec)
        at |= {head + a * per_vector, head + b * per_vector - 1, head + b * per_vector - per_vector}
    return sorted(x for x in at if 0 <= x < vocab)


def check(lm, z, ids, far):
    """Teachers of one symbol each, `far` above the others."""
    T, V = z.shape
    z[torch.arange(T, device="cuda"), put(ids[:, 0]).long()] = far
    rng = np.random.default_rng(len(ids))
    logp = np.log(rng.uniform(0.2, 0.8, ids.shape)).astype(np.float32)
    g = torch.linspace(0.5, 2.0, T, device="cuda")
    got = lm.mca_distill(z, put(logp, np.float32), put(ids), True)
    grad = host(lm.mca_distill_grad(z, put(logp, np.float32), put(ids), got.lse, got.lse_rest, g, True)).astype(np.float64)
    loss, lse, lrest, d = olm.distill(host(z), logp, ids, 1.0, True)
    e = (V / 64 + 186) * U
    for name, a, w, lim in (("lse", got.lse, lse, e), ("lse_rest", got.lse_rest, lrest, e), ("loss", got.loss, loss, 2 * e)):
        a = host(a).astype(np.float64)
        bad = ~(np.abs(a - w) <= lim + U * np.abs(w))
        assert not bad.any(), (name, ids[bad][:5], a[bad][:5], w[bad][:5])
    # a gradient: its probabilities under the student and among the others from sums off by e, logits less sums of at
    # most `far` (rounded once, as are the sums), then half a step of its type
    want = d * host(g).astype(np.float64)[:, None]
    eps, tiny = torch.finfo(z.dtype).eps / 2, torch.finfo(z.dtype).smallest_normal
    x = host(z).astype(np.float64)
    size = np.exp(np.minimum(x - lse[:, None], 0)) + np.exp(np.minimum(x - lrest[:, None], 0)) * (x < far)
    rel = 2 * e + 4 * U * (4 + np.abs(x - lse[:, None]).clip(max=200) + np.abs(lse)[:, None])
    bad = ~(np.abs(grad - want) <= eps * np.abs(want) * (1 + 2.0 ** -6) + 2 * (rel * size + 4 * U) + tiny)
    assert not bad.any(), (np.argwhere(bad)[:5], grad[bad][:5], want[bad][:5])


@pytest.mark.parametrize("far", [30.0, 86.0, 100.0, 300.0, 10000.0])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("vocab", [70, 600, 1025, 2000, 2048, 8192, 8200, 50001])
def test_a_symbol_far_above_the_others(lm, typ, vocab, far):
    """A row in one part: every place of its first and last vectors."""
    per = 4 if typ == "f32" else 8
    at = sorted({x for x in list(range(2 * per)) + list(range(vocab - 3 * per, vocab)) if 0 <= x < vocab})
    gen = torch.Generator("cuda").manual_seed(vocab)
    z = torch.randn(len(at), vocab, device="cuda", generator=gen).clamp(-6, 6).to(TYPES[typ])
    check(lm, z, np.array(at)[:, None], far)


@pytest.mark.parametrize("far", [30.0, 86.0, 100.0, 300.0, 10000.0])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("vocab", [65537, 70000, 100003])
def test_a_symbol_far_above_the_others_of_rows_in_parts(lm, typ, vocab, far):
    per = 4 if typ == "f32" else 8
    splits = -(-vocab // 8192)
    at = sorted({x for head in (0, 1, per - 1) for x in ends(vocab, head, per, splits)})
    gen = torch.Generator("cuda").manual_seed(vocab)
    for part in (at[:32], at[32:64], at[64:96]):  # rows few enough that each is worked on in parts
        if part:
            z = torch.randn(len(part), vocab, device="cuda", generator=gen).clamp(-6, 6).to(TYPES[typ])
            check(lm, z, np.array(part)[:, None], far)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("vocab", [2000, 70000])
def test_several_symbols_of_the_last_vector(lm, typ, vocab):
    """All of the last vector's symbols, and others' masked by a large negative number."""
    per = 4 if typ == "f32" else 8
    ids = np.tile(np.arange(vocab - per, vocab), (5, 1))
    z = torch.full((5, vocab), -1e4, device="cuda").to(TYPES[typ])
    z += torch.randn(5, vocab, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(z.dtype)
    z[:, vocab - per:] = torch.linspace(-1.0, 1.0, per, device="cuda").to(z.dtype)
    logp = np.full(ids.shape, np.log(0.9 / per), np.float32)
    got = lm.mca_distill(z, put(logp, np.float32), put(ids), True)
    loss, lse, lrest, _ = olm.distill(host(z), logp, ids, 1.0, True)
    e = (vocab / 64 + 186) * U
    for a, w in ((got.lse, lse), (got.lse_rest, lrest), (got.loss, loss)):
        assert (np.abs(host(a).astype(np.float64) - w) <= 2 * e + U * np.abs(w)).all()
