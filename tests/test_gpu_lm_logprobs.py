"""GPU parity of mca_token_logprobs and its gradient against the fp64 oracle.

Tolerances, from the arithmetic (32 bits throughout): an exponent's argument
y = (z - max) log2 e is rounded once, and a log probability is the difference of
one such and log2 of a sum, so both are off by 2^-24 of their size a few times;
a lane sums V / 64 terms one after the other in the longest form and the rest in
a tree of at most 40; the hardware's exponential and logarithm are good to
2^-22.  The gradient is its formula from lse and entropy as given, rounded once
to the logits' type.
"""
import numpy as np
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


def check(logits, tokens, res, n_top):
    z = logits.float().cpu().numpy().astype(np.float64)
    tok = tokens.cpu().numpy()
    V = z.shape[1]
    lp, ent, lse, logp = olm.token_logprobs(z, tok)
    got = [x.cpu().numpy() for x in res]
    with np.errstate(invalid="ignore"):
        top = z.max(1)
        p = np.exp(logp)
        spread = np.where(p > 0, p * np.abs(np.where(p > 0, z - top[:, None], 0)), 0).sum(1)  # mean |z - max|
    sums = (V / 64 + 40) * 2.0 ** -24

    def tol(dist):
        return 2.0 ** -22 * (4 + dist + spread) + sums

    def near(a, b, t, what):
        same = (a == b) | (np.abs(a - b) <= t)
        assert same.all(), (what, np.abs(a - b)[~same], t[~same] if np.ndim(t) else t)

    with np.errstate(invalid="ignore"):
        dist = np.abs(np.where(np.isfinite(lp) & (tok >= 0) & (tok < V), z[np.arange(len(z)), np.clip(tok, 0, V - 1)] - top, 0))
        near(got[0], lp, tol(np.where(np.isfinite(dist), dist, 0)), "logprob")
        near(got[1], ent, tol(spread) + sums * spread, "entropy")
        near(got[2], lse, tol(0) + 2.0 ** -22 * np.where(np.isfinite(lse), np.abs(lse), 0), "lse")
    want = olm.top(z, n_top)
    assert got[4].shape == (len(z), n_top) and (got[4] == want).all()
    if n_top:
        val = np.take_along_axis(logp, want, 1)
        with np.errstate(invalid="ignore"):
            same = (got[3] == val) | (np.abs(got[3] - val) <= tol(0)[:, None] + 2.0 ** -22 * np.abs(val))
        assert same.all()


def make(seed, typ, rows, vocab, scale=3.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.normal(size=(rows, vocab)) * scale + 5).to(TYPES[typ]).cuda()
    tok = torch.from_numpy(rng.integers(0, vocab, rows)).cuda()
    return z, tok


SIZES = [1, 2, 63, 64, 65, 127, 128, 129, 200, 256, 257, 500, 513, 1000, 1024, 1025, 1031, 2047, 4099, 9001, 33000, 70001]


@pytest.mark.parametrize("vocab", SIZES)
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_sizes(lm, typ, vocab):
    z, tok = make(vocab, typ, 5, vocab)
    for n in (0, min(vocab, 7), min(vocab, 32)):
        check(z, tok, lm.mca_token_logprobs(z, tok, n), n)


@pytest.mark.parametrize("rows", [1, 3, 64, 700])
def test_row_counts(lm, rows):
    """From a row split over many workgroups to a workgroup a row."""
    for vocab in (40001,) if rows > 3 else (40001, 262144, 262145, 600011):
        z, tok = make(rows, "bf16", rows, vocab)
        for n in (0, 20):
            check(z, tok, lm.mca_token_logprobs(z, tok, n), n)


@pytest.mark.parametrize("vocab", [300, 5000, 50000, 300000])
def test_ties(lm, vocab):
    """Equal values, the two zeros among them: the lowest symbols, in order."""
    for rows in (4, 600):
        _ties(lm, vocab, rows)


def _ties(lm, vocab, rows):
    rng = np.random.default_rng(vocab)
    z = torch.from_numpy(rng.integers(-2, 2, (rows, vocab)).astype(np.float32)).to(torch.bfloat16).cuda()
    z[1] = 0.0
    z[1, ::3] = -0.0
    z[2] = 1.0
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    res = lm.mca_token_logprobs(z, tok, 32)
    check(z[:8], tok[:8], [x[:8] for x in res], 32)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_ordered_rows(lm, typ, order):
    """Every chunk (or none) passes the largest so far."""
    z = torch.linspace(-20, 20, 60000)
    for rows in (2, 600):
        y = (z if order == "rising" else z.flip(0)).to(TYPES[typ]).cuda()[None].repeat(rows, 1)
        tok = torch.arange(rows, device="cuda")
        res = lm.mca_token_logprobs(y, tok, 32)
        check(y[:2], tok[:2], [x[:2] for x in res], 32)


@pytest.mark.parametrize("vocab", [70, 900, 3001, 80000])
def test_masked_symbols(lm, vocab):
    """Symbols of -inf: no probability, behind every other alternative; a row with one symbol, one with none; the
    type's lowest value instead of -inf."""
    z, tok = make(vocab, "f32", 6, vocab)
    z[0, torch.rand(vocab, device="cuda") < 0.5] = -float("inf")
    z[1] = -float("inf")
    z[1, vocab // 2] = 2.0
    z[2] = -float("inf")
    z[3, 1:] = torch.finfo(torch.float32).min
    z[4, tok[4]] = -float("inf")
    z[5] = torch.finfo(torch.float32).min
    res = lm.mca_token_logprobs(z, tok, 8)
    check(z, tok, res, 8)
    g, ge = torch.randn(2, 6, device="cuda")
    check_grad(z, tok, res.lse, res.entropy, g, ge, lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, g, ge))


@pytest.mark.parametrize("vocab", [65, 5001])
def test_tokens_that_are_none(lm, vocab):
    for dt in (torch.int32, torch.int64):
        z, _ = make(vocab, "bf16", 5, vocab)
        tok = torch.tensor([-1, vocab, 0, vocab - 1, -2 ** 31], dtype=dt, device="cuda")
        res = lm.mca_token_logprobs(z, tok, 3)
        check(z, tok, res, 3)
        assert (res.logprob[[0, 1, 4]] == 0).all()
        g, ge = torch.randn(2, 5, device="cuda")
        check_grad(z, tok, res.lse, res.entropy, g, ge, lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, g, ge))
    tok = torch.tensor([2 ** 32, 2 ** 40, -2 ** 33, 2 ** 32 + 1, 1], device="cuda")  # not what their low words say
    res = lm.mca_token_logprobs(z, tok)
    assert (res.logprob[:4] == 0).all() and res.logprob[4] != 0


@pytest.mark.parametrize("vocab", [90, 30000])
def test_not_a_number(lm, vocab):
    """NaN and +inf: floating results NaN, other rows as ever."""
    z, tok = make(vocab, "f16", 4, vocab)
    z[1, vocab // 3] = float("nan")
    z[2, vocab // 2] = float("inf")
    res = lm.mca_token_logprobs(z, tok, 4)
    for x in (res.logprob, res.entropy, res.lse):
        assert torch.isnan(x[1:3]).all() and torch.isfinite(x[[0, 3]]).all()
    assert ((res.top_id[[0, 3]] >= 0) & (res.top_id[[0, 3]] < vocab)).all()
    check(z[[0, 3]], tok[[0, 3]], [x[[0, 3]] for x in res], 4)


@pytest.mark.parametrize("vocab,pad,shift", [(100, 3, 1), (5000, 8, 0), (5001, 7, 3), (40000, 5, 5)])
@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_strides_and_alignment(lm, typ, vocab, pad, shift):
    z, tok = make(vocab, typ, 6, vocab + pad + shift)
    z = z[:, shift:shift + vocab]
    tok = tok.clamp(max=vocab - 1)
    res = lm.mca_token_logprobs(z, tok, 9)
    check(z, tok, res, 9)
    g, ge = torch.randn(2, 6, device="cuda")
    for out in (None, torch.zeros(6, vocab + 2 * pad, dtype=z.dtype, device="cuda")[:, pad:pad + vocab]):
        got = lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, g, ge, out=out)
        check_grad(z, tok, res.lse, res.entropy, g, ge, got)


def test_large_logits_keep_precision(lm):
    z, tok = make(61, "f32", 3, 20000)
    z += 3.0e4
    check(z, tok, lm.mca_token_logprobs(z, tok, 3), 3)
    for vocab, at in ((100, 2.0 ** 20), (20000, -2.0 ** 20), (20000, 3e7)):  # around where the reference changes
        z, tok = make(63, "f32", 3, vocab)
        z = torch.round(z * 8) / 8 + at
        check(z, tok, lm.mca_token_logprobs(z, tok, 3), 3)
    for scale in (1e6, 1e30, 7e37):
        z, tok = make(62, "f32", 3, 20000, scale=scale)
        check(z, tok, lm.mca_token_logprobs(z, tok, 3), 3)


def check_grad(z, tok, lse, ent, g, ge, got):
    h = lambda x: x.float().cpu().numpy().astype(np.float64)  # noqa: E731
    n = len(z)
    gn = h(g) if g is not None else np.zeros(n)
    gen = h(ge) if ge is not None else np.zeros(n)
    zz, lz, en = h(z), h(lse), h(ent)
    want = olm.token_logprobs_grad(zz, tok.cpu().numpy(), lz, en, gn, gen)
    with np.errstate(invalid="ignore"):
        lp = np.where(np.isfinite(zz) & np.isfinite(lz)[:, None], zz - lz[:, None], -1e3)
    p = np.exp(lp)
    size = np.abs(gn)[:, None] + np.abs(gen)[:, None] * (np.abs(lp) + np.abs(en)[:, None] + 1)
    info = torch.finfo(got.dtype)
    tol = 2.0 ** -22 * (4 + np.abs(lp)) * p * size + info.eps / 2 * np.abs(want) * (1 + 2 ** -6) + info.smallest_normal * info.eps
    a = got.float().cpu().numpy().astype(np.float64)
    # p and its token's 1 - p are subtracted in 32 bits
    tol[np.arange(n), np.clip(tok.cpu().numpy(), 0, zz.shape[1] - 1)] += 2.0 ** -23 * np.abs(gn)
    bad = np.abs(a - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], a[bad][:3], want[bad][:3], tol[bad][:3])


@pytest.mark.parametrize("vocab", [1, 2, 65, 300, 511, 512, 513, 1500, 8192, 20011])
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_gradient(lm, typ, vocab):
    z, tok = make(vocab, typ, 7, vocab)
    res = lm.mca_token_logprobs(z, tok)
    g, ge = torch.randn(2, 7, device="cuda")
    for a, b in ((g, ge), (g, None), (None, ge), (None, None)):
        got = lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, a, b)
        check_grad(z, tok, res.lse, res.entropy, a, b, got)
    mine = z.clone()
    assert lm.mca_token_logprobs_grad(mine, tok, res.lse, res.entropy, g, ge, out=mine) is mine
    check_grad(z, tok, res.lse, res.entropy, g, ge, mine)


@pytest.mark.parametrize("vocab", [70, 5001])
@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_large_gradients_of_masked_symbols(lm, typ, vocab):
    """Symbols of probability 0 get 0, however large the gradient of the entropy is."""
    z, tok = make(vocab + 1, typ, 5, vocab)
    z[:, 3::2] = -float("inf")
    z[:, 2] = -3e4
    tok[:] = 0
    res = lm.mca_token_logprobs(z, tok)
    g, ge = torch.randn(2, 5, device="cuda")
    ge = ge * 1e12
    got = lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, g, ge)
    assert (got[:, 2:4] == 0).all()
    check_grad(z, tok, res.lse, res.entropy, g, ge, got)


def test_gradient_against_differences(lm):
    z, tok = make(5, "f32", 2, 1200)
    g, ge = torch.randn(2, 2, device="cuda")
    res = lm.mca_token_logprobs(z, tok)
    got = lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, g, ge)
    d = torch.randn_like(z)

    def f(y):
        r = lm.mca_token_logprobs(y, tok)
        return (g.double() * r.logprob.double() + ge.double() * r.entropy.double()).sum()

    # a step of 2^-6: second-order terms cancel, results are good to about 2^-20
    h = 2.0 ** -6
    diff = float((f(z + h * d) - f(z - h * d)) / (2 * h))
    assert abs(diff - float((got.double() * d.double()).sum())) <= 2e-3 * (1 + abs(diff))


def test_many_rows(lm):
    z, tok = make(9, "bf16", 70000, 600)
    res = lm.mca_token_logprobs(z, tok, 2)
    g = torch.randn(70000, device="cuda")
    got = lm.mca_token_logprobs_grad(z, tok, res.lse, res.entropy, g)
    at = torch.tensor([0, 1, 65534, 65535, 65536, 69999], device="cuda")
    check(z[at], tok[at], [x[at] for x in res], 2)
    check_grad(z[at], tok[at], res.lse[at], res.entropy[at], g[at], None, got[at])


def test_refusals(lm):
    from paper_2607_08406_amd.mca import MCAError
    z, tok = make(1, "bf16", 2, 300000)
    for bad in (lambda: lm.mca_token_logprobs(z, tok, 33), lambda: lm.mca_token_logprobs(z.T, tok[:1]),
                lambda: lm.mca_token_logprobs(z, tok.float()), lambda: lm.mca_token_logprobs(z, tok.cpu()),
                lambda: lm.mca_token_logprobs(z, tok[:1]), lambda: lm.mca_token_logprobs(z.double(), tok),
                lambda: lm.mca_token_logprobs(z, tok, 3, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
                lambda: lm.mca_token_logprobs_grad(z, tok, tok.float()[:1], tok.float(), tok.float()),
                lambda: lm.mca_token_logprobs_grad(z, tok, tok.float(), None, None, tok.float().int())):
        with pytest.raises(MCAError):
            bad()
