"""mca_distill and mca_distill_grad against the fp64 oracle, autograd and differences.

Bounds, u = 2^-24: an exponential of 32 bits is off by (2 + |exponent|) u (its argument
is rounded once, its result once), a sum of n of them in parts of at most n / 64
terms by (n / 64 + 8) u more; lse and lse_rest are off by that and half a step of their
own.  The loss is sum q (log q - scale z + lse) with the teacher's part in 64 bits: off by
that of lse (and of lse_rest times q_r) and half a step of its own.  The gradient is
g (Q s - q) rounded to the logits' type: s relative by u (3 + 2 |scale z - lse| + |lse|).
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


def make(seed, typ, rows, vocab, top, rest, scale=1.0, pad=0, size=3.0, noise=0.7):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(rows, vocab + pad)) * size
    t = z[:, :vocab] + rng.normal(size=(rows, vocab)) * noise
    t = t - t.max(1, keepdims=True)
    t = t - np.log(np.exp(t).sum(1, keepdims=True))
    ids = np.argsort(-t, 1)[:, :top]
    logp = np.take_along_axis(t, ids, 1)
    return dict(logits=torch.from_numpy(z).to(TYPES[typ]).cuda()[:, :vocab], logprob=put(logp, np.float32), ids=put(ids), rest=rest,
                scale=scale)


def check(lm, s, g=None, out=None):
    z = host(s["logits"]).astype(np.float64)
    T, V = z.shape
    sc = float(np.float32(s["scale"]))
    loss, lse, lrest, d = olm.distill(z, host(s["logprob"]), host(s["ids"]), sc, s["rest"])
    got = lm.mca_distill(**s)
    g = torch.linspace(-1.0, 2.0, T, device="cuda") if g is None else g
    grad = lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], got.lse, got.lse_rest, g, s["rest"], s["scale"], out=out)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.where(np.isfinite(z), np.abs(z), 0).max(1) * sc
        e = (V / 64 + 10 + 2 * 88) * U  # exponents below -88 weigh nothing
        for name, a, w, lim in (("lse", got.lse, lse, e + 2 * U * np.abs(lse) + 2 * U * top), ) + \
                ((("lse_rest", got.lse_rest, lrest, e + 2 * U * np.abs(lrest) + 2 * U * top),) if s["rest"] else ()) + \
                (("loss", got.loss, loss, 2 * e + 2 * U * np.abs(loss) + 4 * U * top),):
            a = host(a).astype(np.float64)
            same = (a == w) | (np.isnan(a) & np.isnan(w))
            bad = ~same & ~(np.abs(a - w) <= lim)
            assert not bad.any(), (name, np.nonzero(bad)[0][:5], a[bad][:5], w[bad][:5], lim[bad][:5])
        want = d * host(g).astype(np.float64)[:, None]
        p = np.where(np.isfinite(want), np.exp(z * sc - lse[:, None]), 0)
        eps = torch.finfo(s["logits"].dtype).eps / 2
        tiny = torch.finfo(s["logits"].dtype).smallest_normal * eps
        # (with rest the others' are two terms, s_v and q_r exp(scale z - lse_rest), q_r at most 1)
        other = np.zeros(z.shape)
        if s["rest"]:
            other = np.where(np.isfinite(want), np.exp(np.minimum(z * sc - lrest[:, None], 0)), 0)
            for t, i in np.argwhere((host(s["ids"]) >= 0) & (host(s["ids"]) < V)):
                other[t, host(s["ids"])[t, i]] = 0
        rel = 3 * U * (4 + 2 * np.minimum(np.abs(z * sc - lse[:, None]), 200) + np.abs(lse)[:, None] + top[:, None]) + 2 * e
        size = np.abs(host(g))[:, None] * sc * (2 * p + other + 4 * U)
        q = np.abs(want) + size
        a = host(grad).astype(np.float64)
        same = (a == want) | (np.isnan(a) & np.isnan(want))
        bad = ~same & ~(np.abs(a - want) <= eps * np.abs(want) * (1 + 2 ** -6) + rel * size + 2 * U * q + 2 * tiny)
        assert not bad.any(), (np.argwhere(bad)[:5], a[bad][:5], want[bad][:5])
    return got, grad


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("rows,vocab,top,rest,scale", [
    (9, 65, 5, False, 0.5), (9, 65, 5, True, 1.0), (3, 1, 1, False, 1.0), (3, 1, 1, True, 1.0), (5, 32, 32, True, 1.0), (6, 200, 32, True, 1.0),
    (4, 500, 7, False, 2.0), (7, 1000, 20, True, 1.0), (5, 1025, 1, True, 1.0), (3, 1030, 32, False, 0.25), (6, 5003, 20, True, 1.0),
    (2, 50001, 20, True, 1.0), (1, 128000, 32, False, 1.0), (3, 40000, 8, True, 1.0)])
def test_distill(lm, typ, rows, vocab, top, rest, scale):
    check(lm, make(rows + vocab, typ, rows, vocab, top, rest, scale))


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("vocab", [100, 3001, 20000])
def test_rows_apart(lm, typ, vocab, pad):
    """Strides beyond the vocabulary; gradients that are new, that lie as the logits do, and in their place."""
    s = make(3, typ, 5, vocab, 9, True, pad=pad)
    _, a = check(lm, s)
    whole = torch.full((5, vocab + pad), 7.0, device="cuda", dtype=s["logits"].dtype)
    _, b = check(lm, s, out=whole[:, :vocab])
    assert torch.equal(a, b) and (whole[:, vocab:] == 7).all()
    got = lm.mca_distill(**s)
    g = torch.linspace(-1.0, 2.0, 5, device="cuda")
    lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], got.lse, got.lse_rest, g, True, 1.0, out=s["logits"])
    assert torch.equal(s["logits"], a)


@pytest.mark.parametrize("vocab", [70, 2000, 30000])
@pytest.mark.parametrize("rest", [False, True])
def test_symbols_that_are_none_and_twice(lm, vocab, rest):
    s = make(5, "f32", 8, vocab, 6, rest)
    ids, logp = host(s["ids"]), host(s["logprob"])
    ids[0] = -1
    ids[1, 2:] = vocab
    ids[2, 0] = 2 ** 31 - 1
    ids[3, 1] = ids[3, 0]
    ids[3, 5] = ids[3, 0]
    logp[3] -= 1.0
    logp[4, 3] = -np.inf
    logp[5] = -np.inf
    ids[6] = ids[6, ::-1]  # any order
    s.update(ids=put(ids), logprob=put(logp, np.float32))
    got, grad = check(lm, s)
    assert got.loss[0] == 0 and (grad[0] == 0).all()


@pytest.mark.parametrize("vocab", [70, 2000, 30000])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("typ", TYPES)
def test_masked_and_undefined(lm, typ, vocab, rest):
    """-inf at symbols, at the teacher's, at all others, everywhere; NaN, infinities, the type's lowest value; teachers of
    NaN and +inf."""
    s = make(6, typ, 12, vocab, 4, rest)
    z = s["logits"].clone()
    ids, logp = host(s["ids"]), host(s["logprob"])
    inf = float("inf")
    z[0, 1::3] = -inf
    z[1, ids[1, 2]] = -inf
    keep = z[2, put(ids[2]).long()].clone()
    z[2] = -inf
    z[2, put(ids[2]).long()] = keep
    z[3] = -inf
    z[4, 5], z[5, 5] = float("nan"), inf
    z[6] = torch.finfo(z.dtype).min
    logp[7, 1], logp[8, 1] = np.nan, inf
    z[9, ids[9, 1]], ids[9] = float("nan"), -1
    logp[10] += 0.5  # more than all probability
    z[11] *= 100
    s.update(logits=z, ids=put(ids), logprob=put(logp, np.float32))
    check(lm, s)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("rows,vocab,top,rest", [(1030, 513, 5, True), (1101, 1000, 20, False), (1024, 767, 3, True), (3, 65537, 20, True), (5, 100003, 32, True)])
def test_where_the_kernels_change(lm, typ, rows, vocab, top, rest):
    """Short rows while they are many, and long ones in parts while they are few."""
    check(lm, make(rows, typ, rows, vocab, top, rest))


@pytest.mark.parametrize("typ", TYPES)
def test_rows_in_parts(lm, typ):
    test_symbols_that_are_none_and_twice(lm, 70000, True)
    test_masked_and_undefined(lm, typ, 70000, True)
    test_masked_and_undefined(lm, typ, 70000, False)


def test_the_teachers_symbols_have_nearly_all_weight(lm):
    """The others' probability is 1e-12 and less: its logarithm is as exact as ever."""
    for vocab in (90, 5000, 40000):
        s = make(7, "f32", 6, vocab, 3, True)
        z = s["logits"]
        z.scatter_(1, s["ids"].long(), z.gather(1, s["ids"].long()) + 30)
        check(lm, s)


def test_gradient_against_differences(lm):
    """Central differences of the 64-bit loss, and autograd of its definition."""
    for rest, scale in ((True, 1.0), (False, 0.5)):
        s = make(8, "f32", 3, 40, 5, rest, scale, size=1.0)
        got = lm.mca_distill(**s)
        grad = lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], got.lse, got.lse_rest, torch.ones(3, device="cuda"), rest, scale)
        z = host(s["logits"]).astype(np.float64)
        num = np.zeros(z.shape)
        for i in range(40):
            for sign in (1, -1):
                x = z.copy()
                x[:, i] += sign * 1e-5
                num[:, i] += sign * olm.distill(x, host(s["logprob"]), host(s["ids"]), scale, rest)[0] / 2e-5
        assert np.abs(host(grad) - num).max() < 1e-6  # h^2 / 6 of the third derivative (1e-10), 1e-16 / h, and the 32-bit result


def test_a_function_of_autograd_around_the_calls(lm):
    class Distil(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z, logprob, ids):
            r = lm.mca_distill(z, logprob, ids, rest=True)
            ctx.save_for_backward(z, logprob, ids, r.lse, r.lse_rest)
            return r.loss

        @staticmethod
        def backward(ctx, g):
            return lm.mca_distill_grad(*ctx.saved_tensors, g.contiguous(), rest=True), None, None

    teacher = torch.randn(7, 90, device="cuda")
    t = lm.mca_token_logprobs(teacher, put([0] * 7), n_top=10)
    x = torch.randn(7, 90, device="cuda", requires_grad=True)
    Distil.apply(x, t.top_logprob, t.top_id).sum().backward()
    y = x.detach().double().requires_grad_()
    s = torch.log_softmax(y, 1)
    q = t.top_logprob.double().exp()
    left = 1 - q.sum(1)
    other = torch.ones_like(y).scatter(1, t.top_id.long(), 0.0)
    loss = (q * (t.top_logprob.double() - s.gather(1, t.top_id.long()))).sum(1) + left * (left.log() - (s.exp() * other).sum(1).log())
    loss.sum().backward()
    # probabilities of at most 1, off by some 32-bit steps of the exponents (at most 16)
    assert (x.grad.double() - y.grad).abs().max() <= 2.0 ** -18


def test_captured(lm):
    s = make(9, "bf16", 40, 20000, 8, True)
    g = torch.rand(40, device="cuda")
    def call():
        r = lm.mca_distill(**s)
        return r, lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], r.lse, r.lse_rest, g, True)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, grad = call()
    for i in range(3):
        s["logits"].normal_(std=1.0 + i)
        s["ids"].copy_(torch.argsort(torch.rand(40, 20000, device="cuda"), 1)[:, :8].to(torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        a, b = call()
        assert torch.equal(a.loss, got.loss) and torch.equal(grad, b)


def test_no_rows(lm):
    z = torch.zeros(0, 10, device="cuda")
    e = torch.zeros(0, 3, device="cuda")
    r = lm.mca_distill(z, e, e.int())
    assert r.loss.numel() == 0
    assert lm.mca_distill_grad(z, e, e.int(), r.lse, None, r.loss).shape == z.shape


def test_many_rows(lm):
    """More rows than a grid's second dimension has, in both directions."""
    s = make(10, "bf16", 66000, 520, 2, False, size=1.0)
    z = s["logits"].double()
    got = lm.mca_distill(**s)
    assert (got.lse.double() - torch.logsumexp(z, 1)).abs().max() < 1e-5
    g = torch.ones(66000, device="cuda")
    grad = lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], got.lse, None, g)
    q = torch.softmax(s["logprob"].double(), 1)
    want = torch.softmax(z, 1).scatter_add(1, s["ids"].long(), -q)
    assert ((grad.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all()


def test_many_longer_rows(lm):
    """The same of the kernels that take a row by vectors."""
    s = make(11, "bf16", 66000, 1032, 2, True, size=1.0)
    z = s["logits"].double()
    got = lm.mca_distill(**s)
    assert (got.lse.double() - torch.logsumexp(z, 1)).abs().max() < 1e-5
    g = torch.ones(66000, device="cuda")
    grad = lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], got.lse, got.lse_rest, g, True)
    q, p, ids = s["logprob"].double().exp(), torch.softmax(z, 1), s["ids"].long()
    other = (1 - q.sum(1, keepdim=True)).clamp(min=0)
    rest = 1 - p.gather(1, ids).sum(1, keepdim=True)
    want = (p - other * p / rest).scatter(1, ids, p.gather(1, ids) - q)
    assert ((grad.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all()


def test_more_rows_than_threads_of_a_grid(lm):
    """2^32 / 320 rows and some."""
    n, v = 13_421_773 + 5, 1025
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("28 GB of logits")
    z = torch.zeros(n, v, device="cuda", dtype=torch.bfloat16)
    z[-1, 3] = z[1 << 23, 3] = 2.0
    logp, ids = torch.zeros(n, 1, device="cuda"), torch.full((n, 1), 3, device="cuda", dtype=torch.int32)
    got = lm.mca_distill(z, logp, ids)
    few = lm.mca_distill(z[-2:], logp[-2:], ids[-2:])
    at = torch.tensor([0, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, n - 2, n - 1], device="cuda")
    assert torch.equal(got.loss[at], few.loss[torch.tensor([0, 0, 1, 0, 0, 1], device="cuda")])
    assert int((got.loss != few.loss[0]).sum()) == 2 and int((got.lse != few.lse[0]).sum()) == 2
