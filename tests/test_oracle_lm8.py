"""The fp64 oracle of the 8-bit cache, the verification of drafts and distillation
against torch's own 8-bit floats, exhaustive expectations and autograd."""
import numpy as np
import pytest
import torch

from oracle import lm


def test_e4m3_is_torchs():
    code = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(code).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(lm.e4m3_value(code), want)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=5000) * 100, rng.normal(size=5000) * 0.01, np.arange(-448 * 16, 448 * 16 + 1) / 16,
                        np.arange(-2048, 2049) / 2.0 ** 16, [0.0, -0.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(lm.e4m3_code(lm.e4m3(x)), want)


def test_append_and_read_of_a_block():
    """Values come back within half a step of e4m3, whole blocks and token by token."""
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(2, 11, 2, 16)).astype(np.float32)
    empty = np.zeros((4, 2, 4, 16), np.uint8), np.zeros((4, 2), np.uint8)
    table = np.array([[2, 0, 3]])
    kc, vc, ks, vs = lm.cache8_append(k, v, empty[0], empty[0], empty[1], empty[1], table, [0], [0, 11], None, "f32")
    got = lm.cache8_read(lm.cache8_values(kc, ks), table, [0], [0, 11], np.zeros((11, 2, 16)))
    assert (np.abs(got - k) <= np.maximum(np.abs(k) / 16, np.abs(k).max() * 2.0 ** -10 / 224)).all()
    one = empty[0], empty[0], empty[1], empty[1]
    for t in range(11):
        one = lm.cache8_append(k[t:t + 1], v[t:t + 1], *one, table, [t], [0, 1], None, "f32")
    assert (one[2][table[0]] == ks[table[0]]).all()
    assert (np.abs(lm.cache8_values(one[0], one[2]) - lm.cache8_values(kc, ks)) <= np.abs(k).max() * 2.0 ** -9 / 224).all()
    assert lm.cache8_exp(448.0, "f32") == 0 and lm.cache8_exp(449.0, "f32") == 1 and lm.cache8_exp(0.0, "f16") == -15


@pytest.mark.parametrize("mode,kids", [("draft", 1), ("draft", 2), ("given", 2)])
def test_the_token_behind_the_root_is_the_targets(mode, kids):
    """Its distribution over a fine grid of random numbers and all drafts is p."""
    V, G = 3, 24
    p, q = np.array([0.5, 0.3, 0.2]), np.array([0.2, 0.2, 0.6])
    drafts = [(0, 2)] if mode == "given" else [t for t in np.ndindex(*[V] * kids)]
    seen = np.zeros(V)
    n = 1 + kids
    rows = np.tile(np.log(p), (n, 1))
    dr = np.tile(np.log(q), (n, 1)) if mode == "draft" else None
    grid = (np.arange(G) + 0.5) / G
    for toks in drafts:
        weight = 1.0 if mode == "given" else np.prod(q[list(toks)])
        for us in np.ndindex(*[G] * kids):
            # the random number of the draw matters only by its quantiles: its mean over a grid
            accept = np.concatenate([[0.0], grid[list(us)]])
            for w in grid[::4]:
                new, path, tok, _, _ = lm.verify_drafts(rows, dr, np.array([0, *toks]), np.array([-1] + [0] * kids), [0, n], [0], accept,
                                                     [w], 1.0, 1.0, False, n)
                first = toks[path[1] - 1] if new[0] > 1 else tok[0]
                seen[first] += weight
    np.testing.assert_allclose(seen / seen.sum(), p, atol=0.06)  # the grids' steps: 1 / 24 and 1 / 6 of what is drawn


def test_greedy_and_paths():
    z = np.zeros((5, 4))
    z[0, 2], z[1, 1], z[3, 3] = 1, 1, 1
    # node 0 has children 1 (token 0), 2 (token 2), 3 (token 2); node 2 has child 4
    new, rows, tok, _, _ = lm.verify_drafts(z, None, np.array([9, 0, 2, 2, 0]), np.array([-1, 0, 0, 0, 2]), [0, 5], [7], None, None, 1, 1,
                                         True, 6)
    assert new[0] == 10 and rows.tolist() == [0, 2, 4, -1, -1, -1] and tok[0] == 0


@pytest.mark.parametrize("rest,scale", [(False, 0.5), (False, 1.0), (True, 1.0)])
def test_distillation_against_autograd(rest, scale):
    rng = np.random.default_rng(3)
    z, t = rng.normal(size=(2, 4, 12)) * 2
    ids = np.argsort(-t, 1)[:, :5]
    t = t - np.log(np.exp(t).sum(1, keepdims=True))
    logp = np.take_along_axis(t, ids, 1)
    loss, lse, lrest, d = lm.distill(z, logp, ids, scale, rest)
    x = torch.tensor(z, requires_grad=True)
    s = torch.log_softmax(x * scale, 1)
    i = torch.tensor(ids)
    lp = torch.tensor(logp)
    if rest:
        q = lp.exp()
        out = torch.ones(4, 12, dtype=torch.float64).scatter(1, i, 0.0)
        left = 1 - q.sum(1)
        want = (q * (lp - s.gather(1, i))).sum(1) + left * (left.log() - (s.exp() * out).sum(1).log())
    else:
        lq = torch.log_softmax(lp * scale, 1)
        want = (lq.exp() * (lq - s.gather(1, i))).sum(1)
    want.sum().backward()
    np.testing.assert_allclose(loss, want.detach().numpy(), rtol=1e-10)
    np.testing.assert_allclose(d, x.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose(lse, torch.logsumexp(x.detach() * scale, 1).numpy(), rtol=1e-12)
