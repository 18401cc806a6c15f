"""The fp64 oracle of the language-model operators against closed forms, brute
force, differences and the Transformer oracle's causal attention."""
import numpy as np
import pytest

from oracle import lm
from oracle.transformer import causal_attention


def test_tree_attention_of_a_chain_is_causal_attention():
    rng = np.random.default_rng(1)
    T, heads, dim, block, cut = 11, 2, 8, 4, 6
    q, k, v = rng.normal(size=(3, T, heads, dim))
    want = causal_attention(*(x.reshape(1, T, -1) for x in (q, k, v)), heads)[0].reshape(T, heads, dim)
    table = np.array([[2, 0]])
    kc, vc = np.full((2, 3, heads, block, dim), np.nan)
    for t in range(cut):
        kc[table[0, t // block], :, t % block], vc[table[0, t // block], :, t % block] = k[t], v[t]
    got = lm.tree_attention(q[cut:], k[cut:], v[cut:], kc, vc, table, [cut], [0, T - cut], np.arange(T - cut) - 1,
                            dim ** -0.5)
    for i in range(T - cut):
        for h in range(heads):
            np.testing.assert_allclose(got[i, h][0], want[cut + i, h], rtol=1e-12)


def test_sees_is_the_ancestor_relation():
    up = [-1, 0, 0, 1, -1, 4, 7, 3]  # node 6 names a later one: it stands alone
    want = np.eye(8, dtype=bool)
    for i in range(8):
        j = i
        while 0 <= up[j] < j:
            j = up[j]
            want[i, j] = True
    assert (lm.sees(up) == want).all()


@pytest.mark.parametrize("masked", [False, True])
def test_logprobs_and_gradient(masked):
    rng = np.random.default_rng(2)
    z = rng.normal(size=(4, 9))
    if masked:
        z[:, 3] = -np.inf
    tok = np.array([0, 8, -1, 5])
    lp, ent, lse, logp = lm.token_logprobs(z, tok)
    p = np.exp(logp)
    np.testing.assert_allclose(p.sum(1), 1, rtol=1e-12)
    assert lp[2] == 0 and np.isclose(lp[3], logp[3, 5])
    g, ge = rng.normal(size=(2, 4))
    got = lm.token_logprobs_grad(z, tok, lse, ent, g, ge)

    def f(y):
        a, b, _, _ = lm.token_logprobs(y, tok)
        return (g * a + ge * b).sum()

    for t in range(4):
        for c in range(9):
            if z[t, c] == -np.inf:
                assert got[t, c] == 0
                continue
            d = np.zeros_like(z)
            d[t, c] = 1e-6
            np.testing.assert_allclose(got[t, c], (f(z + d) - f(z - d)) / 2e-6, atol=1e-8)


def test_logprobs_edges():
    lp, ent, lse, _ = lm.token_logprobs(np.full((1, 5), -np.inf), [2])
    assert lse[0] == -np.inf and ent[0] == 0 and lp[0] == -np.inf
    _, ent, lse, _ = lm.token_logprobs(np.zeros((1, 8)), [0])
    np.testing.assert_allclose([ent[0], lse[0]], np.log(8))
    assert (lm.top([[1.0, 3.0, 3.0, -np.inf]], 3) == [[1, 2, 0]]).all()


def test_block_tables_by_hand():
    table = np.array([[4, 1, 9], [0, 9, 9], [2, 9, 9]], np.int32)
    free = np.array([3, 5, 7, 7, 7, 7], np.int32)  # 6 blocks, 4 held: 2 free (3 and 5)
    # request 0 drops to 3 tokens (gives up block 1), 1 grows by 3 into two more blocks, 2 stays
    t, f, off, slots, st = lm.block_tables(np.array([7, 4, 3]), np.array([3, 9, 3]), table, free, 4, 6)
    assert list(t[1]) == [0, 1, 5] and list(t[0]) == [4, 1, 9]
    assert list(off) == [0, 0, 5, 5] and list(slots) == [4, 5, 6, 7, 20, -1]
    assert st == (0, 1, 5, 2) and list(f) == list(free)
    assert lm.block_tables(np.array([7, 4, 3]), np.array([12, 12, 3]), table, free, 4, 99)[4] == (1, 2, 0, 0)
    assert lm.block_tables(np.array([7, 4, 3]), np.array([7, 13, 3]), table, free, 4, 99)[4][0] == 2
    assert lm.block_tables(np.array([7, 4, 3]), np.array([8, 5, 3]), table, free, 4, 1)[4] == (3, 2, 0, 0)
