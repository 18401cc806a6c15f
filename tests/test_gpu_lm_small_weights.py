"""Attention of 16-bit values where nearly all weight lies on tokens whose values are 0
(a first token that every query attends to, as trained nets have it): the result is made
of weights far below the largest, which a 16-bit format must still hold.

Tolerance, beside that of 32-bit scores and sums and of one rounding of the result: a
weight is rounded once, half a step relative to itself, as long as its tile's largest is
within 2^-19 of the largest of a tile near it; a token that shares its tile (64 tokens)
with one at least 2^10 steps of fp16's smallest normal number larger may lose 2^-35 of
that one's weight, 2^-29 over a tile.  fp16 results below the normal range are off by
half of 2^-24.
"""
import numpy as np
import pytest
import torch

from oracle import lm as olm

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def make(typ, scores, nodes, group, dim, block=16, spread=0.0, seed=1):
    """One key head; scores[r] are request r's cached tokens' (those of 0 have values of 0), and a draft that is a
    chain sees itself at the lowest of them."""
    rng = np.random.default_rng(seed)
    dt = TYPES[typ]
    lens = [len(s) for s in scores]
    width = -(-max(lens) // block)
    held = [-(-n // block) for n in lens]
    pool = rng.permutation(sum(held) + 1)
    table = np.full((len(lens), width), -1, np.int32)
    kc, vc = (np.zeros((len(pool), 1, block, dim), np.float32) for _ in range(2))
    at = 0
    for r, s in enumerate(scores):
        table[r, :held[r]] = pool[at:at + held[r]]
        at += held[r]
        t = np.arange(lens[r])
        x = np.where(s == 0, 0, s + np.round(rng.uniform(-spread, spread, lens[r]) * 64) / 64)
        kc[table[r, t // block], 0, t % block, 0] = x
        vc[table[r, t // block], 0, t % block] = np.where((s == 0)[:, None], 0, rng.uniform(200, 500, (lens[r], dim)))
    T = nodes * len(lens)
    q, k, v = np.zeros((T, group, dim)), np.zeros((T, 1, dim)), rng.uniform(200, 500, (T, 1, dim))
    q[:, :, 0] = 1.0
    k[:, 0, 0] = np.repeat([min(s) for s in scores], nodes)
    put = lambda a, t=torch.int32: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()  # noqa: E731
    return dict(q=put(q, dt), k=put(k, dt), v=put(v, dt), k_cache=put(kc, dt), v_cache=put(vc, dt), table=put(table),
                lengths=put(lens), offsets=put(np.arange(len(lens) + 1) * nodes),
                parents=put(np.tile(np.arange(nodes) - 1, len(lens)))), nodes


def check(lm, s, nodes, max_len):
    out, lse = lm.mca_tree_attention(*s.values(), nodes, max_len=max_len, scale=1.0)
    h = {n: t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy() for n, t in s.items()}
    want = olm.tree_attention(*h.values(), 1.0)
    got, norms = out.double().cpu().numpy(), lse.cpu().numpy()
    eps = torch.finfo(out.dtype).eps / 2
    most = max(np.abs(h["v"]).max(), np.abs(h["v_cache"]).max())
    for (row, head), (o, norm, pv, _, size, L) in want.items():
        # one product a score, which is exact
        e32 = 16 * 2.0 ** -24 * (size + 1) + (L + 16) * 2.0 ** -24
        tol = eps * np.abs(o) * (1 + 2 ** -6) + (e32 + eps) * pv * (1 + 2 ** -6) + 2.0 ** -29 * most + 2.0 ** -25
        d = np.abs(got[row, head] - o)
        assert (d <= tol).all(), (row, head, float((d / np.abs(o)).max()), float((d / tol).max()))
        assert abs(norms[row, head] - norm) <= e32 + 2.0 ** -20 * (abs(norm) + 1)


GAPS = [9, 13, 15, 17, 20, 23]
# max_len, requests, nodes, query heads: the kernel of few rows in one and in several chunks, of many rows with work
# shared and not, of one group of 16 rows, and of eight waves
FORMS = {"few": (120, 1, 2, 2), "chunks": (8192, 1, 2, 4), "shared": (1 << 17, 2, 40, 1), "many": (2048, 300, 5, 8),
         "sixteen": (1 << 22, 1, 3, 4), "eight": (1 << 17, 2, 32, 7)}


@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("typ,dim", [("f16", 64), ("f16", 128), ("f16", 256), ("bf16", 64)])
def test_a_token_of_no_value_takes_the_weight(lm, typ, dim, form, gap):
    max_len, R, nodes, group = FORMS[form]
    some = 3 if R > 3 else R
    scores = [np.full(min(max_len, 1500) - 7 * r, -float(gap)) for r in range(some)]
    scores[0][0] = 0.0
    for s in scores[1:]:
        s[len(s) // 2] = 0.0
    scores += [np.full(1, -1.0)] * (R - some)
    s, n = make(typ, scores, nodes, group, dim)
    if some < R:  # only the first requests have nodes
        s["offsets"][some + 1:] = some * nodes
        s = {k: v[:some * nodes] if k in ("q", "k", "v", "parents") else v for k, v in s.items()}
    check(lm, s, n, max_len)


@pytest.mark.parametrize("form", ["few", "chunks", "shared", "eight"])
@pytest.mark.parametrize("steps", [(0, -18, 0, -18, 0), (-24, -12, 0, -12, -24), (-30, -20, -10, 0), (0, -10, -20, -30)])
def test_levels_rise_and_fall(lm, form, steps):
    """Stretches of tokens at several levels, those at 0 without values."""
    max_len, R, nodes, group = FORMS[form]
    scores = [np.repeat(np.array(steps, np.float64), min(max_len, 2000) // len(steps)) for _ in range(R)]
    s, n = make("f16", scores, nodes, group, 64, spread=0.25)
    check(lm, s, n, max_len)


def test_many_tokens_far_below(lm):
    """60000 tokens 20 below the first one: together 1.2e-4 of its weight, and all of the result."""
    scores = [np.full(60000, -20.0)]
    scores[0][0] = 0.0
    for nodes, group in ((1, 4), (24, 2)):
        s, n = make("f16", scores, nodes, group, 64)
        check(lm, s, n, 60000)


def test_levels_too_far_apart_to_matter(lm):
    """Differences beyond every format: neither infinite nor NaN, and the rows that follow are right again."""
    scores = [np.concatenate([[0.0], np.full(700, -400.0)]), np.concatenate([np.full(700, -400.0), [0.0]]),
              np.tile(np.concatenate([np.full(64, -1000.0), np.full(64, 1000.0)]), 5)]
    s, n = make("f16", scores, 2, 2, 64)
    for max_len in (1408, 1 << 17):
        check(lm, s, n, max_len)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("form", ["few", "chunks", "shared", "eight"])
def test_a_single_token_is_exact(lm, typ, form):
    """All weight lies on one token, whatever its score: nodes that see themselves alone, and cached tokens 40 above
    the others.  The result is its value to the last bit (a weight of one power of two, and 2^-22 of its sum)."""
    max_len, R, nodes, group = FORMS[form]
    dim, dt, block = 64, TYPES[typ], 16
    rng = np.random.default_rng(nodes)
    n = min(max_len, 1200)
    width = -(-n // block)
    put = lambda a, t=torch.int32: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()  # noqa: E731
    T = 2 * nodes
    q, k, v = rng.normal(size=(T, group, dim)), rng.normal(size=(T, 1, dim)), rng.normal(size=(T, 1, dim))
    kc, vc = np.zeros((width, 1, block, dim)), rng.normal(size=(width, 1, block, dim))
    at = n // 3
    q[nodes:, :, 0], q[nodes:, :, 1:], k[nodes:, 0, 0] = 1.0, 0, -3.0
    kc[at // block, 0, at % block, 0] = 40.28125
    out, _ = lm.mca_tree_attention(put(q, dt), put(k, dt), put(v, dt), put(kc, dt), put(vc, dt),
                                   put(np.tile(np.arange(width), (2, 1))), put([0, n]), put([0, nodes, T]), put(np.full(T, -1)),
                                   nodes, max_len=max_len, scale=1.0)
    assert torch.equal(out[:nodes], put(v, dt)[:nodes].expand(nodes, group, dim))
    assert torch.equal(out[nodes:], put(vc, dt)[at // block, 0, at % block].expand(nodes, group, dim))
