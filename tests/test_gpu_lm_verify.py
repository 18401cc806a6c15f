"""mca_verify_drafts against the fp64 oracle: the accepted paths, their rows, the tokens.

All outputs are whole numbers and have to be equal.  A decision can differ only where
it lies closer to its border than the arithmetic resolves.  Where a child is tried these
are sums of 32-bit exponentials, which are off by (2 + |exponent|) 2^-24 each and by
another 2^-24 for each of a lane's terms: below 2^-16 of the sum at the sizes here, as
exponents of more than 30 weigh nothing.  Where a token is drawn they are sums of V 64-bit
ones, each off by 2^-47, and c is a sum of such sums: below 2^-40.  The seeds' margins, which the oracle gives, are
asserted to be wider.
"""
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


def make(seed, typ, nodes, vocab, width=1, mode="draft", pad=0, chain=None, noise=0.6, scale=0.9, draft_scale=1.1):
    """Requests of so many nodes; a node's token is drawn from the draft's distribution at its parent."""
    rng = np.random.default_rng(seed)
    nodes = np.array(nodes)
    first = np.concatenate([[0], np.cumsum(nodes)])
    T = int(first[-1]) + 2
    dt = TYPES[typ]
    parents = np.full(T, -1)
    for a, n in zip(first, nodes):
        for i in range(1, n):
            parents[a + i] = i - 1 if chain else (rng.integers(0, i) if width == 0 else (i - 1) // width)
    draft = rng.normal(size=(T, vocab + pad)) * 3
    target = draft + rng.normal(size=draft.shape) * noise
    draft, target = (torch.from_numpy(x).to(dt).cuda()[:, :vocab] for x in (draft, target))
    tokens = rng.integers(0, vocab, T)
    z = host(target if mode == "greedy" else draft).astype(np.float64)
    for r, a in enumerate(first[:-1]):
        for i in range(1, nodes[r]):
            if parents[a + i] >= 0:
                row = z[a + parents[a + i]] * draft_scale
                p = np.exp(row - row.max())
                tokens[a + i] = np.argmax(row) if mode == "greedy" and rng.random() < 0.7 else rng.choice(vocab, p=p / p.sum())
    return dict(target=target, draft=draft if mode == "draft" else None, tokens=put(tokens), parents=put(parents), offsets=put(first),
                lengths=put(rng.integers(0, 100, len(nodes))), max_nodes=max(1, int(nodes.max())),
                accept=put(rng.random(T), np.float32), sample=put(rng.random(len(nodes)), np.float32), scale=scale,
                draft_scale=draft_scale, greedy=mode == "greedy")


def expected(s):
    h = {n: host(t) if isinstance(t, torch.Tensor) else t for n, t in s.items()}
    return olm.verify_drafts(h["target"], h["draft"], h["tokens"], h["parents"], h["offsets"], h["lengths"], h["accept"], h["sample"],
                             h["scale"], h["draft_scale"], h["greedy"], len(h["tokens"]))


def check(lm, s, got=None, margins=(2.0 ** -16, 2.0 ** -40)):
    want = expected(s)
    assert s["greedy"] or (want[3] > margins[0] and want[4] > margins[1]), want[3:]
    got = lm.mca_verify_drafts(**s) if got is None else got
    for name, g, w in zip(got._fields, got, want):
        np.testing.assert_array_equal(host(g), w, err_msg=name)
    return want


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("mode", ["draft", "given", "greedy"])
@pytest.mark.parametrize("vocab,nodes,width", [(65, [5] * 30 + [1, 4, 3], 1), (300, [9, 1, 16, 7, 12], 2), (1, [3, 2], 1),
                                               (1001, [40, 128, 3], 3), (50, [60, 100, 9], 0), (20011, [9, 4, 6, 5], 2)])
def test_verify(lm, typ, mode, vocab, nodes, width):
    got = 0
    for seed in range(3):
        s = make(seed, typ, nodes, vocab, width, mode)
        # margins of given drafts of one symbol are 0: nothing is left of it
        want = check(lm, s, margins=(-1, -1)) if vocab == 1 else check(lm, s)
        got += int((want[0] - host(s["lengths"]) > 1).sum())
    assert got > 0 or vocab == 1 or mode == "given"  # a given symbol among 20011 is seldom accepted


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("mode", ["draft", "given"])
@pytest.mark.parametrize("vocab", [400, 9000, 40001])
def test_many_rejections_at_a_node(lm, typ, mode, vocab):
    """One to nine children, all or nearly all of which are rejected: the token is drawn from what all of them leave."""
    lost = 0
    for kids in (1, 2, 3, 4, 5, 9):
        s = make(kids, typ, [kids + 1] * 8, vocab, kids, mode, noise=0.4)
        s["accept"].uniform_(0.9, 1.0, generator=torch.Generator("cuda").manual_seed(kids))
        want = check(lm, s)
        lost += int((want[0] - host(s["lengths"]) == 1).sum())
    assert lost > 6


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("vocab", [3, 5, 7, 8, 9, 15, 33, 8191, 8193, 8200, 32767, 32775, 65537])
def test_sums_at_the_ends_of_rows(lm, typ, vocab):
    """Vocabularies about the vectors, workgroups and rounds of the sums that rejections need."""
    for kids in (2, 4):
        s = make(100 + kids, typ, [kids + 1] * 6 + [2 * kids + 1] * 2, vocab, kids, "draft", noise=0.5)
        s["accept"].uniform_(0.7, 1.0, generator=torch.Generator("cuda").manual_seed(kids))
        check(lm, s)


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_rows_apart(lm, typ, pad):
    """Strides beyond the vocabulary, target's and draft's rows aligned differently."""
    s = make(1, typ, [7, 9, 3], 999, 2, pad=pad)
    s["draft"] = s["draft"].contiguous()
    check(lm, s)


def test_distribution(lm):
    """Path and token are distributed as if drawn one by one: the first token behind the root over 40000 requests
    against the target, by chi squared, for drawn and given drafts, one child and three."""
    V, R = 7, 40000
    rng = np.random.default_rng(5)
    z, d = rng.normal(size=V) * 1.2, rng.normal(size=V) * 1.2
    p, q = (np.exp(x) / np.exp(x).sum() for x in (z, d))
    for mode, kids in (("draft", 1), ("draft", 3), ("given", 2)):
        n = 1 + kids
        T = R * n
        tokens = np.zeros((R, n), int)
        tokens[:, 1:] = rng.choice(V, size=(R, kids), p=q) if mode == "draft" else [2, 5]
        parents = np.tile([-1] + [0] * kids, R)
        rows = torch.from_numpy(z).float().cuda().expand(T, V).contiguous()
        drafts = torch.from_numpy(d).float().cuda().expand(T, V).contiguous()
        got = lm.mca_verify_drafts(rows, drafts if mode == "draft" else None, put(tokens.reshape(-1)), put(parents),
                                   put(np.arange(R + 1) * n), put(np.zeros(R)), n, put(rng.random(T), np.float32),
                                   put(rng.random(R), np.float32))
        count, path, token = host(got.new_len), host(got.rows), host(got.token)
        ends = np.cumsum(count)
        first = np.where(count > 1, tokens.reshape(-1)[path[np.minimum(ends - count + 1, T - 1)]], token)
        seen = np.bincount(first, minlength=V)
        chi = ((seen - R * p) ** 2 / (R * p)).sum()
        assert chi < 30, (mode, kids, chi)  # 6 degrees of freedom: 4e-5
        assert 0 < (count > 1).sum() < R


@pytest.mark.parametrize("mode", ["draft", "given", "greedy"])
def test_rows_without_a_softmax(lm, mode):
    """NaN, +inf and nothing but -inf in the target end a path without a token; in the draft only where there are
    children; masked symbols are never drawn; children outside the vocabulary are passed over."""
    s = make(2, "f32", [3] * 12, 130, 1, mode, noise=0.0, scale=1.0, draft_scale=1.0)
    z = s["target"].clone()
    nan, inf = float("nan"), float("inf")
    first = host(s["offsets"])
    z[first[0], 7], z[first[1], 7], z[first[2]] = nan, inf, -inf
    z[first[3] + 1, 100] = nan
    z[first[4], 1:] = -inf
    z[first[5]] = torch.finfo(torch.float32).min
    z[first[6], 5] = -inf
    if mode == "draft":
        d = s["draft"].clone()
        d[first[7], 3], d[first[8]] = nan, -inf
        d[first[9] + 2] = nan  # a leaf's
        d[first[6], 5] = -inf
        s["draft"] = d
    tok = host(s["tokens"])
    tok[first[10] + 1], tok[first[11] + 1] = -1, 130
    tok[first[6] + 1] = 5  # a symbol that has no probability
    s.update(target=z, tokens=put(tok))
    want = check(lm, s, margins=(-1, -1))
    assert (want[2][[0, 1, 2]] == -1).all() and want[2][5] >= 0


def test_random_numbers_at_their_ends(lm):
    """accept 0 takes whatever has a probability, 1 nothing that the target likes less; sample 0 and 1, NaN, and out of
    range."""
    for u, w in ((0.0, 0.0), (1.0, 1.0), (1.0 - 2.0 ** -24, 1.0 - 2.0 ** -24), (float("nan"), float("nan")), (-1.0, 5.0)):
        s = make(4, "f32", [4] * 9, 77, 1)
        s["accept"].fill_(u)
        s["sample"].fill_(w)
        want = expected({**s, "sample": torch.nan_to_num(s["sample"])})
        got = lm.mca_verify_drafts(**s)
        for g, x in zip(got, want):
            np.testing.assert_array_equal(host(g), x)


def test_the_draft_is_the_target(lm):
    """Equal logits: every child is accepted (accept < 1), nothing is ever left to draw from a residual."""
    s = make(6, "bf16", [9] * 20, 5000, 1, noise=0.0, scale=1.0, draft_scale=1.0)
    got = lm.mca_verify_drafts(**s)
    assert (host(got.new_len) - host(s["lengths"]) == 9).all() and (host(got.token) >= 0).all()


def test_nothing_left_is_drawn_from_the_target(lm):
    """Rejected by accept = 1 although both agree: the token comes from p itself."""
    s = make(6, "f32", [2] * 30, 3000, 1, noise=0.0, scale=1.0, draft_scale=1.0)
    s["accept"].fill_(1.0)
    got = lm.mca_verify_drafts(**s)
    z = host(s["target"]).astype(np.float64)[host(s["offsets"])[:-1]]
    p = np.exp(z - z.max(1, keepdims=True))
    ends = np.cumsum(p, 1)
    want = (ends <= host(s["sample"]).astype(np.float64)[:, None] * ends[:, -1:]).sum(1)
    assert (host(got.new_len) - host(s["lengths"]) == 1).all()
    # (borders of two sums in 64 bits)
    assert (host(got.token) == want).mean() > 0.9 and (host(got.token) >= 0).all()


def test_offsets_and_parents_out_of_range(lm):
    """Requests without nodes, of too many, of offsets that pass the rows: no token, lengths as they were.  Parents
    behind their node or none: not reached."""
    s = make(7, "bf16", [3, 4, 6, 3, 2], 90, 1, "given")
    n = len(s["tokens"])
    par = host(s["parents"])
    par[1], par[4], par[5] = 2, -9, 4
    s["parents"] = put(par)
    s["offsets"] = put([0, 3, 7, 7, 13, n + 1])
    s["max_nodes"] = 5
    want = expected(s)
    got = lm.mca_verify_drafts(**s)
    lens = host(s["lengths"])
    assert (host(got.new_len)[2:] == lens[2:]).all() and (host(got.token)[2:] == -1).all()
    k = int((want[0][:2] - lens[:2]).sum())
    assert (host(got.new_len)[:2] == want[0][:2]).all() and (host(got.token)[:2] == want[2][:2]).all()
    assert (host(got.rows)[:k] == want[1][:k]).all() and (host(got.rows)[k:] == -1).all()


def test_no_requests_and_no_rows(lm):
    z = torch.zeros(3, 10, device="cuda")
    e = put([])
    got = lm.mca_verify_drafts(z, None, put([0] * 3), put([-1] * 3), put([0]), e, 1, put([0] * 3, np.float32), put([], np.float32))
    assert (host(got.rows) == -1).all() and got.token.numel() == 0
    got = lm.mca_verify_drafts(z[:0], None, e, e, put([0, 0, 0]), put([4, 5]), 1, put([], np.float32), put([0, 0], np.float32))
    assert (host(got.new_len) == [4, 5]).all() and (host(got.token) == -1).all()


def test_captured(lm):
    """Replays with other logits and random numbers; two graphs of a workspace each."""
    s = make(8, "bf16", [6] * 9, 20000, 2)
    torch.manual_seed(5)
    graphs = []
    for _ in range(2):
        lm.mca_verify_drafts(**s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = lm.mca_verify_drafts(**s)
        graphs.append((g, got))
    for i in range(3):
        s["accept"].uniform_()
        s["sample"].uniform_()
        s["target"].copy_(s["draft"].float() + torch.randn_like(s["draft"].float()) * (0.3 + 0.3 * i))
        for g, got in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, got in graphs:
            check(lm, s, got)


def test_equal_inputs_give_equal_results(lm):
    s = make(9, "f16", [16] * 40, 50001, 2)
    a = lm.mca_verify_drafts(**s)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(a, lm.mca_verify_drafts(**s)))
