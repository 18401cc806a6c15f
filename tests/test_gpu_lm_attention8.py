"""GPU parity of mca_tree_attention8 against the fp64 oracle on the values that the
codes stand for.

Those values are exact in every type here, so the bounds are those of attention over a
cache of its own type: a score is a 32-bit sum of head_dim exact products, off by at
most (head_dim + 8) 2^-24 of sum |q k| scale, and a weight relative to another by
twice that; the sum over L tokens adds (L + 16) 2^-24; weights of 16-bit values are
rounded once (half a step, and 2^-25 of the largest weight below fp16's normal range);
the result is rounded once (half a step).  Below 2^-126, where 32-bit numbers have no full
precision, a weight or a result may be off by all of itself: 2^-126 (1 + sum |v|).
"""
import numpy as np
import pytest
import torch

from lm8_util import TYPES, cache, codes, host, pages, put
from oracle import lm as olm

pytestmark = pytest.mark.gpu

LONG = 1 << 17  # a max_len at which many rows are worked on in shares


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def make(seed, typ, lens, nodes, heads, kv, dim, block, chain=False, spread=2, spare=2):
    rng = np.random.default_rng(seed)
    dt = TYPES[typ]
    R, T = len(lens), int(np.sum(nodes)) + 3
    table, blocks = pages(rng, lens, block, spare=spare)
    (kc, ks), (vc, vs) = cache(rng, blocks, kv, block, dim, spread)
    ks, vs = ks - 2, vs - 2  # values of up to 7, give or take the spread
    qkv = torch.from_numpy(rng.normal(size=(T, (heads + 2 * kv) * dim))).to(dt).cuda()
    q, k, v = qkv.split([heads * dim, kv * dim, kv * dim], 1)
    parents = np.full(T, -1, np.int32)
    first = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    for r in range(R):
        for i in range(1, nodes[r]):
            parents[first[r] + i] = i - 1 if chain else rng.integers(-1, i)
    return dict(q=q.view(T, heads, dim), k=k.view(T, kv, dim), v=v.view(T, kv, dim), k_cache=codes(kc), v_cache=codes(vc),
                k_scale=put(ks, np.uint8), v_scale=put(vs, np.uint8), table=put(table), lengths=put(lens), offsets=put(first),
                parents=put(parents), max_nodes=max(1, max(nodes)))


def check(s, got, scale=None):
    out, lse = got
    h = {n: host(t) for n, t in s.items() if isinstance(t, torch.Tensor)}
    dim = h["q"].shape[2]
    sc = np.float32(dim ** -0.5 if scale is None else scale)
    want = olm.tree_attention(h["q"], h["k"], h["v"], olm.cache8_values(h["k_cache"], h["k_scale"]),
                              olm.cache8_values(h["v_cache"], h["v_scale"]), h["table"], h["lengths"], h["offsets"], h["parents"],
                              float(sc))
    got_o, got_l = host(out).astype(np.float64), host(lse)
    eps = torch.finfo(s["q"].dtype).eps / 2
    narrow = s["q"].dtype != torch.float32
    used = np.zeros(len(got_o), bool)
    for (row, head), (o, norm, pv, sv, size, L) in want.items():
        used[row] = True
        e32 = 2 * (dim + 8) * 2.0 ** -24 * size + (L + 16) * 2.0 ** -24
        tol = eps * np.abs(o) * (1 + 2 ** -6) + (e32 + (eps if narrow else 0)) * pv * (1 + 2 ** -6)
        tol = tol + 2.0 ** (-25 if s["q"].dtype == torch.float16 else -126) * (sv + 1)
        d = np.abs(got_o[row, head] - o)
        assert (np.isnan(o) == np.isnan(got_o[row, head])).all(), (row, head)
        fin = np.isfinite(o)
        assert (d[fin] <= tol[fin]).all(), (row, head, float((d[fin] - tol[fin]).max()), float(d[fin].max()))
        assert abs(got_l[row, head] - norm) <= e32 + 2.0 ** -23 * abs(norm) or (np.isnan(norm) and np.isnan(got_l[row, head]))
    return used


CASES = [
    # lens, nodes, heads, kv, dim, block
    ([0, 1, 120, 33], [8, 1, 3, 5], 4, 4, 32, 16),
    ([700, 65, 0, 64], [1, 1, 1, 1], 8, 2, 128, 64),
    ([300, 17], [40, 12], 8, 1, 64, 20),
    ([50, 129], [3, 2], 6, 3, 80, 7),
    ([200], [9], 2, 1, 256, 33),
    ([64, 31], [2, 7], 5, 1, 16, 8),
    ([95], [128], 2, 2, 112, 1),
    ([1000, 1], [100, 128], 4, 2, 128, 128),
]


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(lm, typ, case):
    s = make(case, typ, *CASES[case])
    keep = torch.full_like(s["q"], 5.0), torch.full(s["q"].shape[:2], 6.0, device="cuda")
    got = lm.mca_tree_attention8(**s, out=keep[0], lse=keep[1])
    used = check(s, got)
    assert (host(got[0])[~used] == 5).all() and (host(got[1])[~used] == 6).all()


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("dim,rows", [(32, 200), (64, 40), (64, 128), (128, 72), (128, 256), (96, 256), (256, 130), (240, 40)])
def test_many_rows(lm, typ, dim, rows):
    """The kernels of many rows: tiles of a workgroup each, and worked on in shares (max_len LONG)."""
    s = make(rows, typ, [900, 0, 77, 1300], [rows // 2, rows // 2, 3, rows // 2], 2, 1, dim, 50)
    check(s, lm.mca_tree_attention8(**s))
    check(s, lm.mca_tree_attention8(**s, max_len=LONG))


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("dim,nodes,group", [(80, 1, 1), (128, 1, 8), (128, 4, 4), (128, 16, 1), (256, 3, 2), (240, 1, 1)])
def test_shares_of_few_rows(lm, typ, dim, nodes, group):
    """At most 16 rows a key head whose max_len lets the work be dealt out: requests that one workgroup has whole, cut at
    its ends, over several of them, without cached tokens, without nodes."""
    lens = [900, 0, 77, 2600, 5, 1300, 128, 3, 3, 3, 500, 1024]
    s = make(dim + nodes, typ, lens, [nodes, nodes, 1, nodes, 0] + [nodes] * 7, 2 * group, 2, dim, 50, spread=3)
    keep = torch.full_like(s["q"], 5.0), torch.full(s["q"].shape[:2], 6.0, device="cuda")
    got = lm.mca_tree_attention8(**s, max_len=LONG, out=keep[0], lse=keep[1])
    used = check(s, got)
    assert (host(got[0])[~used] == 5).all()
    table = host(s["table"])
    table[3, 7], table[0, 3:5] = -1, 10 ** 6  # blocks that are not there
    s["table"] = put(table)
    check(s, lm.mca_tree_attention8(**s, max_len=LONG))


@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_split_over_one_request(lm, typ):
    """Few rows over a long context, in chunks that are joined."""
    s = make(3, typ, [9001], [2], 4, 2, 64, 16)
    check(s, lm.mca_tree_attention8(**s))


@pytest.mark.parametrize("typ", TYPES)
def test_scales_differ_widely(lm, typ):
    """Neighbouring blocks whose scales are up to 2^16 apart."""
    s = make(21, typ, [333, 90], [5, 33], 4, 2, 64, 9, spread=8)
    check(s, lm.mca_tree_attention8(**s), None)


@pytest.mark.parametrize("nodes", [3, 70])
def test_what_is_not_seen_reaches_nothing(lm, nodes):
    """NaN codes behind the last token, in blocks that are not the request's and in those that no request has; blocks
    outside the pool are not there."""
    s = make(5, "bf16", [45, 130, 0], [nodes, nodes, nodes], 4, 1, 64, 16)
    table, lens = host(s["table"]), host(s["lengths"])
    kc, vc = host(s["k_cache"]), host(s["v_cache"])
    seen = np.zeros(kc.shape[:3], bool)
    for r, n in enumerate(lens):
        for t in range(n):
            seen[table[r, t // 16], :, t % 16] = True
    kc[~seen], vc[~seen] = 0x7f, 0xff
    table[1, 3] = 10 ** 6
    s.update(k_cache=codes(kc), v_cache=codes(vc), table=put(table))
    check(s, lm.mca_tree_attention8(**s))


@pytest.mark.parametrize("typ", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [128, 112])
@pytest.mark.parametrize("heads,nodes", [(2, 20), (2, 128), (4, 12), (2, 40)])
def test_many_rows_over_what_is_not_there(lm, typ, dim, heads, nodes):
    """The same of many rows: tiles that end inside a block of odd size, blocks outside the pool in the middle, at a
    tile's end, at a request's, all of one."""
    block = 19
    s = make(31, typ, [345, 64, 128, 700, 19], [nodes, 3, nodes, nodes, 2], heads, 1, dim, block)
    table, lens = host(s["table"]), host(s["lengths"])
    kc, vc = host(s["k_cache"]), host(s["v_cache"])
    seen = np.zeros(kc.shape[:3], bool)
    for r, n in enumerate(lens):
        for t in range(n):
            seen[table[r, t // block], :, t % block] = True
    kc[~seen], vc[~seen] = 0x7f, 0xff
    table[0, 3], table[0, 345 // block], table[3, 5:9], table[4, 0] = 10 ** 6, -1, -7, kc.shape[0]
    s.update(k_cache=codes(kc), v_cache=codes(vc), table=put(table))
    check(s, lm.mca_tree_attention8(**s))
    check(s, lm.mca_tree_attention8(**s, max_len=LONG))
    vc[table[2, 1], 0, 3, 7] = 0x7f  # and a NaN that is seen
    s["v_cache"] = codes(vc)
    check(s, lm.mca_tree_attention8(**s, max_len=LONG))


@pytest.mark.parametrize("nodes", [2, 70])
def test_nan_that_is_seen(lm, nodes):
    """A NaN among a request's values makes its rows' columns NaN, one among its keys its rows; other requests' are
    theirs."""
    s = make(6, "f16", [45, 60], [nodes, nodes], 4, 1, 64, 16)
    vc, table = host(s["v_cache"]), host(s["table"])
    vc[table[0, 1], 0, 3, 7] = 0x7f
    s["v_cache"] = codes(vc)
    check(s, lm.mca_tree_attention8(**s))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.7])
def test_scale(lm, scale):
    s = make(8, "bf16", [77], [6], 4, 2, 32, 16)
    check(s, lm.mca_tree_attention8(**s, scale=scale), scale)


def test_lengths_and_offsets_out_of_range(lm):
    s = make(9, "bf16", [50, 60, 20], [3, 4, 2], 2, 1, 64, 16)
    base = lm.mca_tree_attention8(**s)
    off = host(s["offsets"])
    s["offsets"] = put([off[0], off[1], off[2], 10 ** 6])
    out = torch.full_like(s["q"], 5.0)
    got, _ = lm.mca_tree_attention8(**s, out=out)
    assert torch.equal(got[:off[2]], base[0][:off[2]]) and (got[off[2]:] == 5).all()


def test_captured_with_new_lengths(lm):
    s = make(12, "bf16", [200, 500, 40], [3, 3, 3], 8, 2, 128, 16)
    room = torch.empty(lm.mca_tree_attention8_plan(s["q"], s["k_cache"], 3, s["table"].shape[1], 3), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:2], device="cuda")
    lm.mca_tree_attention8(**s, out=out, lse=lse, workspace=room)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lm.mca_tree_attention8(**s, out=out, lse=lse, workspace=room)
    for lens in ([200, 500, 40], [7, 33, 0], [1, 499, 48]):
        s["lengths"].copy_(put(lens))
        s["q"].normal_()
        graph.replay()
        torch.cuda.synchronize()
        check(s, (out, lse))


def test_a_cache_past_four_gigabytes(lm):
    """Blocks whose bytes and scales lie behind 2^32 (32-bit offsets would read others)."""
    kv, dim, block = 8, 256, 64
    blocks = (1 << 32) // (kv * dim * block) + 4
    k_cache = torch.zeros(blocks, kv, block, dim, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v_cache = torch.zeros(blocks, kv, block, dim, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scale = torch.full((blocks, kv), 119, dtype=torch.uint8, device="cuda")
    for nodes in (1, 24):
        s = make(15, "bf16", [150], [nodes], 16, kv, dim, block)
        small = host(s["table"])[0]
        table = put([[blocks - 1, 1, blocks - 3]])
        for to, big in (("k", k_cache), ("v", v_cache)):
            big.view(torch.uint8)[table[0].long()] = s[to + "_cache"].view(torch.uint8)[put(small).long()]
        ks, vs = scale.clone(), scale.clone()
        ks[table[0].long()], vs[table[0].long()] = s["k_scale"][put(small).long()], s["v_scale"][put(small).long()]
        got = lm.mca_tree_attention8(**{**s, "k_cache": k_cache, "v_cache": v_cache, "k_scale": ks, "v_scale": vs, "table": table})
        check(s, got)
