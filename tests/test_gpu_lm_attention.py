"""GPU parity of mca_tree_attention against the fp64 oracle.

Tolerance of an output, from the arithmetic: a score is a 32-bit sum of
head_dim exact products, so it is off by at most (head_dim + 8) 2^-24 of
sum |q k| scale (the 8: scaling, exponent's argument, exponential), and a
weight relative to another by twice that; the sum over L tokens adds
(L + 16) 2^-24; weights of 16-bit values are rounded once (half a step, and
2^-25 of the largest weight below fp16's normal range); the result is rounded
once (half a step).
"""
import numpy as np
import pytest
import torch

from oracle import lm as olm

pytestmark = pytest.mark.gpu

LONG = 1 << 17  # a max_len at which many rows are worked on in shares

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def make(seed, typ, lens, nodes, heads, kv, dim, block, chain=False, spare=2, qscale=1.0):
    """One call's tensors; q, k and v are parts of one projection's rows, with rows behind the last request."""
    rng = np.random.default_rng(seed)
    dt = TYPES[typ]
    R, total = len(lens), int(np.sum(nodes))
    T = total + 3
    width = max(1, max(-(-n // block) for n in lens))
    held = [-(-n // block) for n in lens]
    pool = rng.permutation(sum(held) + spare)
    table = np.full((R, width), -7, np.int32)
    at = 0
    for r, n in enumerate(held):
        table[r, :n] = pool[at:at + n]
        at += n
    qkv = torch.from_numpy(rng.normal(size=(T, (heads + 2 * kv) * dim))).to(dt).cuda()
    q, k, v = qkv.split([heads * dim, kv * dim, kv * dim], 1)
    caches = [torch.from_numpy(rng.normal(size=(len(pool), kv, block, dim))).to(dt).cuda() for _ in range(2)]
    parents = np.full(T, -1, np.int32)
    first = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    for r in range(R):
        for i in range(1, nodes[r]):
            parents[first[r] + i] = i - 1 if chain else rng.integers(-1, i)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    return dict(q=(q * qscale).to(dt).view(T, heads, dim) if qscale != 1.0 else q.view(T, heads, dim), k=k.view(T, kv, dim),
                v=v.view(T, kv, dim), k_cache=caches[0], v_cache=caches[1], table=put(table), lengths=put(lens),
                offsets=put(first), parents=put(parents), max_nodes=max(1, max(nodes)))


def check(s, got, scale=None, skip=()):
    out, lse = got
    host = {n: (t.float() if t.is_floating_point() else t).cpu().numpy() for n, t in s.items() if isinstance(t, torch.Tensor)}
    dim = host["q"].shape[2]
    sc = np.float32(dim ** -0.5 if scale is None else scale)
    want = olm.tree_attention(host["q"], host["k"], host["v"], host["k_cache"], host["v_cache"], host["table"],
                              host["lengths"], host["offsets"], host["parents"], float(sc))
    got_o, got_l = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy()
    eps = torch.finfo(s["q"].dtype).eps / 2
    narrow = s["q"].dtype != torch.float32
    for (row, head), (o, norm, pv, sv, size, L) in want.items():
        if row in skip:
            continue
        e32 = 2 * (dim + 8) * 2.0 ** -24 * size + (L + 16) * 2.0 ** -24
        tol = eps * np.abs(o) * (1 + 2 ** -6) + (e32 + (eps if narrow else 0)) * pv * (1 + 2 ** -6)
        if s["q"].dtype == torch.float16:
            tol = tol + 2.0 ** -25 * (sv + 1)
        d = np.abs(got_o[row, head] - o)
        assert (np.isnan(o) == np.isnan(got_o[row, head])).all(), (row, head)
        fin = np.isfinite(o)
        assert (got_o[row, head][~fin & ~np.isnan(o)] == o[~fin & ~np.isnan(o)]).all()
        assert (d[fin] <= tol[fin]).all(), (row, head, float((d[fin] - tol[fin]).max()), float(d[fin].max()))
        if np.isfinite(norm):
            assert abs(got_l[row, head] - norm) <= e32 + 2.0 ** -22 * (abs(norm) + 1), (row, head, got_l[row, head], norm)


def call(lm, s, **kw):
    return lm.mca_tree_attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["offsets"],
                                 s["parents"], s["max_nodes"], **kw)


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 64, 128, 256])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2)])
def test_types_and_heads(lm, typ, dim, heads, kv):
    s = make(3, typ, [0, 1, 37, 130], [1, 5, 2, 9], heads, kv, dim, 16)
    check(s, call(lm, s))


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [16, 24, 40, 48, 80, 96, 112, 136, 192, 200])
def test_odd_head_dims(lm, typ, dim):
    s = make(5, typ, [3, 65], [4, 3], 4, 2, dim, 8)
    check(s, call(lm, s))


@pytest.mark.parametrize("block", [1, 3, 8, 16, 20, 32, 48, 64, 256])
def test_block_sizes(lm, block):
    """Pages that end inside a tile, and tiles inside a page."""
    s = make(7, "bf16", [31, 32, 33, 64, 95], [1, 3, 2, 4, 1], 4, 2, 64, block)
    check(s, call(lm, s))


@pytest.mark.parametrize("length", [1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 511, 513, 1025, 2600])
@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_single_tokens_over_lengths(lm, typ, length):
    """A decoding step; lengths around tiles, rounds of the waves and chunks."""
    s = make(length, typ, [length], [1], 8, 2, 64, 16)
    check(s, call(lm, s))


@pytest.mark.parametrize("nodes", [2, 31, 32, 33, 64, 97, 128])
@pytest.mark.parametrize("chain", [False, True])
def test_many_nodes(lm, nodes, chain):
    s = make(nodes, "bf16", [70, 0], [nodes, max(1, nodes - 3)], 4, 2, 32, 16, chain=chain)
    check(s, call(lm, s))


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_many_rows_share_a_key_head(lm, typ):
    s = make(11, typ, [300, 40], [24, 17], 16, 1, 128 if typ != "f32" else 64, 32)
    check(s, call(lm, s))


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 96, 128, 136, 256])
@pytest.mark.parametrize("rows", [17, 32, 33, 64, 65, 128, 224, 256, 257])
@pytest.mark.parametrize("more", [0, 600])
def test_rows_of_a_key_head(lm, typ, dim, rows, more):
    """Numbers of rows around those at which waves and workgroups take more; contexts of few tiles.  With many
    requests (which are empty) a tile is read once for many rows."""
    group, nodes = (1, rows) if rows < 100 else ((2, rows // 2) if rows % 2 == 0 else (257, 1))
    s = make(rows, typ, [200, 33, 0] + [0] * more, [nodes, max(1, nodes // 3), 1] + [0] * more, group, 1, dim, 16)
    check(s, call(lm, s))


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 64, 80, 128, 200, 256])
@pytest.mark.parametrize("group,nodes", [(1, 40), (4, 13), (8, 20), (8, 30)])
def test_shared_work(lm, typ, dim, group, nodes):
    """Many rows over long and short contexts: the workgroups' shares begin and end inside requests, key heads, tiles
    of rows and drafted tiles."""
    s = make(dim + nodes, typ, [0, 2300, 70, 2049, 1], [nodes, max(1, nodes - 5), 0, nodes, 3], 2 * group, 2, dim, 16)
    a = call(lm, s, max_len=LONG)
    check(s, a)
    b = call(lm, s, max_len=LONG)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_shared_work_of_many_requests(lm, typ):
    """More requests than a workgroup has threads, most of them short or without nodes."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 700)
    lens[[5, 300, 699]] = [2500, 1200, 3000]
    nodes = np.where(rng.random(700) < 0.8, 0, rng.integers(1, 3, 700))
    nodes[[5, 300, 699]] = [40, 3, 33]
    s = make(61, typ, list(lens), list(nodes), 1, 1, 32, 16)
    check(s, call(lm, s, max_len=LONG))


def test_shared_work_with_bad_blocks_and_values(lm):
    """Blocks that are not there inside whole tiles, and drafted values that are not finite, at every place of a share."""
    s = make(67, "bf16", [2500, 1500], [60, 37], 4, 2, 64, 16)
    for r, c in ((0, 3), (0, 70), (0, 71), (0, 155), (1, 0), (1, 93)):
        s["table"][r, c] = -1
    s["parents"][:60] = torch.arange(-1, 59, dtype=torch.int32, device="cuda")
    s["parents"][50:60] = 20
    s["v"][40] = float("nan")  # nodes 40 to 49 see it
    s["k"][51], s["v"][51] = float("inf"), float("nan")  # node 51 alone
    out, lse = call(lm, s, max_len=LONG)
    check(s, (out, lse), skip=[51])
    assert torch.isnan(out[40:50]).all() and torch.isfinite(out[:40]).all() and torch.isfinite(out[52:97]).all()


@pytest.mark.parametrize("typ,dim", [("bf16", 64), ("f16", 128), ("bf16", 256), ("f32", 128), ("f32", 64)])
def test_single_tokens_over_long_contexts_in_plenty(lm, typ, dim):
    s = make(71, typ, [2300, 0, 70, 3000, 16, 1], [1, 2, 1, 0, 4, 1], 8, 2, dim, 16)
    check(s, call(lm, s, max_len=1 << 20))


def test_ragged_and_empty_requests(lm):
    """Requests without nodes between others, and rows behind the last request left as they were."""
    s = make(13, "bf16", [9, 50, 0, 18, 400], [2, 0, 3, 0, 1], 4, 4, 64, 16)
    out = torch.full_like(s["q"], 7.0)
    lse = torch.full(s["q"].shape[:2], 5.0, device="cuda")
    check(s, call(lm, s, out=out, lse=lse))
    assert (out[6:] == 7).all() and (lse[6:] == 5).all()


def test_peaked_scores(lm):
    """Large scores: one weight near 1, the running maximum moves many times."""
    for typ in ("bf16", "f16", "f32"):
        s = make(17, typ, [700], [6], 4, 2, 64, 16, qscale=12.0)
        check(s, call(lm, s))


def test_scale_and_rising_scores(lm):
    s = make(19, "f32", [500], [1], 1, 1, 32, 16)
    s["k_cache"][:] = 0
    t = torch.arange(500, device="cuda")
    s["k_cache"][s["table"][0, t // 16].long(), 0, t % 16, 0] = t.float()
    s["q"][0, 0, 0] = 1.0
    check(s, call(lm, s, scale=0.25), scale=0.25)
    check(s, call(lm, s, scale=-0.25), scale=-0.25)
    check(s, call(lm, s, scale=0.0), scale=0.0)


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_seen_do_not_matter(lm, typ, bad):
    """Not finite: cached places behind a request's tokens, other requests' blocks, and a node that others do not see."""
    s = make(23, typ, [37, 70], [5, 1], 4, 2, 128, 16)
    s["parents"][:6] = torch.tensor([-1, 0, -1, 1, 2, -1], dtype=torch.int32, device="cuda")
    tab = s["table"].cpu().numpy()
    s["k_cache"][int(tab[0, 2]), :, 5:] = bad
    s["v_cache"][int(tab[0, 2]), :, 5:] = bad
    unused = set(range(s["k_cache"].shape[0])) - set(tab[0, :3]) - set(tab[1, :5])
    for b in unused:
        s["k_cache"][b], s["v_cache"][b] = bad, bad
    # node 2 (seen by 2 and 4 alone); the row of its scores is not finite for those two
    s["k"][2], s["v"][2] = bad, bad
    s["v"][1, 0, 3] = bad  # seen by 1 and 3: its value alone
    s["q"][6:] = bad
    s["k"][6:], s["v"][6:] = bad, bad
    out, lse = call(lm, s)
    check(s, (out, lse), skip=(2, 4))
    assert torch.isfinite(out[[0, 5]]).all() and torch.isfinite(lse[[0, 1, 3, 5]]).all()


def test_bad_blocks_are_absent(lm):
    """Table entries outside the cache: their tokens are not there."""
    s = make(29, "bf16", [100, 64], [2, 1], 4, 2, 64, 16)
    s["table"][0, 2] = -1
    s["table"][0, 5] = s["k_cache"].shape[0]
    s["table"][1, :] = 2 ** 31 - 1
    check(s, call(lm, s))


def test_bad_lengths_offsets_and_parents(lm):
    s = make(31, "f32", [20, 40, 33], [3, 2, 4], 4, 4, 32, 16)
    want, _ = call(lm, s)
    s["lengths"][0] = 10 ** 9  # counts as what max_len and the table hold
    s["lengths"][2] = -5       # counts as none
    out, _ = call(lm, s, max_len=40)
    s["lengths"][0], s["lengths"][2] = 40, 0
    check(s, call(lm, s))
    assert torch.equal(out, call(lm, s)[0])
    s["parents"][3:5] = torch.tensor([7, -9], dtype=torch.int32, device="cuda")  # request 1: both stand alone
    check(s, call(lm, s))
    s["offsets"][3] = 10 ** 6  # request 2's rows are out of range: left as they were
    out, _ = call(lm, s, out=torch.full_like(s["q"], 3.0))
    assert (out[5:] == 3).all() and torch.isfinite(out[:5]).all() and torch.isfinite(want).all()


def test_max_nodes_bounds_a_request(lm):
    s = make(37, "f32", [20, 40], [3, 6], 4, 4, 32, 16)
    s["max_nodes"] = 5
    out, _ = call(lm, s, out=torch.full_like(s["q"], 3.0))
    assert (out[3:] == 3).all() and (out[:3] != 3).any()


def test_strides_of_queries_and_results(lm):
    s = make(41, "f16", [90, 12], [3, 2], 4, 2, 64, 16)
    T = s["q"].shape[0]
    s["q"] = s["q"].transpose(0, 1).contiguous().transpose(0, 1)  # heads outermost
    s["k"] = torch.cat([s["k"], s["k"]], 2)[:, :, :64]
    out = torch.zeros(T, 4, 80, dtype=torch.float16, device="cuda")[:, :, 8:72]
    check(s, call(lm, s, out=out))


def test_results_do_not_depend_on_the_run(lm):
    s = make(43, "bf16", [3000, 10, 777], [7, 1, 3], 8, 2, 128, 16)
    a = call(lm, s)
    for _ in range(3):
        b = call(lm, s)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_rows_behind_32_bit_offsets(lm):
    """A cache of more than 2^32 bytes: the request's blocks lie behind them."""
    dim, block, kv = 128, 64, 8
    n_blocks = (2 ** 32 // (dim * 2 * block * kv)) + 40
    s = make(47, "bf16", [1000], [2], 8, kv, dim, block)
    held = s["k_cache"].shape[0]
    for n in ("k_cache", "v_cache"):
        big = torch.zeros(n_blocks, kv, block, dim, dtype=torch.bfloat16, device="cuda")
        big[n_blocks - held:] = s[n]
        s[n] = big
    small = dict(s, k_cache=s["k_cache"][n_blocks - held:].contiguous(), v_cache=s["v_cache"][n_blocks - held:].contiguous())
    want = call(lm, small)
    s["table"] = s["table"] + (n_blocks - held)
    got = call(lm, s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_many_rows_behind_32_bit_offsets(lm):
    dim, block, kv = 128, 64, 8
    n_blocks = (2 ** 32 // (dim * 2 * block * kv)) + 40
    s = make(73, "bf16", [1000], [40], 8, kv, dim, block)
    held = s["k_cache"].shape[0]
    small = dict(s)
    for n in ("k_cache", "v_cache"):
        big = torch.zeros(n_blocks, kv, block, dim, dtype=torch.bfloat16, device="cuda")
        big[n_blocks - held:] = s[n]
        s[n] = big
    s["table"] = s["table"] + (n_blocks - held)
    want, got = call(lm, small, max_len=LONG), call(lm, s, max_len=LONG)
    check(small, want)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals(lm):
    from paper_2607_08406_amd.mca import MCAError
    s = make(53, "bf16", [20], [2], 4, 2, 64, 16)
    for kw in (dict(q=s["q"].float()), dict(k=s["k"][:, :1]), dict(table=s["table"].long()), dict(lengths=s["lengths"].cpu()),
               dict(k_cache=s["k_cache"].transpose(1, 2)), dict(max_nodes=129), dict(parents=s["parents"][:-1]),
               dict(q=s["q"].transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(MCAError):
            call(lm, dict(s, **kw))
    s = make(53, "bf16", [9000], [2], 4, 2, 64, 16)
    with pytest.raises(MCAError):
        call(lm, s, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
