"""The language-model operators together, as they answer with a Transformer
context's committed net: prompts and drafts through mca_extend over a paged
cache whose blocks mca_block_tables hands out and mca_cache_append fills, and log
probabilities from its logits, against the fp64 oracle of the net.

Logits: eight products of at most 512 terms one after the other, each sum off by
at most 512 2^-24 of its terms.
"""
import ctypes
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import lm as olm
from oracle.transformer import TransformerModel
from workloads import CONFIGS, transformer_workload

pytestmark = pytest.mark.gpu
TOL = 8 * 512 * 2.0 ** -24


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def make(stream=None, **kw):
    from paper_2607_08406_amd import mca
    cfg = replace(CONFIGS["transformer"], **kw)
    w = transformer_workload(cfg)
    rng = np.random.default_rng(5)
    # weights of a trained net's size, so that attention is not uniform
    params = [p if p.ndim == 1 else (p * rng.uniform(1, 6)).astype(np.float32) for p in w["params"]]
    desc = mca.transformer_desc(cfg.vocab, cfg.ctx, cfg.d_model, cfg.n_layer, cfg.n_head, cfg.d_mlp, delta=cfg.delta,
                                ln_eps=cfg.ln_eps, seed=cfg.seed_stream, stream_tag=cfg.stream_tag)
    ctx = mca.TransformerContext(desc, params, w["tokens"], w["targets"], k_max=2, stream=stream)
    return ctx, cfg, params


def oracle_logits(cfg, params, seq):
    seq = np.asarray(seq)[None]
    m = TransformerModel(params, seq, seq, cfg.vocab, cfg.ctx, cfg.d_model, cfg.n_layer, cfg.n_head, cfg.d_mlp, cfg.ln_eps)
    return m.logits_of(m.params)[0]


def put(a, dt=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()


class Server:
    """What a program keeps: texts, the cache and its tables."""

    def __init__(self, lm, cfg, R, block, n_blocks):
        self.lm, self.cfg, self.R, self.block = lm, cfg, R, block
        self.cache = [torch.full((cfg.n_layer, n_blocks, cfg.n_head, block, 32), float("nan"), device="cuda") for _ in range(2)]
        self.width = -(-cfg.ctx // block)
        self.table = torch.full((R, self.width), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(n_blocks, device="cuda").int()
        self.lens = np.zeros(R, np.int64)

    def extend(self, ctx, tokens, parents, counts, max_nodes):
        first = np.concatenate([[0], np.cumsum(counts)])
        return ctx.extend(put(tokens), put(parents), put(first), put(self.lens), self.table, *self.cache, max_nodes,
                          max_len=self.cfg.ctx)

    def keep(self, qkv, rows, counts):
        """The given rows of a call, counts of them per request, become cached tokens."""
        new = self.lens + counts
        n = int(np.sum(counts))
        offsets, status = put(np.zeros(self.R + 1)), put(np.zeros(4))
        slots = torch.zeros(n + 2, dtype=torch.int64, device="cuda")
        self.lm.mca_block_tables(put(self.lens), put(new), self.table, self.free, self.block, offsets, slots, status)
        assert status[0] == 0 and status[2] == n
        idx = put(np.concatenate([rows, [0, 0]]))
        for b in range(self.cfg.n_layer):
            self.lm.mca_cache_append(qkv[b, :, 1], qkv[b, :, 2], self.cache[0][b], self.cache[1][b], slots, idx)
        self.lens = new


@pytest.mark.parametrize("kw,block", [(dict(ctx=32, d_model=64, n_head=2, n_seq=2, d_mlp=96), 4),
                                      (dict(n_seq=2), 16), (dict(n_seq=2, d_model=160, n_head=5, vocab=100), 5)])
def test_prompts_drafts_and_single_tokens(lm, kw, block):
    ctx, cfg, params = make(**kw)
    rng = np.random.default_rng(7)
    R = 4
    srv = Server(lm, cfg, R, block, 4 * (-(-cfg.ctx // block)) + 3)
    plen = np.array([cfg.ctx - 9, 1, 7, 18])
    text = [list(rng.integers(0, cfg.vocab, n)) for n in plen]
    # prompts, as chains
    tokens = np.concatenate(text)
    parents = np.concatenate([np.arange(n) - 1 for n in plen])
    logits, qkv = srv.extend(ctx, tokens, parents, plen, cfg.ctx)
    got = logits.cpu().numpy()
    at = 0
    for r in range(R):
        want = oracle_logits(cfg, params, text[r])
        assert np.abs(got[at:at + plen[r]] - want).max() <= TOL * np.abs(want).max()
        at += plen[r]
    # the given next symbols' log probabilities
    nxt = np.concatenate([t[1:] + [-1] for t in text])
    res = lm.mca_token_logprobs(logits, put(nxt), 3)
    lp = olm.token_logprobs(got, nxt)[0]
    assert np.abs(res.logprob.cpu().numpy() - lp).max() <= 1e-5
    srv.keep(qkv, np.arange(len(tokens)), plen)
    # three rounds of drafts: a tree for each request, an accepted path each
    for rnd in range(3):
        counts = np.array([3, 5, 2, 1]) if rnd < 2 else np.ones(R, int)  # the last round: single tokens
        trees = [[-1] + [int(rng.integers(-1, i)) for i in range(1, n)] for n in counts]
        draft = [list(rng.integers(0, cfg.vocab, n)) for n in counts]
        logits, qkv = srv.extend(ctx, np.concatenate(draft), np.concatenate(trees), counts, int(counts.max()))
        got, at, rows, taken = logits.cpu().numpy(), 0, [], []
        for r in range(R):
            paths = []
            for i in range(counts[r]):
                p = paths[trees[r][i]] + [i] if trees[r][i] >= 0 else [i]
                paths.append(p)
                want = oracle_logits(cfg, params, text[r] + [draft[r][j] for j in p])[-1]
                assert np.abs(got[at + i] - want).max() <= TOL * np.abs(want).max(), (rnd, r, i)
            best = paths[-1][:2]
            rows += [at + j for j in best]
            taken.append(len(best))
            text[r] += [draft[r][j] for j in best]
            at += counts[r]
        srv.keep(qkv, rows, np.array(taken))
    assert [len(t) for t in text] == list(srv.lens)
    ctx.close()


def test_symbols_and_positions_out_of_range(lm):
    """They give NaN to their node and to those that see it, and to no others."""
    ctx, cfg, params = make(ctx=8, d_model=64, n_head=2, n_seq=2, d_mlp=96)
    srv = Server(lm, cfg, 2, 4, 8)
    tokens = np.array([1, cfg.vocab, 2, 3, -1, 0])
    logits, _ = srv.extend(ctx, tokens, [-1, 0, 1, 0, -1, -1], [4, 2], 4)
    bad = torch.isnan(logits).any(1).cpu().tolist()
    assert bad == [False, True, True, False, True, False]
    want = oracle_logits(cfg, params, [1, 3])
    assert np.abs(logits[3].cpu().numpy() - want[1]).max() <= TOL * np.abs(want).max()
    logits, qkv = srv.extend(ctx, np.ones(10), np.concatenate([np.arange(9) - 1, [-1]]), [9, 1], 9)
    bad = torch.isnan(logits).any(1).cpu().tolist()
    assert bad == [False] * 8 + [True, False]  # the context has 8 positions
    ctx.close()


def test_rows_behind_the_last_request_and_the_committed_state(lm):
    """A call leaves padding rows, the training state and the next steps as they were, and uses the committed weights."""
    ctx, cfg, params = make(ctx=32, d_model=64, n_head=2, n_seq=2, d_mlp=96)
    srv = Server(lm, cfg, 2, 8, 8)
    logits = torch.full((7, cfg.vocab), 9.0, device="cuda")
    args = [put(x) for x in ([1, 2, 3, 0, 0, 0, 0], [-1, 0, -1, -1, -1, -1, -1], [0, 2, 3], [0, 0])]
    cands = ctx.propose(0, 2)
    before, _ = ctx.eval_losses(cands)
    ctx.extend(*args, srv.table, *srv.cache, 2, max_len=0, logits=logits)  # a batch is pending
    ctx.rollback()
    again, _ = ctx.eval_losses(cands)
    assert (before == again).all()
    assert (logits[3:] == 9).all() and torch.isfinite(logits[:3]).all()
    ctx.rollback()
    moved = [p.copy() for p in params]
    moved[0][2] += 0.5
    ctx.set_state(moved, None, 0)
    out, _ = ctx.extend(*args, srv.table, *srv.cache, 2, max_len=0)
    want = oracle_logits(cfg, moved, [1, 2])
    assert np.abs(out[:2].cpu().numpy() - want).max() <= TOL * np.abs(want).max()
    ctx.close()


def test_refusals(lm):
    from paper_2607_08406_amd import mca
    ctx, cfg, _ = make(ctx=32, d_model=64, n_head=2, n_seq=2, d_mlp=96)
    srv = Server(lm, cfg, 2, 8, 8)
    a = [put([1, 2, 3]), put([-1, 0, -1]), put([0, 2, 3]), put([0, 0]), srv.table, *srv.cache]
    for i, bad in ((0, a[0].long()), (1, a[1][:2]), (2, a[2][:2]), (3, a[3].cpu()), (4, srv.table.long()),
                   (5, srv.cache[0][:1]), (6, srv.cache[1].half())):
        with pytest.raises(mca.MCAError):
            ctx.extend(*a[:i], bad, *a[i + 1:], 2)
    for kw in (dict(max_nodes=129), dict(max_nodes=0), dict(max_nodes=2, max_len=-1),
               dict(max_nodes=2, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")),
               dict(max_nodes=2, qkv=torch.empty(1, device="cuda")), dict(max_nodes=2, logits=torch.empty(3, 4, device="cuda"))):
        with pytest.raises(mca.MCAError):
            ctx.extend(*a, **kw)
    w = np.zeros((8, 4), np.float32), np.zeros((3, 8), np.float32)
    mlp = mca.Context(mca.mlp_desc((4, 8, 3)), w, np.zeros((5, 4), np.float32), np.zeros(5, np.int32), 1)
    n = mca.mca_extend_args()
    assert mca.load_library().mca_extend(mlp.ctx, ctypes.byref(n)) == mca.MCA_EINVAL
    mlp.close()
    ctx.close()


def test_extend_refuses_more_rows_than_it_can_address(lm):
    from paper_2607_08406_amd import mca
    ctx, cfg, _ = make(ctx=32, d_model=64, n_head=2, n_seq=2, d_mlp=96)
    lib, room = mca.load_library(), ctypes.c_size_t()
    a = mca.mca_extend_args(n_req=1, n_rows=2 ** 31 // (3 * 64) + 1, max_nodes=1, max_len=32, block_size=8, n_blocks=4, max_blocks=4)
    assert lib.mca_extend_plan(ctx.ctx, ctypes.byref(a), ctypes.byref(room)) == mca.MCA_EUNSUPPORTED
    assert lib.mca_extend(ctx.ctx, ctypes.byref(a)) == mca.MCA_EUNSUPPORTED
    a.n_rows -= 1
    assert lib.mca_extend_plan(ctx.ctx, ctypes.byref(a), ctypes.byref(room)) == mca.MCA_OK
    ctx.close()


def test_captured_step(lm):
    """Tables, net, rows and log probabilities in one graph; each replay on new inputs equals the eager calls, with
    eager work and other graphs' replays in between."""
    s = torch.cuda.Stream()
    ctx, cfg, _ = make(stream=s, ctx=32, d_model=64, n_head=2, n_seq=2, d_mlp=96)
    R, n, block, n_blocks = 3, 4, 4, 30

    def state():
        d = dict(tokens=torch.zeros(R * n, dtype=torch.int32), parents=torch.full((R * n,), -1, dtype=torch.int32),
                 offsets=torch.zeros(R + 1, dtype=torch.int32), old=torch.zeros(R, dtype=torch.int32),
                 new=torch.zeros(R, dtype=torch.int32), table=torch.zeros(R, 8, dtype=torch.int32),
                 free=torch.arange(n_blocks, dtype=torch.int32), taken=torch.zeros(R + 1, dtype=torch.int32),
                 slots=torch.zeros(R * n, dtype=torch.int64), status=torch.zeros(4, dtype=torch.int32),
                 next=torch.zeros(R * n, dtype=torch.int64), logits=torch.zeros(R * n, cfg.vocab),
                 qkv=torch.zeros(cfg.n_layer, R * n, 3, 2, 32), kc=torch.zeros(cfg.n_layer, n_blocks, 2, block, 32),
                 vc=torch.zeros(cfg.n_layer, n_blocks, 2, block, 32))
        return {k: v.cuda() for k, v in d.items()}

    def step(d):
        lm.mca_extend(ctx, d["tokens"], d["parents"], d["offsets"], d["old"], d["table"], d["kc"], d["vc"], n, max_len=32,
                      qkv=d["qkv"], logits=d["logits"])
        lm.mca_block_tables(d["old"], d["new"], d["table"], d["free"], block, d["taken"], d["slots"], d["status"])
        for b in range(cfg.n_layer):
            lm.mca_cache_append(d["qkv"][b, :, 1], d["qkv"][b, :, 2], d["kc"][b], d["vc"][b], d["slots"])
        r = lm.mca_token_logprobs(d["logits"], d["next"], 5)
        g = lm.mca_token_logprobs_grad(d["logits"], d["next"], r.lse, r.entropy, r.entropy, r.logprob)
        return [*r, g]

    def fill(d, old, seed):
        g = np.random.default_rng(seed)
        d["tokens"].copy_(put(g.integers(0, cfg.vocab, R * n)))
        d["next"].copy_(put(g.integers(0, cfg.vocab, R * n), torch.int64))
        d["parents"].copy_(put(np.tile(np.arange(n) - 1, R)))
        d["offsets"].copy_(put(np.arange(R + 1) * n))
        d["old"].copy_(put(old))
        d["new"].copy_(put(old + n))

    a, b = state(), state()
    with torch.cuda.stream(s):
        fill(a, np.zeros(R, int), 0)
        step(a)  # warm-up
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = step(a)
        a2 = state()
        for k in a:
            a[k].copy_(a2[k])
        for rnd in range(4):
            fill(a, np.full(R, rnd * n), rnd + 1)
            fill(b, np.full(R, rnd * n), rnd + 1)
            graph.replay()
            want = step(b)
            s.synchronize()
            for x, y in zip(outs, want):
                assert torch.equal(x, y), rnd
            for k in a:
                assert torch.equal(a[k], b[k]), (rnd, k)
            torch.randn(1000, device="cuda").sum().item()
    ctx.close()


def test_calls_on_another_stream(lm):
    """The work goes on the current stream, behind what fills its inputs there."""
    s = torch.cuda.Stream()
    z = torch.zeros(64, 30000, device="cuda")
    tok = torch.arange(64, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            z.normal_()
        r = lm.mca_token_logprobs(z, tok, 4)
        g = lm.mca_token_logprobs_grad(z, tok, r.lse, r.entropy, r.entropy)
    s.synchronize()
    w = lm.mca_token_logprobs(z, tok, 4)
    assert all(torch.equal(x, y) for x, y in zip(r, w))
    assert torch.equal(g, lm.mca_token_logprobs_grad(z, tok, r.lse, r.entropy, r.entropy))
