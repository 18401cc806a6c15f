"""The calls that answer with a trained language model, as measurable cases.

A case describes one call of one operator on data that the program has on the
GPU (kind):

* tables         the block tables and the slot map of a paged cache from the
                 requests' lengths before and after (mca_block_tables);
* append         rows of keys and values into their slots of the cache
                 (mca_cache_append);
* attention      attention of every request's tree of drafted tokens over its
                 cached tokens and over the tree itself (mca_tree_attention);
* logprobs       log probabilities of given tokens, entropies and the most
                 probable alternatives (mca_token_logprobs);
* logprobs_grad  the gradient of those log probabilities and entropies with
                 respect to the logits (mca_token_logprobs_grad).

Inputs are drawn from the seed alone.  With `own` false run() computes the
operators with elementary torch operations in 32 bits; exact() computes them in
64 bits, written apart from that.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------


def listed():
    return [
        # One decoding step of 256 running requests: each grows by a token, few need a block.
        dict(name="tables decode", kind="tables", n_req=256, block=16, max_len=8192, mix="decode"),
        # A scheduler's step over many requests: prompts enter, drafts are accepted, some end.
        dict(name="tables serve", kind="tables", n_req=4001, block=32, max_len=20000, mix="serve"),
        # The accepted nodes of 64 small drafts of the char-level net (4 heads of 32, fp32).
        dict(name="append drafts", kind="append", type="f32", rows=256, kv=4, dim=32, block=16, gather=True),
        # The keys and values of a batch of prompts.
        dict(name="append prompts", kind="append", type="bf16", rows=65000, kv=8, dim=128, block=64, gather=False),
        # The char-level net (4 heads of 32, at most 128 positions, fp32) on 64 drafts of up to 8 tokens.
        dict(name="attention char", kind="attention", type="f32", n_req=64, nodes=8, heads=4, kv=4, dim=32,
             block=16, max_len=120, chain=False),
        # One token of each of 32 requests with long ragged contexts: the cache is read once.
        dict(name="attention decode", kind="attention", type="bf16", n_req=32, nodes=1, heads=32, kv=8, dim=128,
             block=64, max_len=32768, chain=False),
        # Bushy drafts, 8 query heads to a key head: 384 rows read the same cached tile.
        dict(name="attention tree", kind="attention", type="f16", n_req=16, nodes=48, heads=32, kv=4, dim=128,
             block=16, max_len=16384, chain=False),
        # One request with a very long context: the work is split over its length.
        dict(name="attention long", kind="attention", type="bf16", n_req=1, nodes=12, heads=16, kv=2, dim=64,
             block=128, max_len=262144, chain=False),
        # Sampled tokens of a serving batch over a large vocabulary, with 20 alternatives.
        dict(name="logprobs serve", kind="logprobs", type="bf16", rows=8, vocab=128000, top=20, masked=False),
        # Scoring of given text: many rows of an odd length.
        dict(name="logprobs score", kind="logprobs", type="f16", rows=4096, vocab=50001, top=5, masked=False),
        # The gradient at the logits of the char-level net's training batch (64 sequences of 128, 65 symbols).
        dict(name="grad char", kind="logprobs_grad", type="f32", rows=8192, vocab=65, masked=False),
        # The same over a large vocabulary.
        dict(name="grad large", kind="logprobs_grad", type="bf16", rows=4096, vocab=50001, masked=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "append", "attention", "attention", "attention", "logprobs", "logprobs",
                       "logprobs_grad"])
    typ = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind == "tables":
        return dict(kind=kind, n_req=_log(rng, 1, 4000), block=rng.choice([8, 16, 24, 32, 64, 128]),
                    max_len=_log(rng, 100, 20000), mix=rng.choice(["decode", "serve", "serve"]))
    if kind == "append":
        return dict(kind=kind, type=typ, rows=_log(rng, 1, 30000), kv=rng.choice([1, 2, 3, 4, 8]),
                    dim=rng.choice([32, 64, 80, 128]), block=rng.choice([8, 16, 20, 64]), gather=rng.random() < 0.5)
    if kind == "attention":
        kv = rng.choice([1, 2, 4, 8])
        group = rng.choice([1, 1, 2, 4, 5, 8])
        dim = rng.choice([32, 64, 64, 96, 128, 128, 256])
        nodes = rng.choice([1, _log(rng, 2, 16), _log(rng, 16, 128)])
        max_len = _log(rng, 30, 100000)
        # the cached values of a case, and the rows that read them, stay under the listed ones'
        most = min(200e6 / (max_len * kv * dim), 30e9 / (4.0 * max_len * nodes * kv * group * dim), 512)
        if most < 1:
            max_len = int(max_len * most)
            most = 1
        return dict(kind=kind, type=typ, n_req=max(1, min(_log(rng, 1, 200), int(most))), nodes=nodes,
                    heads=kv * group, kv=kv, dim=dim, block=rng.choice([8, 16, 16, 32, 50, 64, 128]),
                    max_len=max(max_len, 16), chain=rng.random() < 0.25)
    vocab = rng.choice([65, _log(rng, 40, 1000), _log(rng, 1000, 200000), _log(rng, 20000, 200000)])
    rows = max(1, min(_log(rng, 1, 20000), 100000000 // vocab))
    if kind == "logprobs":
        return dict(kind=kind, type=typ, rows=rows, vocab=vocab, top=rng.choice([0, 1, 5, 20, 32]),
                    masked=rng.random() < 0.3)
    return dict(kind=kind, type=typ, rows=rows, vocab=vocab, masked=rng.random() < 0.3)


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------


def _host(seed):
    return np.random.default_rng([seed, 11])


def _device(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 13)
    return g


def _put(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def _paged(rng, blocks_of, width, spare):
    """A table of the given numbers of blocks, the pool's blocks in random order, and the free ones behind them."""
    total = int(blocks_of.sum())
    pool = rng.permutation(total + spare).astype(np.int32)
    table = np.zeros((len(blocks_of), width), np.int32)
    held = np.arange(width)[None, :] < blocks_of[:, None]
    table[held] = pool[:total]
    return table, pool, total


def _prepare_tables(case, seed):
    rng = _host(seed)
    R, B, most = case["n_req"], case["block"], case["max_len"]
    old = rng.integers(0, most, R)
    if case["mix"] == "decode":
        new = old + 1
    else:
        what = rng.random(R)
        old = np.where(what < 0.2, 0, old)  # waiting requests, whose prompts enter now
        new = old + rng.integers(0, 9, R)   # running ones: the accepted tokens of a draft
        new = np.where(what < 0.2, rng.integers(1, min(most, 2000), R), new)
        new = np.where(what > 0.85, 0, new)  # ended
        new = np.minimum(new, most)
    # at most so many tokens a step: later requests wait
    n = R * (1 if case["mix"] == "decode" else 9 + min(most, 2000) // 9) + 5
    new = np.where(np.cumsum(np.maximum(new - old, 0)) > n, np.minimum(old, new), new)
    width = -(-most // B)
    have = -(-old // B)
    table, pool, held = _paged(rng, have, width, R * width - int(have.sum()))
    free = np.zeros(len(pool), np.int32)
    free[:len(pool) - held] = pool[held:]
    return dict(kind="tables", block=B, old=_put(old), new=_put(new), table=_put(table), free=_put(free),
                offsets=torch.zeros(R + 1, dtype=torch.int32, device=DEV),
                slots=torch.zeros(n, dtype=torch.int64, device=DEV),
                status=torch.zeros(4, dtype=torch.int32, device=DEV))


def _prepare_append(case, seed):
    rng, g = _host(seed), _device(seed)
    n, H, D, B, dt = case["rows"], case["kv"], case["dim"], case["block"], TYPES[case["type"]]
    blocks = -(-(n + n // 4 + 1) // B)
    slots = rng.permutation(blocks * B)[:n]
    slots[rng.random(n) < 0.02] = -1  # rows that are not kept
    src = n + n // 2 if case["gather"] else n
    qkv = torch.randn(src, 3, H, D, device=DEV, generator=g).to(dt)  # as a projection leaves them
    return dict(kind="append", k=qkv[:, 1], v=qkv[:, 2], slots=_put(slots, torch.int64),
                rows=_put(rng.integers(0, src, n)) if case["gather"] else None,
                k_cache=torch.randn(blocks, H, B, D, device=DEV, generator=g).to(dt),
                v_cache=torch.randn(blocks, H, B, D, device=DEV, generator=g).to(dt))


def _prepare_attention(case, seed):
    rng, g = _host(seed), _device(seed)
    R, n, Hq, H, D, B = (case[x] for x in ("n_req", "nodes", "heads", "kv", "dim", "block"))
    dt = TYPES[case["type"]]
    lens = rng.integers(case["max_len"] // 4, case["max_len"] + 1, R)
    if R > 4:
        lens[rng.integers(0, R)] = 0  # a request that begins
    lens[rng.integers(0, R)] = case["max_len"]
    nodes = rng.integers(max(1, n // 2), n + 1, R)
    nodes[rng.integers(0, R)] = n
    first = np.concatenate([[0], np.cumsum(nodes)])
    total = int(first[-1])
    at = np.arange(total) - np.repeat(first[:-1], nodes)
    parents = at - 1 if case["chain"] else np.maximum(rng.integers(-1, np.maximum(at, 1)), at - 6)
    parents = np.where(at == 0, -1, parents)
    width = -(-case["max_len"] // B)
    table, pool, _ = _paged(rng, -(-lens // B), width, 3)
    T = R * n + 3  # a step has room for whole drafts: rows behind the last request
    qkv = torch.randn(T, (Hq + 2 * H) * D, device=DEV, generator=g).to(dt)  # as a projection leaves them
    q, k, v = qkv.split([Hq * D, H * D, H * D], 1)
    return dict(kind="attention", q=q.view(T, Hq, D), k=k.view(T, H, D), v=v.view(T, H, D),
                k_cache=torch.randn(len(pool), H, B, D, device=DEV, generator=g).to(dt),
                v_cache=torch.randn(len(pool), H, B, D, device=DEV, generator=g).to(dt),
                table=_put(table), lengths=_put(lens), offsets=_put(first),
                parents=_put(np.concatenate([parents, np.full(T - total, -1)])), nodes=n, max_len=case["max_len"],
                out=torch.zeros(T, Hq, D, device=DEV, dtype=dt), lse=torch.zeros(T, Hq, device=DEV))


def _prepare_logprobs(case, seed):
    g = _device(seed)
    T, V = case["rows"], case["vocab"]
    z = torch.randn(T, V, device=DEV, generator=g) * 2.5
    z += 6 * torch.rand(T, 1, device=DEV, generator=g)
    tokens = torch.randint(0, V, (T,), device=DEV, generator=g, dtype=torch.int32)
    # half of the tokens are probable ones
    tokens = torch.where(torch.rand(T, device=DEV, generator=g) < 0.5, z.argmax(1).to(torch.int32), tokens)
    if case["masked"]:  # a vocabulary of which a third is not allowed
        z[:, torch.rand(V, device=DEV, generator=g) < 0.33] = -math.inf
        z[:, 1] = 0.0
    z = z.to(TYPES[case["type"]])
    s = dict(kind=case["kind"], logits=z, tokens=tokens)
    if case["kind"] == "logprobs":
        return dict(s, top=case["top"])
    x = z.double()
    s["lse"] = torch.logsumexp(x, 1).float()
    p = torch.softmax(x, 1)
    s["entropy"] = -torch.where(p > 0, p * torch.log(p), 0.0).sum(1).float()
    s["g_logprob"] = torch.randn(T, device=DEV, generator=g)
    s["g_entropy"] = 0.1 * torch.randn(T, device=DEV, generator=g)
    return s


def prepare(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return _prepare_tables(case, seed)
    if kind == "append":
        return _prepare_append(case, seed)
    if kind == "attention":
        return _prepare_attention(case, seed)
    return _prepare_logprobs(case, seed)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------


def _plain_tables(s):
    B, table, free = s["block"], s["table"], s["free"]
    old, new = s["old"].long(), s["new"].long()
    have, want, add = (old + B - 1) // B, (new + B - 1) // B, (new - old).clamp(min=0)
    grow, back = (want - have).clamp(min=0), (have - want).clamp(min=0)
    ends, grown, given = add.cumsum(0), grow.cumsum(0), back.cumsum(0)
    taken, total = grown[-1], ends[-1]
    n_free = len(free) - have.sum()
    # the stack of free blocks with the returned ones on top, in the order of the requests
    at = torch.arange(len(free), device=DEV)
    one = (at - n_free).clamp(min=0)
    r = torch.searchsorted(given, one, right=True).clamp(max=len(old) - 1)
    page = (want[r] + one - (given[r] - back[r])).clamp(0, table.shape[1] - 1)
    stack = torch.where(at < n_free, free, table[r, page])
    top = n_free + given[-1]
    left = top - taken
    # tables
    column = torch.arange(table.shape[1], device=DEV)[None, :]
    fresh = (column >= have[:, None]) & (column < want[:, None])
    nth = (grown - grow)[:, None] + column - have[:, None]
    table.copy_(torch.where(fresh, stack[(top - 1 - nth).clamp(0, len(free) - 1)], table))
    free.copy_(torch.where((at >= n_free) & (at < left), stack, free))
    # slots
    i = torch.arange(len(s["slots"]), device=DEV)
    r = torch.searchsorted(ends, i, right=True).clamp(max=len(old) - 1)
    pos = old[r] + i - (ends[r] - add[r])
    slot = table[r, (pos // B).clamp(max=table.shape[1] - 1)].long() * B + pos % B
    s["slots"].copy_(torch.where(i < total, slot, -1))
    s["offsets"][1:].copy_(ends)
    s["status"].copy_(torch.stack([torch.zeros_like(left), left, total, taken]))
    return s["table"], s["free"], s["offsets"], s["slots"], s["status"]


def _plain_append(s):
    blocks, H, B, D = s["k_cache"].shape
    slots = s["slots"]
    k, v = (s["k"], s["v"]) if s["rows"] is None else (s["k"][s["rows"].long()], s["v"][s["rows"].long()])
    keep = slots >= 0
    slots, k, v = slots[keep], k[keep], v[keep]
    s["k_cache"][slots // B, :, slots % B] = k
    s["v_cache"][slots // B, :, slots % B] = v
    return s["k_cache"], s["v_cache"]


def _plain_attention(s):
    q, k, v, first = s["q"], s["k"], s["v"], s["offsets"].long()
    T, Hq, D = q.shape
    H, B = s["k_cache"].shape[1], s["k_cache"].shape[2]
    G, n, L = Hq // H, s["nodes"], s["max_len"]
    node = torch.arange(n, device=DEV)
    count = first[1:] - first[:-1]
    row = (first[:-1, None] + node).clamp(max=T - 1)
    live = node < count[:, None]
    R = len(row)
    qs = q[row].float().view(R, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(R, H, n * G, D)
    pos = torch.arange(L, device=DEV)
    block = s["table"].long()[:, pos // B]
    kc = s["k_cache"][block, :, pos % B].float().permute(0, 2, 1, 3).contiguous()
    vc = s["v_cache"][block, :, pos % B].float().permute(0, 2, 1, 3).contiguous()
    kn = k[row].float().permute(0, 2, 1, 3).contiguous()
    vn = v[row].float().permute(0, 2, 1, 3).contiguous()
    # a node sees itself and its ancestors: powers of (1 + parent matrix) count the paths
    up = s["parents"].long()[row]
    step = ((up[:, :, None] == node) & live[:, :, None]).double() + torch.eye(n, device=DEV, dtype=torch.float64)
    sees = torch.linalg.matrix_power(step, n) > 0
    sees = sees[:, None, :, None].expand(R, 1, n, G, n).reshape(R, 1, n * G, n)
    cached = (pos < s["lengths"][:, None])[:, None, None]
    a = torch.cat([torch.where(cached, qs @ kc.transpose(2, 3).contiguous(), -math.inf),
                   torch.where(sees, qs @ kn.transpose(2, 3).contiguous(), -math.inf)], 3) / math.sqrt(D)
    top = a.amax(3, keepdim=True)
    p = torch.exp(a - top)
    total = p.sum(3, keepdim=True)
    o = (p[..., :L] @ vc + p[..., L:] @ vn) / total
    lse = top + torch.log(total)
    # back to rows
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(first[1:], t, right=True).clamp(max=R - 1)
    i = (t - first[r]).clamp(max=n - 1)
    o = o.view(R, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(R, n, Hq, D)[r, i]
    lse = lse.view(R, H, n, G).permute(0, 2, 1, 3).reshape(R, n, Hq)[r, i]
    used = t < first[-1]
    s["out"].copy_(torch.where(used[:, None, None], o, s["out"]))
    s["lse"].copy_(torch.where(used[:, None], lse, s["lse"]))
    return s["out"], s["lse"]


def _plain_logprobs(s):
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    logp = z - lse
    entropy = -torch.where(e > 0, (e / total) * logp, 0.0).sum(1)
    given = logp.gather(1, s["tokens"].long()[:, None])[:, 0]
    if not s["top"]:
        return given, entropy, lse[:, 0], logp[:, :0], s["tokens"].view(-1, 1)[:, :0]
    value, index = torch.sort(logp, dim=1, descending=True, stable=True)
    return given, entropy, lse[:, 0], value[:, :s["top"]].contiguous(), index[:, :s["top"]].to(torch.int32)


def _plain_logprobs_grad(s):
    z = s["logits"].float()
    logp = z - s["lse"][:, None]
    p = torch.exp(logp)
    d = -p * s["g_logprob"][:, None]
    d -= torch.where(p > 0, p * (logp + s["entropy"][:, None]), 0.0) * s["g_entropy"][:, None]
    d.scatter_add_(1, s["tokens"].long()[:, None], s["g_logprob"][:, None])
    return d.to(s["logits"].dtype)


def run(s):
    kind = s["kind"]
    if own:
        from paper_2607_08406_amd import lm
        if kind == "tables":
            lm.mca_block_tables(s["old"], s["new"], s["table"], s["free"], s["block"], s["offsets"], s["slots"],
                                s["status"])
            return s["table"], s["free"], s["offsets"], s["slots"], s["status"]
        if kind == "append":
            lm.mca_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], s["rows"])
            return s["k_cache"], s["v_cache"]
        if kind == "attention":
            return lm.mca_tree_attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"],
                                         s["lengths"], s["offsets"], s["parents"], s["nodes"],
                                         max_len=s["max_len"], out=s["out"], lse=s["lse"])
        if kind == "logprobs":
            return tuple(lm.mca_token_logprobs(s["logits"], s["tokens"], s["top"]))
        return lm.mca_token_logprobs_grad(s["logits"], s["tokens"], s["lse"], s["entropy"], s["g_logprob"],
                                          s["g_entropy"])
    if kind == "tables":
        return _plain_tables(s)
    if kind == "append":
        return _plain_append(s)
    if kind == "attention":
        return _plain_attention(s)
    if kind == "logprobs":
        return _plain_logprobs(s)
    return _plain_logprobs_grad(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and the operators' definitions in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "tables":
        new = case["n_req"] * (1 if case["mix"] == "decode" else 9 + min(case["max_len"], 2000) // 9) + 5
        return {"bytes": 12 * case["n_req"] + 8 * new + 8 * new // case["block"], "flops": 0}
    if kind == "append":
        return {"bytes": case["rows"] * (4 * case["kv"] * case["dim"] * BYTES[case["type"]] + 8), "flops": 0}
    if kind == "attention":
        R, el, D = case["n_req"], BYTES[case["type"]], case["dim"]
        cached = R * case["max_len"] * 0.625
        rows = R * max(1.0, 0.75 * case["nodes"])
        per = rows / R * case["heads"] * D
        return {"bytes": int(2 * (cached + rows) * case["kv"] * D * el + 2 * rows * case["heads"] * D * el),
                "flops": int(4 * cached * per)}
    size = case["rows"] * case["vocab"] * BYTES[case["type"]]
    if kind == "logprobs":
        return {"bytes": size + case["rows"] * (16 + 8 * case["top"]), "flops": 6 * case["rows"] * case["vocab"]}
    return {"bytes": 2 * size + 20 * case["rows"], "flops": 8 * case["rows"] * case["vocab"]}


def _exact_attention(case, seed):
    s = prepare(case, seed)
    if case["n_req"] > 600:
        return None
    out, norm = s["out"].double(), s["lse"].double()
    first, lens = s["offsets"].tolist(), s["lengths"].tolist()
    up = s["parents"].tolist()
    B, H = case["block"], case["kv"]
    G = case["heads"] // H
    for r, L in enumerate(lens):
        a, b = first[r], first[r + 1]
        sees = np.zeros((b - a, b - a), bool)
        for i in range(b - a):
            if up[a + i] >= 0:
                sees[i] = sees[up[a + i]]
            sees[i, i] = True
        sees = torch.from_numpy(sees).to(DEV)
        ids = s["table"][r, :-(-L // B)].long()
        for h in range(H):
            keys = torch.cat([s["k_cache"][ids, h].reshape(-1, case["dim"])[:L], s["k"][a:b, h]]).double()
            vals = torch.cat([s["v_cache"][ids, h].reshape(-1, case["dim"])[:L], s["v"][a:b, h]]).double()
            mask = torch.cat([torch.ones(b - a, L, dtype=torch.bool, device=DEV), sees], 1)
            for head in range(h * G, h * G + G):
                x = (s["q"][a:b, head].double() @ keys.T) * case["dim"] ** -0.5
                x = x.masked_fill(~mask, -math.inf)
                norm[a:b, head] = torch.logsumexp(x, 1)
                out[a:b, head] = torch.softmax(x, 1) @ vals
    return out, norm


def exact(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return None  # whole numbers
    if kind == "append":
        s = prepare(case, seed)
        slots = s["slots"].cpu().numpy()
        rows = np.arange(len(slots)) if s["rows"] is None else s["rows"].cpu().numpy()
        to, of = slots[slots >= 0], rows[slots >= 0]
        caches = []
        for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
            c = cache.double().transpose(1, 2).flatten(0, 1)  # [slot][head][dim]
            c[_put(to, torch.int64)] = new.double()[_put(of, torch.int64)]
            caches.append(c.view(cache.shape[0], cache.shape[2], *c.shape[1:]).transpose(1, 2))
        return caches
    if kind == "attention":
        return _exact_attention(case, seed)
    s = prepare(case, seed)
    z = s["logits"].double()
    at = torch.arange(len(z), device=DEV), s["tokens"].long()
    if kind == "logprobs":
        p = torch.softmax(z, 1)
        entropy = torch.special.entr(p).sum(1)
        lse = torch.logsumexp(z, 1)
        best = torch.topk(z, s["top"], 1).values - lse[:, None] if s["top"] else z[:, :0]
        return z[at] - lse, entropy, lse, best, None
    # through autograd of the definition; a row's masked logits have no gradient
    ok = torch.isfinite(z)
    x = torch.where(ok, z, 0.0).requires_grad_()
    logp = torch.log_softmax(x.masked_fill(~ok, -math.inf), 1)
    logq = logp.masked_fill(~ok, 0.0)
    entropy = -(torch.exp(logq) * logq * ok).sum(1)
    pick = logq[at]
    (pick * s["g_logprob"].double() + entropy * s["g_entropy"].double()).sum().backward()
    grad = x.grad.detach()
    # a given token that is masked: the row's other logits still feel its log probability's normalizer
    lost = ~ok[at]
    if bool(lost.any()):
        grad = grad - (lost * s["g_logprob"].double())[:, None] * torch.softmax(z, 1)
        grad[at] += torch.where(lost, s["g_logprob"].double(), 0.0)
    return grad
