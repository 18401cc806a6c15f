"""The calls that draft, verify and keep a cache in 8 bits, as measurable cases.

A case describes one call of one operator on data that the program has on the
GPU (kind):

* append8     rows of keys and values quantised into their places of a cache of
              8-bit values with a scale for each block of tokens and key head
              (mca_cache8_append);
* read8       a request's cached tokens read back in the model's type
              (mca_cache8_read);
* attention8  attention of every request's tree of drafted tokens over its
              tokens in such a cache and over the tree itself
              (mca_tree_attention8);
* verify      which drafted tokens are accepted under the target's
              probabilities, and the token that follows them
              (mca_verify_drafts);
* distill     the loss of a student's logits against a teacher's most probable
              symbols and its gradient (mca_distill, mca_distill_grad).

Inputs are drawn from the seed alone.  With `own` false run() computes the
operators with elementary torch operations in 32 bits (in 64 for verify, whose
tokens hang on the borders between sums); exact() computes them in 64 bits,
written apart from that.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
E4M3 = torch.float8_e4m3fn

# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------


def listed():
    return [
        # The accepted nodes of 64 small drafts of the char-level net (4 heads of 32, fp32).
        dict(name="append8 drafts", kind="append8", type="f32", n_req=64, new=8, kv=4, dim=32, block=16,
             max_len=120, gather=True),
        # The keys and values of a batch of prompts, some of which continue a cached part.
        dict(name="append8 prompts", kind="append8", type="bf16", n_req=32, new=3000, kv=8, dim=128, block=64,
             max_len=2000, gather=False),
        # The char-level net's cached tokens in fp32 again.
        dict(name="read8 char", kind="read8", type="f32", n_req=64, kv=4, dim=32, block=16, max_len=120),
        # Four long contexts that leave for another program's cache.
        dict(name="read8 long", kind="read8", type="bf16", n_req=4, kv=8, dim=128, block=64, max_len=20000),
        # The char-level net (4 heads of 32, at most 128 positions, fp32) on 64 drafts of up to 8 tokens.
        dict(name="attention8 char", kind="attention8", type="f32", n_req=64, nodes=8, heads=4, kv=4, dim=32,
             block=16, max_len=120, chain=False),
        # One token of each of 32 requests with long ragged contexts: the cache is read once.
        dict(name="attention8 decode", kind="attention8", type="bf16", n_req=32, nodes=1, heads=32, kv=8, dim=128,
             block=64, max_len=32768, chain=False),
        # Bushy drafts, 8 query heads to a key head: 384 rows read the same cached tile.
        dict(name="attention8 tree", kind="attention8", type="f16", n_req=16, nodes=48, heads=32, kv=4, dim=128,
             block=16, max_len=16384, chain=False),
        # Chains of four drafted characters behind the last one.
        dict(name="verify char", kind="verify", type="f32", n_req=64, nodes=5, width=1, vocab=65, mode="draft"),
        # Drafted trees with two continuations a node over a large vocabulary.
        dict(name="verify tree", kind="verify", type="bf16", n_req=32, nodes=9, width=2, vocab=128000, mode="draft"),
        # Chains that were looked up, not drawn, an odd vocabulary.
        dict(name="verify lookup", kind="verify", type="f16", n_req=16, nodes=7, width=1, vocab=50001, mode="given"),
        # A training batch of the char-level net (64 sequences of 128, 65 symbols) under a larger one.
        dict(name="distill char", kind="distill", type="f32", rows=8192, vocab=65, top=5, rest=False, scale=0.5,
             masked=False),
        # A batch over a large vocabulary, the teacher's other symbols as one.
        dict(name="distill large", kind="distill", type="bf16", rows=4096, vocab=50001, top=20, rest=True, scale=1.0,
             masked=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append8", "append8", "read8", "attention8", "attention8", "attention8", "verify", "verify",
                       "verify", "distill", "distill"])
    typ = rng.choice(["f32", "bf16", "bf16", "f16"])
    kv = rng.choice([1, 2, 3, 4, 8])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
    block = rng.choice([8, 16, 16, 20, 32, 50, 64, 128])
    if kind == "append8":
        R = _log(rng, 1, 300)
        most = 40e6 / (R * kv * dim)
        return dict(kind=kind, type=typ, n_req=R, new=max(1, min(rng.choice([1, _log(rng, 2, 16), _log(rng, 16, 3000)]),
                                                                  int(most))),
                    kv=kv, dim=dim, block=block, max_len=max(1, min(_log(rng, 10, 10000), int(most))),
                    gather=rng.random() < 0.5)
    if kind == "read8":
        R = _log(rng, 1, 200)
        return dict(kind=kind, type=typ, n_req=R, kv=kv, dim=dim, block=block,
                    max_len=max(1, min(_log(rng, 10, 50000), int(60e6 / (R * kv * dim)))))
    if kind == "attention8":
        group = rng.choice([1, 1, 2, 4, 5, 8])
        nodes = rng.choice([1, _log(rng, 2, 16), _log(rng, 16, 128)])
        max_len = _log(rng, 30, 100000)
        # the cached values of a case, and the rows that read them, stay under the listed ones'
        most = min(200e6 / (max_len * kv * dim), 30e9 / (4.0 * max_len * nodes * kv * group * dim), 512)
        if most < 1:
            max_len = int(max_len * most)
            most = 1
        return dict(kind=kind, type=typ, n_req=max(1, min(_log(rng, 1, 200), int(most))), nodes=nodes,
                    heads=kv * group, kv=kv, dim=dim, block=block, max_len=max(max_len, 16),
                    chain=rng.random() < 0.25)
    vocab = rng.choice([65, _log(rng, 40, 1000), _log(rng, 1000, 130000), _log(rng, 20000, 130000)])
    if kind == "verify":
        nodes = rng.choice([1, 2, _log(rng, 2, 16), _log(rng, 3, 48)])
        return dict(kind=kind, type=typ, n_req=max(1, min(_log(rng, 1, 200), 30000000 // (nodes * vocab))),
                    nodes=nodes, width=rng.choice([1, 1, 2, 3, 4]), vocab=vocab,
                    mode=rng.choice(["draft", "draft", "given", "greedy"]))
    rest = rng.random() < 0.5
    return dict(kind=kind, type=typ, rows=max(1, min(_log(rng, 1, 20000), 100000000 // vocab)), vocab=vocab,
                top=rng.choice([1, 5, 8, 20, 32]), rest=rest, scale=1.0 if rest else rng.choice([1.0, 0.5, 0.25]),
                masked=rng.random() < 0.3)


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------


def _host(seed):
    return np.random.default_rng([seed, 17])


def _device(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    return g


def _put(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def _paged(rng, blocks_of, width):
    """A table of the given numbers of blocks, taken in random order from a pool that has `width` for each request
    and three more; how many blocks that are."""
    blocks = len(blocks_of) * width + 3
    table = np.zeros((len(blocks_of), width), np.int32)
    held = np.arange(width)[None, :] < blocks_of[:, None]
    table[held] = rng.permutation(blocks)[:int(blocks_of.sum())]
    return table, blocks


def _cache8(g, blocks, H, B, D):
    """A pool of blocks that hold normal values of about 1, and their scales (2^-7 to 2^-5)."""
    caches, scales = [], []
    for _ in range(2):
        code = torch.empty(blocks, H, B, D, dtype=E4M3, device=DEV)
        scale = torch.randint(120, 123, (blocks, H), device=DEV, generator=g, dtype=torch.int32)
        for b in range(0, blocks, 4096):
            part = scale[b:b + 4096]
            x = torch.randn(len(part), H, B, D, device=DEV, generator=g)
            code[b:b + 4096] = torch.ldexp(x, 127 - part[:, :, None, None]).clamp(-448, 448).to(E4M3)
        caches.append(code)
        scales.append(scale.to(torch.uint8))
    return dict(k_cache=caches[0], v_cache=caches[1], k_scale=scales[0], v_scale=scales[1])


def _prepare_append8(case, seed):
    rng, g = _host(seed), _device(seed)
    R, H, D, B, dt = case["n_req"], case["kv"], case["dim"], case["block"], TYPES[case["type"]]
    old = rng.integers(0, case["max_len"] + 1, R)
    old[rng.random(R) < 0.4] = 0  # requests that begin
    new = rng.integers(max(1, case["new"] // 3), case["new"] + 1, R)
    new[rng.random(R) < 0.05] = 0  # and such that wait
    new[rng.integers(0, R)] = case["new"]
    first = np.concatenate([[0], np.cumsum(new)])
    table, blocks = _paged(rng, -(-(old + new) // B), -(-(case["max_len"] + case["new"]) // B))
    n = int(first[-1])
    src = n + n // 2 if case["gather"] else n
    qkv = torch.randn(src, 3, H, D, device=DEV, generator=g)  # as a projection leaves them
    qkv *= torch.exp(torch.randn(src, 1, 1, 1, device=DEV, generator=g) * 0.3)
    qkv = qkv.to(dt)
    return dict(_cache8(g, blocks, H, B, D), kind="append8", k=qkv[:, 1], v=qkv[:, 2], table=_put(table),
                lengths=_put(old), offsets=_put(first), rows=_put(rng.permutation(src)[:n]) if case["gather"] else None)


def _prepare_read8(case, seed):
    rng, g = _host(seed), _device(seed)
    R, H, D, B, dt = case["n_req"], case["kv"], case["dim"], case["block"], TYPES[case["type"]]
    lens = rng.integers(max(1, case["max_len"] // 2), case["max_len"] + 1, R)
    lens[rng.integers(0, R)] = case["max_len"]
    start = np.where(rng.random(R) < 0.3, rng.integers(0, lens), 0)  # some go on from where they were
    first = np.concatenate([[0], np.cumsum(lens - start)])
    table, blocks = _paged(rng, -(-lens // B), -(-case["max_len"] // B))
    T = R * case["max_len"] + 2  # rows behind the last request stay as they were
    return dict(_cache8(g, blocks, H, B, D), kind="read8", table=_put(table), start=_put(start), offsets=_put(first),
                k=torch.zeros(T, H, D, dtype=dt, device=DEV), v=torch.zeros(T, H, D, dtype=dt, device=DEV))


def _prepare_attention8(case, seed):
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
    table, blocks = _paged(rng, -(-lens // B), -(-case["max_len"] // B))
    T = R * n + 3  # a step has room for whole drafts: rows behind the last request
    qkv = torch.randn(T, (Hq + 2 * H) * D, device=DEV, generator=g).to(dt)  # as a projection leaves them
    q, k, v = qkv.split([Hq * D, H * D, H * D], 1)
    return dict(_cache8(g, blocks, H, B, D), kind="attention8", q=q.view(T, Hq, D), k=k.view(T, H, D),
                v=v.view(T, H, D), table=_put(table), lengths=_put(lens), offsets=_put(first),
                parents=_put(np.concatenate([parents, np.full(T - total, -1)])), nodes=n, max_len=case["max_len"],
                out=torch.zeros(T, Hq, D, device=DEV, dtype=dt), lse=torch.zeros(T, Hq, device=DEV))


def _prepare_verify(case, seed):
    rng, g = _host(seed), _device(seed)
    R, n, W, V, dt = case["n_req"], case["nodes"], case["width"], case["vocab"], TYPES[case["type"]]
    nodes = rng.integers(max(1, n // 2), n + 1, R)
    nodes[rng.integers(0, R)] = n
    first = np.concatenate([[0], np.cumsum(nodes)])
    total = int(first[-1])
    T = R * n + 2  # a step has room for whole drafts: rows behind the last request
    at = np.arange(T) - np.concatenate([np.repeat(first[:-1], nodes), [total] * (T - total)])
    parents = np.where((at == 0) | (np.arange(T) >= total), -1, (at - 1) // W)
    # the draft's logits, and the target's, which differ somewhat
    draft = torch.randn(T, V, device=DEV, generator=g) * 3
    target = (draft + torch.randn(T, V, device=DEV, generator=g) * 0.6).to(dt)
    draft = draft.to(dt)
    # a node's token is drawn from the draft's distribution at its parent
    up = _put(np.where(parents < 0, np.arange(T), np.arange(T) - at + parents), torch.int64)
    z = (target if case["mode"] == "greedy" else draft)[up].float() * 0.9
    for b in range(0, T, 64):
        u = torch.rand(len(z[b:b + 64]), V, device=DEV, generator=g).clamp(min=1e-20)
        z[b:b + 64] -= torch.log(-torch.log(u)) * (0.3 if case["mode"] == "greedy" else 1.0)
    return dict(kind="verify", target=target, draft=draft if case["mode"] == "draft" else None,
                greedy=case["mode"] == "greedy", tokens=z.argmax(1).to(torch.int32), parents=_put(parents),
                offsets=_put(first), lengths=_put(rng.integers(0, 5000, R)), nodes=n, width=W,
                accept=torch.rand(T, device=DEV, generator=g), sample=torch.rand(R, device=DEV, generator=g),
                scale=0.9, draft_scale=0.9)


def _prepare_distill(case, seed):
    g = _device(seed)
    T, V, K = case["rows"], case["vocab"], case["top"]
    z = torch.randn(T, V, device=DEV, generator=g) * 2.5
    z += 4 * torch.rand(T, 1, device=DEV, generator=g)
    teacher = z + torch.randn(T, V, device=DEV, generator=g) * 0.7
    if case["masked"]:  # a vocabulary of which a third is not allowed
        gone = torch.rand(V, device=DEV, generator=g) < 0.33
        gone[:K] = False
        z[:, gone] = -math.inf
        teacher[:, gone] = -math.inf
    logp, ids = torch.topk(torch.log_softmax(teacher, 1), K, dim=1)
    ids = ids.to(torch.int32)
    ids[torch.rand(T, device=DEV, generator=g) < 0.03] = -1  # rows behind a sequence's end have no teacher
    return dict(kind="distill", logits=z.to(TYPES[case["type"]]), logprob=logp.contiguous(), ids=ids,
                rest=case["rest"], scale=case["scale"], grad=torch.rand(T, device=DEV, generator=g) / T)


def prepare(case, seed):
    return {"append8": _prepare_append8, "read8": _prepare_read8, "attention8": _prepare_attention8,
            "verify": _prepare_verify, "distill": _prepare_distill}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------


def _plain_append8(s):
    table, old, first = s["table"].long(), s["lengths"].long(), s["offsets"].long()
    blocks, H, B, D = s["k_cache"].shape
    n, dt = int(s["k"].shape[0]) if s["rows"] is None else len(s["rows"]), s["k"].dtype
    i = torch.arange(n, device=DEV)
    r = torch.searchsorted(first[1:], i, right=True)
    pos = old[r] + i - first[r]
    block = table[r, pos // B]
    # the block in which a request goes on behind tokens of its own
    live = (old % B > 0) & (first[1:] > first[:-1])
    kept = torch.zeros(blocks, dtype=torch.int64, device=DEV)
    part = table.gather(1, (old // B).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    kept.index_add_(0, part, torch.where(live, old % B, 0))
    touched = torch.zeros(blocks, dtype=torch.bool, device=DEV)
    touched[block] = True
    lowest, highest = (-15, 8) if dt == torch.float16 else (-100, 120)
    for x, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        x = (x if s["rows"] is None else x[s["rows"].long()]).float()
        size = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(2)
        top = torch.zeros(blocks, H, device=DEV).scatter_reduce_(0, block[:, None].expand(n, H), size, "amax")
        m, e = torch.frexp(top)
        e = torch.where(top > 0, e - 9 + (m > 0.875).to(torch.int32), lowest).clamp(min=lowest)
        before = scale.to(torch.int32) - 127
        e = torch.where(touched[:, None], torch.where(kept[:, None] > 0, torch.maximum(e, before), e), before)
        # the tokens that stay, in the new scale
        again = cache[part].float() * torch.exp2((before - e)[part].float())[:, :, None, None]
        stays = (live[:, None] & (torch.arange(B, device=DEV) < (old % B)[:, None]))[:, None, :, None]
        some = torch.where(stays, again.to(E4M3).float(), cache[part].float()).to(E4M3)
        cache[part[live]] = some[live]
        y = torch.ldexp(x, -e[block][:, :, None])
        most = torch.where(e[block] >= highest, 240.0, 448.0)[:, :, None]
        y = torch.where(torch.isfinite(x), torch.minimum(torch.maximum(y, -most), most), math.nan)
        cache[block, :, pos % B] = y.to(E4M3)
        scale.copy_((e + 127).to(torch.uint8))
    return s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]


def _plain_read8(s):
    table, start, first = s["table"].long(), s["start"].long(), s["offsets"].long()
    B = s["k_cache"].shape[2]
    i = torch.arange(len(s["k"]), device=DEV)
    r = torch.searchsorted(first[1:], i, right=True).clamp(max=len(start) - 1)
    pos = (start[r] + i - first[r]).clamp(max=table.shape[1] * B - 1)
    block = table[r, pos // B]
    used = (i < first[-1])[:, None, None]
    for out, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        x = cache[block, :, pos % B].float() * torch.exp2(scale[block].float() - 127)[:, :, None]
        out.copy_(torch.where(used, x, out))
    return s["k"], s["v"]


def _plain_attention8(s):
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
    # [R, H, L, D] of the request's tokens, in the values that they stand for
    kc = (s["k_cache"][block, :, pos % B].float() * torch.exp2(s["k_scale"][block].float() - 127)[..., None])
    kc = kc.permute(0, 2, 1, 3).contiguous()
    vc = (s["v_cache"][block, :, pos % B].float() * torch.exp2(s["v_scale"][block].float() - 127)[..., None])
    vc = vc.permute(0, 2, 1, 3).contiguous()
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


def _plain_verify(s):
    first, tokens = s["offsets"].long(), s["tokens"].long()
    T, V = s["target"].shape
    R = len(first) - 1
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(first[1:], t, right=True).clamp(max=R - 1)
    root = t == first[r]
    drafted = (t < first[-1]) & ~root
    up = torch.where(drafted, first[r] + s["parents"].long(), t)
    p = torch.softmax(s["target"].double() * (1.0 if s["greedy"] else s["scale"]), 1)
    accepted = torch.zeros(T, dtype=torch.bool, device=DEV)
    open_ = torch.ones(T, dtype=torch.bool, device=DEV)  # none of a node's children has been accepted
    left = p.clone()  # what a node's further children and its token are drawn from, up to its sum
    if s["greedy"]:
        best = s["target"].argmax(1)
    if s["draft"] is not None:
        q = torch.softmax(s["draft"].double() * s["draft_scale"], 1)
    nth = (t - first[r] - 1) % s["width"]  # among its parent's children
    u = s["accept"].double()
    for k in range(s["width"]):
        now = drafted & (nth == k)
        if s["greedy"]:
            ok = now & open_[up] & (tokens == best[up])
        elif s["draft"] is not None:
            total = left.sum(1)
            ok = now & open_[up] & (u * total[up] * q[up, tokens] < left[up, tokens])
        else:
            total = left.sum(1)
            ok = now & open_[up] & (u * total[up] < left[up, tokens])
        accepted |= ok
        open_[up[ok]] = False
        lost = torch.zeros(T, dtype=torch.bool, device=DEV)
        lost[up[now & open_[up]]] = True
        if s["greedy"]:
            continue
        if s["draft"] is not None:  # max(left - total q, 0)
            left = torch.where(lost[:, None], (left - total[:, None] * q).clamp(min=0), left)
        else:
            gone = now & open_[up]
            left[up[gone], tokens[gone]] = 0.0
    # the path: nodes whose ancestors are all accepted
    n = s["nodes"]
    node = torch.arange(n, device=DEV)
    row = (first[:-1, None] + node).clamp(max=T - 1)
    here = node < (first[1:] - first[:-1])[:, None]
    above = ((up[row] - first[:-1, None])[:, :, None] == node) & (node > 0)[:, None] & here[:, :, None]
    step = above.double() + torch.eye(n, device=DEV, dtype=torch.float64)
    sees = torch.linalg.matrix_power(step, n) > 0
    fine = (accepted | root)[row] & here
    path = fine & ~(sees & ~fine[:, None, :]).any(2)
    count = path.sum(1)
    depth = torch.where(path, sees.sum(2), 0)
    last = first[:-1] + depth.argmax(1)
    if s["greedy"]:
        token = best[last]
    else:
        w = left[last]
        w = torch.where(w.sum(1, keepdim=True) > 0, w, p[last])
        ends = w.cumsum(1)
        token = (ends <= s["sample"].double()[:, None] * ends[:, -1:]).sum(1).clamp(max=V - 1)
    rows = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    starts = count.cumsum(0) - count
    at = torch.where(path, starts[:, None] + path.cumsum(1) - 1, T)
    rows = torch.cat([rows, rows[:1]]).scatter_(0, at.reshape(-1), row.to(torch.int32).reshape(-1))[:T]
    return (s["lengths"] + count).to(torch.int32), rows.contiguous(), token.to(torch.int32)


def _plain_distill(s):
    z, ids, rest = s["logits"].float() * s["scale"], s["ids"].long(), s["rest"]
    T, V = z.shape
    # the loss is what large terms leave: sums in 64 bits
    here = (ids >= 0) & (ids < V)
    at = torch.where(here, ids, 0)
    lse = torch.logsumexp(z.double(), 1)
    t = torch.where(here, s["logprob"].double() * s["scale"], -math.inf)
    if not rest:
        t = t - torch.logsumexp(t, 1, keepdim=True)
    q = torch.where(here, torch.exp(t), 0.0)
    q = torch.where(here.any(1, keepdim=True), q, 0.0)
    logs = z.gather(1, at).double() - lse[:, None]
    loss = torch.where(q > 0, q * (t - logs), 0.0).sum(1)
    p = torch.exp(z - lse.float()[:, None])
    total, lse_rest = q.sum(1), lse[:0]
    if rest:
        known = torch.zeros(T, V + 1, dtype=torch.bool, device=DEV)
        known.scatter_(1, torch.where(here, ids, V), True)
        lse_rest = torch.logsumexp(torch.where(known[:, :V], -math.inf, z.double()), 1)
        left = (1 - total).clamp(min=0)
        loss = loss + torch.where(left > 0, left * (torch.log(left) - (lse_rest - lse)), 0.0)
        total = total + left
        less = torch.where(left > 0, left * torch.exp(lse - lse_rest), 0.0)
        known = known[:, :V]
        d = torch.where(known, p * total.float()[:, None], p * (total - less).float()[:, None])
    else:
        d = p * total.float()[:, None]
    d = d.scatter_add(1, at, -q.float())
    d = d * (s["grad"] * s["scale"])[:, None]
    return loss.float(), lse.float(), lse_rest.float(), d.to(s["logits"].dtype)


def run(s):
    kind = s["kind"]
    if own:
        from paper_2607_08406_amd import lm
        if kind == "append8":
            lm.mca_cache8_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"],
                                 s["lengths"], s["offsets"], s["rows"])
            return s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
        if kind == "read8":
            return lm.mca_cache8_read(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                                      s["table"], s["start"], s["offsets"])
        if kind == "attention8":
            return lm.mca_tree_attention8(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"],
                                          s["v_scale"], s["table"], s["lengths"], s["offsets"], s["parents"],
                                          s["nodes"], max_len=s["max_len"], out=s["out"], lse=s["lse"])
        if kind == "verify":
            return tuple(lm.mca_verify_drafts(s["target"], s["draft"], s["tokens"], s["parents"], s["offsets"],
                                              s["lengths"], s["nodes"], s["accept"], s["sample"], scale=s["scale"],
                                              draft_scale=s["draft_scale"], greedy=s["greedy"]))
        d = lm.mca_distill(s["logits"], s["logprob"], s["ids"], rest=s["rest"], scale=s["scale"])
        grad = lm.mca_distill_grad(s["logits"], s["logprob"], s["ids"], d.lse, d.lse_rest, s["grad"], rest=s["rest"],
                                   scale=s["scale"])
        return d.loss, d.lse, d.lse_rest, grad
    if kind == "append8":
        return _plain_append8(s)
    if kind == "read8":
        return _plain_read8(s)
    if kind == "attention8":
        return _plain_attention8(s)
    if kind == "verify":
        return _plain_verify(s)
    return _plain_distill(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and the operators' definitions in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    kind, el = case["kind"], BYTES[case["type"]]
    if kind == "append8":
        rows = case["n_req"] * (0.63 * case["new"] + 0.3)
        return {"bytes": int(2 * rows * case["kv"] * case["dim"] * (el + 1) + 12 * case["n_req"]), "flops": 0}
    if kind == "read8":
        rows = case["n_req"] * case["max_len"] * 0.64
        return {"bytes": int(2 * rows * case["kv"] * case["dim"] * (el + 1) + 8 * case["n_req"]), "flops": 0}
    if kind == "attention8":
        R, D = case["n_req"], case["dim"]
        cached = R * case["max_len"] * 0.625
        rows = R * max(1.0, 0.75 * case["nodes"])
        per = rows / R * case["heads"] * D
        return {"bytes": int(2 * (cached + rows * el) * case["kv"] * D + 2 * rows * case["heads"] * D * el),
                "flops": int(4 * cached * per)}
    if kind == "verify":
        rows = case["n_req"] * max(1.0, 0.75 * case["nodes"])
        size = rows * case["vocab"] * el * (2 if case["mode"] == "draft" else 1)
        return {"bytes": int(size + 16 * rows + 16 * case["n_req"]), "flops": int(3 * size / el)}
    size = case["rows"] * case["vocab"] * el
    return {"bytes": 3 * size + case["rows"] * (16 * case["top"] + 20), "flops": 12 * case["rows"] * case["vocab"]}


def _exact_append8(case, seed):
    s = prepare(case, seed)
    B = case["block"]
    old, first, table = s["lengths"].tolist(), s["offsets"].tolist(), s["table"].tolist()
    low = -15 if case["type"] == "f16" else -100
    out = []
    for x, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        x = (x if s["rows"] is None else x[s["rows"].long()]).double()
        code, byte = cache.double(), scale.double()
        for r, a in enumerate(old):
            end = a + first[r + 1] - first[r]
            page = a // B
            while page * B < end and end > a:
                lo, hi, b = max(a, page * B), min(end, page * B + B), table[r][page]
                part = x[first[r] + lo - a:first[r] + hi - a].transpose(0, 1)  # [H, tokens, D]
                e = torch.ceil(torch.log2(part.abs().amax((1, 2)) / 448)).clamp(min=low)
                keep = lo - page * B
                if keep:
                    e = torch.maximum(e, byte[b] - 127)
                    code[b, :, :keep] *= torch.exp2(byte[b] - 127 - e)[:, None, None]
                code[b, :, keep:hi - page * B] = part * torch.exp2(-e)[:, None, None]
                byte[b] = e + 127
                page += 1
        out.append(code)
    return out[0], out[1], None, None


def _values8(s, which, ids):
    """[blocks, H, B, D] of a table's blocks in 64 bits."""
    scale = torch.exp2(s[which + "_scale"][ids].double() - 127)
    return s[which + "_cache"][ids].double() * scale[:, :, None, None]


def _exact_read8(case, seed):
    s = prepare(case, seed)
    out = s["k"].double(), s["v"].double()
    start, first = s["start"].tolist(), s["offsets"].tolist()
    for r, a in enumerate(start):
        n = first[r + 1] - first[r]
        ids = s["table"][r, :-(-(a + n) // case["block"])].long()
        for o, which in zip(out, "kv"):
            x = _values8(s, which, ids).transpose(1, 2).flatten(0, 1)  # [token, H, D]
            o[first[r]:first[r + 1]] = x[a:a + n]
    return out


def _exact_attention8(case, seed):
    s = prepare(case, seed)
    out, norm = s["out"].double(), s["lse"].double()
    first, lens = s["offsets"].tolist(), s["lengths"].tolist()
    up = s["parents"].tolist()
    H = case["kv"]
    G = case["heads"] // H
    for r, L in enumerate(lens):
        a, b = first[r], first[r + 1]
        sees = np.zeros((b - a, b - a), bool)
        for i in range(b - a):
            if up[a + i] >= 0:
                sees[i] = sees[up[a + i]]
            sees[i, i] = True
        mask = torch.cat([torch.ones(b - a, L, dtype=torch.bool, device=DEV), torch.from_numpy(sees).to(DEV)], 1)
        ids = s["table"][r, :-(-L // case["block"])].long()
        cached = [_values8(s, which, ids).transpose(0, 1).flatten(1, 2)[:, :L] for which in "kv"]
        for h in range(H):
            keys = torch.cat([cached[0][h], s["k"][a:b, h].double()])
            vals = torch.cat([cached[1][h], s["v"][a:b, h].double()])
            for head in range(h * G, h * G + G):
                x = (s["q"][a:b, head].double() @ keys.T) * case["dim"] ** -0.5
                x = x.masked_fill(~mask, -math.inf)
                norm[a:b, head] = torch.logsumexp(x, 1)
                out[a:b, head] = torch.softmax(x, 1) @ vals
    return out, norm


def _exact_distill(case, seed):
    """Through autograd of the definition, masked logits left out; the teacher's symbols of a row differ."""
    s = prepare(case, seed)
    T, V = s["logits"].shape
    parts = []
    for a in range(0, T, 256):
        z = s["logits"][a:a + 256].double()
        ok = torch.isfinite(z)
        x = torch.where(ok, z, 0.0).requires_grad_()
        logp = torch.log_softmax((x * case["scale"]).masked_fill(~ok, -math.inf), 1)
        lse = torch.logsumexp((z * case["scale"]), 1)
        ids = s["ids"][a:a + 256].long()
        none = ids[:, :1] < 0  # a row has all of its teacher's symbols or none
        pick = logp.gather(1, ids.clamp(min=0))
        t = s["logprob"][a:a + 256].double() * case["scale"]
        if case["rest"]:
            q = torch.exp(t)
            other = (1 - q.sum(1)).clamp(min=0)
            outside = torch.ones_like(z).scatter_(1, ids.clamp(min=0), 0.0).bool() & ok
            outside = torch.where(none, ok, outside)
            lrest = torch.logsumexp(logp.masked_fill(~outside, -math.inf), 1)
            log_other = torch.where(other > 0, torch.log(other.clamp(min=1e-300)), 0.0)
            loss = (q * (t - pick)).sum(1) + torch.where(other > 0, other * (log_other - lrest), 0.0)
        else:
            t = torch.log_softmax(t, 1)
            loss = (torch.exp(t) * (t - pick)).sum(1)
            lrest = loss[:0]
        loss = torch.where(none[:, 0], 0.0, loss)
        (loss * s["grad"][a:a + 256].double()).sum().backward()
        parts.append((loss.detach(), lse, (lrest + lse).detach() if case["rest"] else lrest.detach(), x.grad))
    return [torch.cat(p) for p in zip(*parts)]


def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None  # whole numbers
    return {"append8": _exact_append8, "read8": _exact_read8, "attention8": _exact_attention8,
            "distill": _exact_distill}[kind](case, seed)
