"""fp64 oracle of the language-model operators: a paged cache of keys and
values, the attention of drafted tokens over it, and token log probabilities.

Plain loops over requests and rows, from the operators' definitions.
"""
from __future__ import annotations

import numpy as np


def ceil_div(a, b):
    return -(-a // b)


def block_tables(old, new, table, free, block, max_tokens):
    """(table, free, offsets, slots, status) after the requests went from old to new tokens."""
    table, free = table.copy(), free.copy()
    R, width, n_blocks = len(old), table.shape[1], len(free)
    fail = np.zeros(R + 1, np.int32), np.full(max_tokens, -1, np.int64)
    lens = np.concatenate([old, new])
    held = sum(ceil_div(int(n), block) for n in old)
    n_free = n_blocks - held
    bad = bool((lens < 0).any() or (lens > width * block).any())
    if bad or held > n_blocks:
        return table, free, *fail, (2, None, 0, 0)
    if sum(max(int(b) - int(a), 0) for a, b in zip(old, new)) > max_tokens:
        return table, free, *fail, (3, n_free, 0, 0)
    stack = list(free[:n_free])
    for r in range(R):
        for page in range(ceil_div(int(new[r]), block), ceil_div(int(old[r]), block)):
            stack.append(table[r, page])
    need = sum(max(0, ceil_div(int(b), block) - ceil_div(int(a), block)) for a, b in zip(old, new))
    if need > len(stack):
        return table, free, *fail, (1, n_free, 0, 0)
    offsets, slots = [0], []
    for r in range(R):
        for page in range(ceil_div(int(old[r]), block), ceil_div(int(new[r]), block)):
            table[r, page] = stack.pop()
        for t in range(int(old[r]), int(new[r])):
            slots.append(int(table[r, t // block]) * block + t % block)
        offsets.append(len(slots))
    free[n_free:max(n_free, len(stack))] = stack[n_free:]
    out = np.full(max_tokens, -1, np.int64)
    out[:len(slots)] = slots
    return table, free, np.array(offsets, np.int32), out, (0, len(stack), len(slots), need)


def sees(parents):
    """[n, n]: whether node i sees node j (itself and its ancestors)."""
    n = len(parents)
    out = np.zeros((n, n), bool)
    for i in range(n):
        if 0 <= parents[i] < i:
            out[i] = out[parents[i]]
        out[i, i] = True
    return out


def cached_rows(cache, table_row, length, h):
    """Keys or values [m, dim] of a request's cached tokens that are there, in order."""
    n_blocks, _, block, _ = cache.shape
    rows = []
    for t in range(min(length, len(table_row) * block)):
        b = table_row[t // block]
        if 0 <= b < n_blocks:
            rows.append(cache[b, h, t % block])
    return np.array(rows, np.float64).reshape(-1, cache.shape[3])


def tree_attention(q, k, v, k_cache, v_cache, table, lengths, offsets, parents, scale):
    """{(row, head): (out, lse, scores, |p| |v|, sum |v|, sum |q k| max)} of every node's row."""
    res = {}
    group = q.shape[1] // k.shape[1]
    for r in range(len(lengths)):
        a, b = int(offsets[r]), int(offsets[r + 1])
        vis = sees(parents[a:b])
        for h in range(k.shape[1]):
            kc = cached_rows(k_cache, table[r], int(lengths[r]), h)
            vc = cached_rows(v_cache, table[r], int(lengths[r]), h)
            for i in range(b - a):
                keys = np.concatenate([kc, k[a:b, h][vis[i]].astype(np.float64)])
                vals = np.concatenate([vc, v[a:b, h][vis[i]].astype(np.float64)])
                for g in range(group):
                    x = q[a + i, h * group + g].astype(np.float64)
                    s = scale * (keys @ x)
                    top = s.max()
                    e = np.exp(s - top)
                    p = e / e.sum()
                    size = abs(scale) * (np.abs(keys) @ np.abs(x)).max()
                    with np.errstate(invalid="ignore"):
                        res[a + i, h * group + g] = (p @ vals, top + np.log(e.sum()), p @ np.abs(vals),
                                                     np.abs(vals).sum(0), size, len(s))
    return res


def token_logprobs(z, tokens):
    """(logprob, entropy, lse, log p) of logits z [T, V]; a token outside the vocabulary gives 0."""
    z = np.asarray(z, np.float64)
    T, V = z.shape
    lse, ent, lp = np.empty(T), np.empty(T), np.empty(T)
    logp = np.empty((T, V))
    for t in range(T):
        top = z[t].max()
        if top == -np.inf:
            lse[t], ent[t], logp[t] = -np.inf, 0.0, -np.inf
        else:
            norm = np.log(np.exp(z[t] - top).sum())
            lse[t] = top + norm
            logp[t] = (z[t] - top) - norm  # also where top is too large for its sum with norm
            fin = logp[t] > -np.inf
            ent[t] = -(np.exp(logp[t][fin]) * logp[t][fin]).sum()
        lp[t] = logp[t, tokens[t]] if 0 <= tokens[t] < V else 0.0
    return lp, ent, lse, logp


def top(z, n):
    """Symbols of the n largest logits of each row, equal ones by rising symbol."""
    return np.argsort(-np.asarray(z, np.float64), axis=1, kind="stable")[:, :n]


def token_logprobs_grad(z, tokens, lse, entropy, g, ge):
    """Gradient of sum g logprob + ge entropy with lse and entropy as given."""
    z = np.asarray(z, np.float64)
    out = np.zeros(z.shape)
    for t in range(len(z)):
        if lse[t] == -np.inf:
            continue
        gt = g[t] if 0 <= tokens[t] < z.shape[1] else 0.0
        fin = z[t] > -np.inf
        lp = z[t][fin] - float(lse[t])
        p = np.exp(lp)
        out[t][fin] = -p * (gt + ge[t] * (lp + float(entropy[t])))
        if gt != 0.0:
            out[t, tokens[t]] += gt
    return out
