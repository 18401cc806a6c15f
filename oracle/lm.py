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


# ---------------------------------------------------------------------------
# a cache of 8-bit values, verification of drafts, distillation
# ---------------------------------------------------------------------------

def e4m3(x):
    """The nearest values of 8-bit floats of 4 exponent and 3 mantissa bits (ties to even); |x| <= 448, or NaN."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.where(np.isfinite(x) & (x != 0), x, 1.0))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)  # of the value's power of two, or of the subnormal ones
    return np.where(np.isfinite(x), np.rint(x / step) * step, np.nan)


def e4m3_value(code):
    """The values of codes (uint8)."""
    c = np.asarray(code, np.uint8).astype(np.int64)
    m, e = c & 7, (c >> 3) & 15
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    return np.where((c & 127) == 127, np.nan, np.where(c >> 7, -x, x))


def e4m3_code(x):
    """The codes of values that e4m3 holds (a NaN's sign is 0)."""
    table = e4m3_value(np.arange(127, dtype=np.uint8))
    at = np.searchsorted(table, np.abs(np.where(np.isnan(x), 0, x)))
    return np.where(np.isnan(x), 127, at + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


LOWEST_EXP = {"f32": -100, "bf16": -100, "f16": -15}
CLAMPED_EXP = {"f32": 120, "bf16": 120, "f16": 8}  # where 256 times the scale is past the type's largest


def cache8_exp(top, typ):
    """The exponent of the smallest scale under which values of up to `top` are at most 448."""
    e = LOWEST_EXP[typ]
    while top > 448 * 2.0 ** e:
        e += 1
    return e


def cache8_append(k, v, k_cache, v_cache, k_scale, v_scale, table, lengths, offsets, rows, typ):
    """(k_cache, v_cache, k_scale, v_scale) after the append; caches hold codes, scales biased exponents (uint8)."""
    block, n_blocks = k_cache.shape[2], k_cache.shape[0]
    out = []
    for x, cache, scale in ((k, k_cache, k_scale), (v, v_cache, v_scale)):
        cache, scale = cache.copy(), scale.copy()
        for r, old in enumerate(lengths):
            old, a, b = int(old), int(offsets[r]), int(offsets[r + 1])
            if old < 0 or a < 0 or b <= a or b > (len(k) if rows is None else len(rows)):
                continue
            pages = {}
            for i in range(a, b):
                pages.setdefault((old + i - a) // block, []).append(i)
            for page, those in pages.items():
                if page >= table.shape[1] or not 0 <= table[r, page] < n_blocks:
                    continue
                blk = int(table[r, page])
                src = [i if rows is None else int(rows[i]) for i in those]
                keep = max(0, old - page * block)
                for h in range(cache.shape[1]):
                    new = np.array([x[s, h] if 0 <= s < len(x) else np.zeros(cache.shape[3]) for s in src], np.float64)
                    fin = np.isfinite(new)
                    e = cache8_exp(np.abs(new[fin]).max(initial=0.0), typ)
                    if keep:
                        before = min(max(int(scale[blk, h]), 1), 254) - 127
                        e = max(e, before)
                        if e > before:
                            kept = e4m3(e4m3_value(cache[blk, h, :keep]) * 2.0 ** (before - e))
                            cache[blk, h, :keep] = np.where(np.isnan(kept), cache[blk, h, :keep], e4m3_code(kept))
                    t = 2.0 ** (CLAMPED_EXP[typ] + 8 - e)  # a code of this is past the type's largest value
                    most = max(0.0, t - max(t / 16, 2.0 ** -9)) if e >= CLAMPED_EXP[typ] else 448.0
                    y = np.clip(np.where(fin, new, 0.0) * 2.0 ** -e, -most, most)
                    code = e4m3_code(e4m3(np.where(fin, y, np.nan)))
                    for i, c in zip(those, code):
                        cache[blk, h, (old + i - a) % block] = c
                    scale[blk, h] = e + 127
        out += [cache, scale]
    return out[0], out[2], out[1], out[3]


def cache8_values(cache, scale):
    """What a cache of codes holds, [n_blocks, n_kv_head, block_size, head_dim] in 64 bits."""
    e = np.clip(np.asarray(scale, np.int64), 1, 254) - 127
    return e4m3_value(cache) * np.exp2(e.astype(np.float64))[:, :, None, None]


def cache8_read(values, table, start, offsets, out):
    """`out` [n, n_kv_head, head_dim] with the requests' rows read; tokens that are not there are 0."""
    out = np.array(out, np.float64)
    n_blocks, _, block, _ = values.shape
    for r, first in enumerate(start):
        a, b = int(offsets[r]), int(offsets[r + 1])
        if first < 0 or a < 0 or b <= a or b > len(out):
            continue
        for i in range(a, b):
            t = int(first) + i - a
            blk = table[r, t // block] if t < table.shape[1] * block else -1
            out[i] = values[blk, :, t % block] if 0 <= blk < n_blocks else 0.0
    return out


def _probabilities(z):
    """softmax, or None where there is none (NaN, +inf, nothing but -inf)."""
    if np.isnan(z).any() or z.max() in (np.inf, -np.inf):
        return None
    e = np.exp(z - z.max())
    return e / e.sum()


def verify_drafts(target, draft, tokens, parents, offsets, lengths, accept, sample, scale, draft_scale, greedy, n_rows):
    """(new_len, rows, token), and the least distances of a child's acceptance and of a draw from their borders, as shares
    of the sum drawn from."""
    V = target.shape[1]
    new_len, rows, out, margin, drawn = [], [], [], 1.0, 1.0
    for r in range(len(lengths)):
        a, b = int(offsets[r]), int(offsets[r + 1])
        if a < 0 or b <= a or b > n_rows:
            new_len.append(int(lengths[r]))
            out.append(-1)
            continue
        path, node, token = [a], 0, -1
        while True:
            z = np.asarray(target[a + node], np.float64)
            kids = [i for i in range(node + 1, b - a) if parents[a + i] == node]
            p = _probabilities(z if greedy else z * np.float64(scale))
            if greedy:
                token = -1 if p is None else int(np.argmax(z))
                go = next((i for i in kids if token >= 0 and tokens[a + i] == token), None)
            else:
                q = None
                if draft is not None and kids:
                    q = _probabilities(np.asarray(draft[a + node], np.float64) * np.float64(draft_scale))
                if p is None or (draft is not None and kids and q is None):
                    token = -1
                    break
                left, go = p.copy(), None
                for i in kids:
                    x = int(tokens[a + i])
                    if not 0 <= x < V:
                        continue
                    qx, s = (1.0 if q is None else q[x]), left.sum()
                    d = left[x] - float(accept[a + i]) * s * qx
                    margin = min(margin, abs(d) / max(s * qx, 1e-300))
                    if d > 0:
                        go = i
                        break
                    if q is None:
                        left[x] = 0.0
                    else:
                        left = np.maximum(left - s * q, 0.0)
                if go is None:
                    if not left.sum() > 0:
                        left = p
                    ends = np.cumsum(left)
                    u = min(max(float(sample[r]), 0.0), 1 - 2.0 ** -24) * ends[-1]
                    drawn = min(drawn, np.abs(ends[:-1] - u).min(initial=ends[-1]) / ends[-1])
                    over = np.nonzero(ends > u)[0]
                    token = int(over[0]) if len(over) else int(np.nonzero(left)[0][-1])
            if go is None:
                break
            node = go
            path.append(a + node)
        new_len.append(int(lengths[r]) + len(path))
        rows += path
        out.append(token)
    return np.array(new_len), np.array(rows + [-1] * (n_rows - len(rows))), np.array(out), margin, drawn


def distill(z, logprob, ids, scale, rest):
    """(loss, lse, lse_rest, d): d [T, V] is the gradient of a row's loss with respect to its logits."""
    z, logprob = np.asarray(z, np.float64) * scale, np.asarray(logprob, np.float64)
    T, V = z.shape
    loss, lse, lrest, d = np.zeros(T), np.empty(T), np.full(T, -np.inf), np.zeros((T, V))
    log = lambda x: -np.inf if x == 0 else np.log(x)  # noqa: E731
    for t in range(T):
        top = z[t].max()
        with np.errstate(invalid="ignore"):
            e = np.zeros(V) if top == -np.inf else np.exp(z[t] - top)
        lse[t] = top + log(e.sum())
        known = [(int(i), float(x) * scale) for i, x in zip(ids[t], logprob[t]) if 0 <= i < V]
        outside = np.ones(V, bool)
        outside[[i for i, _ in known]] = False
        others = z[t][outside]
        peak = others.max(initial=-np.inf)
        with np.errstate(invalid="ignore"):
            lrest[t] = -np.inf if peak == -np.inf else peak + log(np.exp(others - peak).sum())
        if not known:
            continue
        x = np.array([x for _, x in known])
        if rest:
            q = np.exp(x)
        else:
            m = x.max()
            with np.errstate(invalid="ignore"):
                q = np.zeros(len(x)) if m == -np.inf else np.exp(x - m) / np.exp(x - m).sum()
        if np.isnan(top) or top == np.inf or np.isnan(q).any() or np.isinf(q).any():
            loss[t], d[t] = np.nan, np.nan
            continue
        p = e / e.sum() if top > -np.inf else np.zeros(V)
        for (i, _), qi in zip(known, q):
            if qi > 0:
                loss[t] += qi * (np.log(qi) - (z[t, i] - lse[t])) if z[t, i] > -np.inf else np.inf
        total = q.sum()
        left = max(0.0, 1 - total) if rest else 0.0
        total += left
        if left > 0:
            loss[t] += left * (np.log(left) - (lrest[t] - lse[t])) if lrest[t] > -np.inf else np.inf
        if top == -np.inf:
            continue
        d[t] = p * total
        if lrest[t] > -np.inf:
            d[t][outside] -= left * np.exp(z[t][outside] - lrest[t])
        for (i, _), qi in zip(known, q):
            d[t, i] -= qi
        d[t] *= scale
    return loss, lse, lrest, d
