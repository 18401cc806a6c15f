"""Inputs of the tests of the 8-bit cache, shared."""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn


def put(a, dtype=np.int32):
    return torch.from_numpy(np.array(a, dtype)).cuda()


def host(t):
    if t is None:
        return None
    t = t.detach().cpu()
    if t.dtype == E4M3:
        return t.view(torch.uint8).numpy().copy()
    return (t.float() if t.is_floating_point() else t).numpy().copy()


def codes(a):
    """A cache of codes (uint8) on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(a, np.uint8)).cuda().view(E4M3)


def pages(rng, tokens, block, width=None, spare=2):
    """(table [R, width], blocks of the pool) with a block for each of the requests' pages, others -7."""
    held = [-(-int(n) // block) for n in tokens]
    width = max(1, max(held, default=1)) if width is None else width
    pool = rng.permutation(sum(held) + spare)
    table, at = np.full((len(tokens), width), -7, np.int32), 0
    for r, n in enumerate(held):
        table[r, :n] = pool[at:at + n]
        at += n
    return table, len(pool)


def cache(rng, blocks, kv, block, dim, spread=0):
    """Random codes (no NaN) and scales of 2^-6 give or take `spread`, for K and V."""
    out = []
    for _ in range(2):
        c = rng.integers(0, 256, (blocks, kv, block, dim)).astype(np.uint8)
        c[(c & 127) == 127] = 0x35
        out.append((c, (121 + rng.integers(-spread, spread + 1, (blocks, kv))).astype(np.uint8)))
    return out
