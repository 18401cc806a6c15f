"""mca_extend from another stream than the context's: tensors that the caller lets go of
right after the call are not given out again before the work on them is done."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from workloads import CONFIGS, transformer_workload

pytestmark = pytest.mark.gpu


def make(stream):
    from paper_2607_08406_amd import mca
    cfg = replace(CONFIGS["transformer"], ctx=32, d_model=64, n_head=2, n_seq=2, d_mlp=96)
    w = transformer_workload(cfg)
    desc = mca.transformer_desc(cfg.vocab, cfg.ctx, cfg.d_model, cfg.n_layer, cfg.n_head, cfg.d_mlp, delta=cfg.delta,
                                ln_eps=cfg.ln_eps, seed=cfg.seed_stream, stream_tag=cfg.stream_tag)
    return mca.TransformerContext(desc, w["params"], w["tokens"], w["targets"], k_max=2, stream=stream), cfg


def inputs(cfg, seed):
    """8 requests of 5 nodes behind 9 cached tokens, 4 tokens a block; freed and made anew they lie in the same memory."""
    rng = np.random.default_rng(seed)
    R, n, blocks = 8, 5, 24
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(seed)
    caches = [torch.randn(cfg.n_layer, blocks, 2, 4, 32, device="cuda", generator=g) for _ in range(2)]
    return [put(rng.integers(0, cfg.vocab, R * n)), put(np.tile(rng.integers(-1, 1, n).clip(max=np.arange(n) - 1), R)),
            put(np.arange(R + 1) * n), put(np.full(R, 9)), put(rng.permutation(blocks).reshape(R, 3)), *caches]


def busy(a):
    for _ in range(12):
        a = (a @ a) * 1e-4
    return a


@pytest.mark.parametrize("given", [False, True])
def test_tensors_let_go_of_after_the_call(given):
    s, mine = torch.cuda.Stream(), torch.cuda.current_stream()
    ctx, cfg = make(s)
    n = 40

    def extend(seed):
        kw = {}
        if given:
            kw = dict(qkv=torch.zeros(cfg.n_layer, n, 3, 2, 32, device="cuda"), logits=torch.zeros(n, cfg.vocab, device="cuda"),
                      workspace=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
        args = inputs(cfg, seed)
        s.wait_stream(mine)
        return ctx.extend(*args, 5, max_len=12, **kw)

    want = []
    for seed in (1, 2):
        got = extend(seed)
        torch.cuda.synchronize()
        want.append([x.clone() for x in got])
    a = torch.randn(6144, 6144, device="cuda") * 0.01
    torch.cuda.synchronize()
    # the context's stream is behind: the inputs are freed and their memory asked for again meanwhile
    with torch.cuda.stream(s):
        busy(a)
    got = extend(1)
    junk = [torch.full_like(x, 3) for x in inputs(cfg, 3) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))
    # the caller's stream is behind: the results are freed and the next call asks for memory meanwhile
    got = extend(1)
    mine.wait_stream(s)
    busy(a)
    kept = [x.clone() for x in got]
    del got, junk
    # (inputs of the second call are on the context's stream, which does not wait)
    with torch.cuda.stream(s):
        args = inputs(cfg, 2)
    again = ctx.extend(*args, 5, max_len=12)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(kept, want[0]))
    assert all(torch.equal(x, y) for x, y in zip(again, want[1]))
    ctx.close()
