"""The operators of drafts and 8-bit caches on two streams at once, in the forms that keep something in a workspace or work
on whole requests: calls that overlap give what they give alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.fixture(scope="module")
def lm():
    from paper_2607_08406_amd import lm as m
    assert torch.cuda.is_available()
    return m


def both(make):
    """make(generator) gives a call without arguments; two of them, of other inputs each, on two streams."""
    calls = [make(torch.Generator("cuda").manual_seed(s)) for s in (1, 2)]
    alone = [[t.clone() for t in c()] for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in calls], [[], []]
    for _ in range(6):
        for i, c in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                got[i].append([t.clone() for t in c()])
    torch.cuda.synchronize()
    for want, runs in zip(alone, got):
        for run in runs:
            for a, b in zip(want, run):
                assert torch.equal(a, b)


def cache(g, blocks, heads, block, dim):
    codes = [torch.randint(0, 120, (blocks, heads, block, dim), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scales = [torch.randint(118, 122, (blocks, heads), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8) for _ in range(2)]
    return [c.view(torch.float8_e4m3fn) for c in codes] + scales


@pytest.mark.parametrize("dim,nodes,group,typ", [(128, 1, 4, torch.bfloat16), (256, 2, 2, torch.float32),  # few rows, shared
                                                 (128, 48, 4, torch.float16), (64, 40, 3, torch.float32),  # many rows, shared
                                                 (64, 2, 2, torch.bfloat16)])  # chunks
def test_attention(lm, dim, nodes, group, typ):
    R, H, block, length = 8, 4, 64, 16384
    width = length // block

    def make(g):
        caches = cache(g, R * width, H, block, dim)
        table = torch.randperm(R * width, generator=g, device="cuda").view(R, width).to(I32)
        lens = torch.randint(0, length + 1, (R,), generator=g, device="cuda").to(I32)
        offsets = torch.arange(R + 1, device="cuda", dtype=I32) * nodes
        parents = torch.arange(-1, nodes - 1, device="cuda").repeat(R).to(I32)
        q = torch.randn(R * nodes, H * group, dim, generator=g, device="cuda").to(typ)
        k, v = (torch.randn(R * nodes, H, dim, generator=g, device="cuda").to(typ) for _ in range(2))
        assert lm.mca_tree_attention8_plan(q, caches[0], R, width, nodes) > 0
        return lambda: lm.mca_tree_attention8(q, k, v, *caches, table, lens, offsets, parents, nodes)
    both(make)


@pytest.mark.parametrize("mode", ["draft", "given", "greedy"])
@pytest.mark.parametrize("vocab", [500, 30000])
def test_verification(lm, mode, vocab):
    R, n = 40, 7

    def make(g):
        draft = torch.randn(R * n, vocab, generator=g, device="cuda") * 2
        target = (draft + torch.randn(R * n, vocab, generator=g, device="cuda")).bfloat16()
        tokens = torch.randint(0, vocab, (R * n,), generator=g, device="cuda").to(I32)
        parents = ((torch.arange(n, device="cuda") + 1) // 2 - 1).repeat(R).to(I32)
        lens, offsets = torch.zeros(R, device="cuda", dtype=I32), torch.arange(R + 1, device="cuda", dtype=I32) * n
        accept, sample = torch.rand(R * n, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda")
        return lambda: lm.mca_verify_drafts(target, draft.bfloat16() if mode == "draft" else None, tokens, parents, offsets, lens, n,
                                            accept, sample, greedy=mode == "greedy")
    both(make)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(5, 100003), (2000, 90)])
def test_distillation(lm, rows, vocab, rest):
    def make(g):
        z = torch.randn(rows, vocab, generator=g, device="cuda")
        ids = torch.randint(0, vocab, (rows, 6), generator=g, device="cuda").to(I32)
        logp = torch.log_softmax(torch.randn(rows, 6, generator=g, device="cuda"), 1) - 0.1
        weight = torch.rand(rows, generator=g, device="cuda")
        assert (lm.mca_distill_plan(z, 6, rest) > 0) == (vocab > 65536)

        def call():
            r = lm.mca_distill(z, logp, ids, rest)
            return [r.loss, r.lse, lm.mca_distill_grad(z, logp, ids, r.lse, r.lse_rest, weight, rest)]
        return call
    both(make)


@pytest.mark.parametrize("block", [16, 128])
def test_cache(lm, block):
    R, H, dim, width = 30, 2, 128, 6

    def make(g):
        start = cache(g, R * width, H, block, dim)
        table = torch.randperm(R * width, generator=g, device="cuda").view(R, width).to(I32)
        lens = torch.randint(0, 2 * block, (R,), generator=g, device="cuda").to(I32)
        offsets = torch.arange(R + 1, device="cuda", dtype=I32) * (3 * block)
        k, v = (torch.randn(R * 3 * block, H, dim, generator=g, device="cuda").bfloat16() for _ in range(2))

        def call():
            caches = [c.clone() for c in start]
            lm.mca_cache8_append(k, v, *caches, table, lens, offsets)
            back = lm.mca_cache8_read(torch.zeros_like(k), torch.zeros_like(v), *caches, table, lens, offsets)
            return [c.view(torch.uint8) for c in caches] + list(back)
        return call
    both(make)
