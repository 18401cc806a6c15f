"""What the binding of the language-model operators refuses before it calls the library, and calls of nothing."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2607_08406_amd import lm, mca


def extend_args(n=3, R=2, heads=2, blocks=4, block=8):
    i32 = torch.int32
    ctx = SimpleNamespace(ctx=None, device=torch.device("cuda"), stream=None,
                          workspace=SimpleNamespace(device=torch.device("cuda", 0)),
                          desc=SimpleNamespace(n_head=heads, n_block=1, vocab=65))
    args = [torch.zeros(n, dtype=i32), torch.full((n,), -1, dtype=i32), torch.zeros(R + 1, dtype=i32),
            torch.zeros(R, dtype=i32), torch.zeros(R, 2, dtype=i32), torch.zeros(1, blocks, heads, block, 32),
            torch.zeros(1, blocks, heads, block, 32), 1]
    return ctx, args, dict(qkv=torch.zeros(1, n, 3, heads, 32), logits=torch.zeros(n, 65))


def test_extend_refuses_tensors_of_another_device_than_the_contexts():
    """Also if they are all on the same one."""
    ctx, args, outs = extend_args()
    with pytest.raises(mca.MCAError, match="is on cpu, not cuda:0"):
        lm.mca_extend(ctx, *args, **outs)


def test_tensors_that_require_a_gradient_are_refused_while_gradients_are_recorded():
    """Under no_grad they are taken (and refused here for another reason: there is no GPU)."""
    z, t = torch.zeros(2, 5), torch.zeros(2, dtype=torch.int32)
    g = torch.zeros(2, 5, requires_grad=True)
    row, q, cache = torch.zeros(2), torch.zeros(2, 1, 8), torch.zeros(2, 1, 4, 8)
    gq, gcache = q.clone().requires_grad_(), cache.clone().requires_grad_()
    tail = (t[:, None], t, torch.zeros(3, dtype=torch.int32), t, 1)
    ctx, args, outs = extend_args()
    calls = [lambda: lm.mca_token_logprobs(g, t), lambda: lm.mca_token_logprobs(g * 2, t),
             lambda: lm.mca_token_logprobs_grad(g, t, row, row, row), lambda: lm.mca_token_logprobs_grad(z, t, row, row, row, out=g),
             lambda: lm.mca_cache_append(gq, q, cache, cache, t.long()), lambda: lm.mca_cache_append(q, q, cache, gcache, t.long()),
             lambda: lm.mca_tree_attention(q, gq, q, cache, cache, *tail), lambda: lm.mca_tree_attention(q, q, q, gcache, cache, *tail),
             lambda: lm.mca_tree_attention(q, q, q, cache, cache, *tail, out=gq),
             lambda: lm.mca_extend(ctx, *args, **dict(outs, logits=outs["logits"].clone().requires_grad_()))]
    for call in calls:
        with pytest.raises(mca.MCAError, match="requires grad"):
            call()
        with torch.no_grad(), pytest.raises(mca.MCAError, match="cpu"):
            call()


@pytest.mark.parametrize("kw", [dict(max_len=2 ** 32), dict(max_len=2 ** 32 + 5), dict(max_nodes=2 ** 32 + 1), dict(n_req=2 ** 32 + 1),
                                dict(max_blocks=2 ** 32 + 1), dict(max_blocks=2 ** 28), dict(max_len=-1), dict(max_nodes=-2 ** 32 + 1)])
def test_numbers_beyond_32_bits_are_refused(kw):
    """Not cut to what is left of them."""
    q, cache = torch.empty(4, 2, 64), torch.empty(9, 1, 16, 64)
    a = dict(n_req=2, max_blocks=4, max_nodes=2)
    assert lm.mca_tree_attention_plan(q, cache, **a) == 0
    with pytest.raises(mca.MCAError):
        lm.mca_tree_attention_plan(q, cache, **{**a, **kw})


def test_numbers_of_alternatives_beyond_32_bits_are_refused():
    for n in (2 ** 32 + 3, -2 ** 32 + 3):
        with pytest.raises(mca.MCAError):
            lm.mca_token_logprobs_plan(torch.empty(2, 500), n)


def test_rows_of_an_empty_source_are_skipped():
    """There is no source row to take: nothing is enqueued, and the arrays may be NULL, as an empty tensor's is."""
    a = mca.mca_cache_append_args(dtype=0, n_kv_head=2, head_dim=32, block_size=16, n_blocks=8, n=5, n_src=0, k_row=64,
                                  k_head=32, v_row=64, v_head=32, k_cache=1 << 20, v_cache=1 << 20, slots=1 << 20, rows=1 << 20)
    assert mca.load_library().mca_cache_append(ctypes.byref(a), None) == mca.MCA_OK
    a.n_src = 1
    assert mca.load_library().mca_cache_append(ctypes.byref(a), None) == mca.MCA_EINVAL
