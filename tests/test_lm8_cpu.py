"""Refusals of the 8-bit cache, the verification of drafts and distillation: the C entry
points validate before anything is enqueued, so they run here with addresses that
nothing reads; and the binding's own."""
import ctypes

import pytest
import torch

from paper_2607_08406_amd import lm, mca

P = 1 << 20  # an aligned address, never read


@pytest.fixture(scope="module")
def lib():
    return mca.load_library()


def refused(lib, rc, code, word):
    msg = lib.mca_last_error(None).decode()
    assert rc == code and word in msg, (rc, msg)


def fill(struct, base, kw):
    a = struct()
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


CACHE = dict(dtype=1, n_req=3, n_kv_head=2, head_dim=32, block_size=16, n_blocks=8, max_blocks=4, n=5, table_stride=4, k=P, v=P,
             k_row=64, k_head=32, v_row=64, v_head=32, k_cache=P, v_cache=P, k_scale=P + 1, v_scale=P + 3, table=P, offsets=P)
COMMON = [
    (dict(dtype=3), mca.MCA_EINVAL, "dtype"),
    (dict(n_req=-1), mca.MCA_EINVAL, "n_req"),
    (dict(n_req=65536), mca.MCA_EINVAL, "n_req"),
    (dict(n=-1), mca.MCA_EINVAL, "negative"),
    (dict(head_dim=0), mca.MCA_EINVAL, "positive"),
    (dict(n_blocks=0), mca.MCA_EINVAL, "positive"),
    (dict(max_blocks=-1), mca.MCA_EINVAL, "positive"),
    (dict(head_dim=40), mca.MCA_EUNSUPPORTED, "multiple of 16"),
    (dict(head_dim=2 ** 24), mca.MCA_EUNSUPPORTED, "2^24"),
    (dict(block_size=2 ** 26, max_blocks=1), mca.MCA_EUNSUPPORTED, "2^30"),
    (dict(max_blocks=2 ** 27, table_stride=2 ** 27), mca.MCA_EUNSUPPORTED, "2^31"),
    (dict(n=2 ** 30, block_size=1), mca.MCA_EUNSUPPORTED, "too many"),
    (dict(k_row=-64), mca.MCA_EINVAL, "strides"),
    (dict(table_stride=3), mca.MCA_EINVAL, "table_stride"),
    (dict(v_head=36), mca.MCA_EINVAL, "16 bytes"),
    (dict(v_cache=None), mca.MCA_EINVAL, "NULL"),
    (dict(k_scale=None), mca.MCA_EINVAL, "NULL"),
    (dict(k=P + 8), mca.MCA_EINVAL, "aligned"),
    (dict(k_cache=P + 8), mca.MCA_EINVAL, "aligned"),
    (dict(offsets=P + 2), mca.MCA_EINVAL, "aligned"),
]


@pytest.mark.parametrize("kw,code,word", COMMON + [(dict(n_src=-1), mca.MCA_EINVAL, "n_src"), (dict(lengths=None), mca.MCA_EINVAL, "NULL"),
                                                   (dict(rows=P + 2), mca.MCA_EINVAL, "aligned")])
def test_append_refuses(lib, kw, code, word):
    refused(lib, lib.mca_cache8_append(ctypes.byref(fill(mca.mca_cache8_append_args, dict(CACHE, n_src=5, lengths=P), kw)), None), code, word)


@pytest.mark.parametrize("kw,code,word", COMMON + [(dict(start=None), mca.MCA_EINVAL, "NULL")])
def test_read_refuses(lib, kw, code, word):
    refused(lib, lib.mca_cache8_read(ctypes.byref(fill(mca.mca_cache8_read_args, dict(CACHE, start=P), kw)), None), code, word)


@pytest.mark.parametrize("kw", [dict(n=0), dict(n_req=0), dict(max_blocks=0, table=None)])
def test_nothing_to_append(lib, kw):
    assert lib.mca_cache8_append(ctypes.byref(fill(mca.mca_cache8_append_args, dict(CACHE, n_src=5, lengths=P), kw)), None) == mca.MCA_OK


ATTENTION = dict(dtype=1, n_req=3, n_head=8, n_kv_head=2, head_dim=64, block_size=16, n_blocks=40, max_blocks=1000,
                 max_nodes=4, max_len=16000, scale=0.125, n_rows=12, table_stride=1000, q=P, k=P, v=P, q_row=512, q_head=64,
                 k_row=128, k_head=64, v_row=128, v_head=64, out_row=512, out_head=64, k_cache=P, v_cache=P, table=P,
                 lengths=P, offsets=P, parents=P, out=P, lse=P, workspace=P, workspace_bytes=1 << 40)


@pytest.mark.parametrize("kw,scales,code,word", [
    (dict(dtype=-1), P, mca.MCA_EINVAL, "dtype"),
    (dict(head_dim=40), P, mca.MCA_EUNSUPPORTED, "multiple of 16"),
    (dict(head_dim=272), P, mca.MCA_EUNSUPPORTED, "256"),
    (dict(max_nodes=129), P, mca.MCA_EINVAL, "max_nodes"),
    (dict(scale=float("inf")), P, mca.MCA_EINVAL, "scale"),
    (dict(k_row=132), P, mca.MCA_EINVAL, "16 bytes"),
    (dict(v_cache=P + 8), P, mca.MCA_EINVAL, "aligned"),
    (dict(), None, mca.MCA_EINVAL, "NULL"),
    (dict(workspace=None), P, mca.MCA_EINVAL, "workspace"),
    (dict(workspace_bytes=16), P, mca.MCA_ENOSPACE, "mca_tree_attention8_plan"),
])
def test_attention_refuses(lib, kw, scales, code, word):
    a = mca.mca_tree_attention8_args(of=fill(mca.mca_tree_attention_args, ATTENTION, kw), k_scale=scales, v_scale=P)
    refused(lib, lib.mca_tree_attention8(ctypes.byref(a), None), code, word)


VERIFY = dict(dtype=0, n_req=3, max_nodes=5, greedy=0, n_rows=12, n_vocab=100, target_row=100, draft_row=104, scale=1.0, draft_scale=1.0,
              target=P, draft=P, tokens=P, parents=P, offsets=P, lengths=P, accept=P, sample=P, new_len=P, rows=P, token=P, workspace=P,
              workspace_bytes=1 << 40)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=3), mca.MCA_EINVAL, "dtype"),
    (dict(n_req=65536), mca.MCA_EINVAL, "n_req"),
    (dict(n_rows=-1), mca.MCA_EINVAL, "negative"),
    (dict(max_nodes=0), mca.MCA_EINVAL, "max_nodes"),
    (dict(max_nodes=129), mca.MCA_EINVAL, "max_nodes"),
    (dict(n_vocab=0), mca.MCA_EINVAL, "n_vocab"),
    (dict(n_rows=2 ** 24), mca.MCA_EUNSUPPORTED, "rows"),
    (dict(n_vocab=2 ** 30 + 1, target_row=2 ** 31, draft_row=2 ** 31), mca.MCA_EUNSUPPORTED, "2^30"),
    (dict(greedy=2), mca.MCA_EINVAL, "greedy"),
    (dict(scale=0.0), mca.MCA_EINVAL, "scale"),
    (dict(scale=float("nan")), mca.MCA_EINVAL, "scale"),
    (dict(draft_scale=-1.0), mca.MCA_EINVAL, "draft_scale"),
    (dict(scale=1e31), mca.MCA_EINVAL, "scale"),
    (dict(draft_scale=1e-31), mca.MCA_EINVAL, "draft_scale"),
    (dict(target_row=99), mca.MCA_EINVAL, "target_row"),
    (dict(draft_row=99), mca.MCA_EINVAL, "draft_row"),
    (dict(accept=None), mca.MCA_EINVAL, "NULL"),
    (dict(sample=None), mca.MCA_EINVAL, "NULL"),
    (dict(token=None), mca.MCA_EINVAL, "NULL"),
    (dict(draft=P + 2), mca.MCA_EINVAL, "aligned"),
    (dict(rows=P + 2), mca.MCA_EINVAL, "aligned"),
    (dict(workspace=P + 16), mca.MCA_EINVAL, "workspace"),
    (dict(workspace_bytes=16), mca.MCA_ENOSPACE, "mca_verify_drafts_plan"),
])
def test_verify_refuses(lib, kw, code, word):
    refused(lib, lib.mca_verify_drafts(ctypes.byref(fill(mca.mca_verify_drafts_args, VERIFY, kw)), None), code, word)


DISTILL = dict(dtype=1, n_top=5, rest=1, scale=1.0, n_rows=4, n_vocab=100000, logits_row=100000, logits=P, logprob=P, ids=P, lse=P,
               lse_rest=P)
BOTH = [
    (dict(dtype=3), mca.MCA_EINVAL, "dtype"),
    (dict(n_rows=-1), mca.MCA_EINVAL, "negative"),
    (dict(n_vocab=0), mca.MCA_EINVAL, "n_vocab"),
    (dict(n_top=0), mca.MCA_EINVAL, "n_top"),
    (dict(n_top=33), mca.MCA_EINVAL, "n_top"),
    (dict(rest=0, scale=0.0), mca.MCA_EINVAL, "scale"),
    (dict(rest=0, scale=1e-31), mca.MCA_EINVAL, "scale"),
    (dict(rest=0, scale=1e31), mca.MCA_EINVAL, "scale"),
    (dict(rest=0, scale=float("inf")), mca.MCA_EINVAL, "scale"),
    (dict(scale=0.5), mca.MCA_EINVAL, "rest"),
    (dict(rest=2), mca.MCA_EINVAL, "rest"),
    (dict(n_rows=2 ** 24), mca.MCA_EUNSUPPORTED, "rows"),
    (dict(n_vocab=2 ** 30 + 1), mca.MCA_EUNSUPPORTED, "2^30"),
    (dict(logits_row=99999), mca.MCA_EINVAL, "logits_row"),
    (dict(lse_rest=None), mca.MCA_EINVAL, "NULL"),
    (dict(ids=None), mca.MCA_EINVAL, "NULL"),
    (dict(logits=P + 1), mca.MCA_EINVAL, "aligned"),
    (dict(logprob=P + 2), mca.MCA_EINVAL, "aligned"),
]


@pytest.mark.parametrize("kw,code,word", BOTH + [
    (dict(loss=None), mca.MCA_EINVAL, "NULL"),
    (dict(workspace=None), mca.MCA_EINVAL, "workspace"),
    (dict(workspace_bytes=16), mca.MCA_ENOSPACE, "mca_distill_plan"),
])
def test_distill_refuses(lib, kw, code, word):
    base = dict(DISTILL, loss=P, workspace=P, workspace_bytes=1 << 30)
    refused(lib, lib.mca_distill(ctypes.byref(fill(mca.mca_distill_args, base, kw)), None), code, word)


@pytest.mark.parametrize("kw,code,word", BOTH + [
    (dict(grad=None), mca.MCA_EINVAL, "NULL"),
    (dict(grad_loss=None), mca.MCA_EINVAL, "NULL"),
    (dict(grad_row=99), mca.MCA_EINVAL, "grad_row"),
    (dict(grad=P, grad_row=100008), mca.MCA_EINVAL, "in place"),
])
def test_distill_grad_refuses(lib, kw, code, word):
    base = dict(DISTILL, grad=P, grad_loss=P, grad_row=100000)
    refused(lib, lib.mca_distill_grad(ctypes.byref(fill(mca.mca_distill_grad_args, base, kw)), None), code, word)


def test_the_binding_refuses():
    """Tensors that require a gradient, of another type or place; numbers beyond 32 bits."""
    z, t, f = torch.zeros(2, 5), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    g = torch.zeros(2, 5, requires_grad=True)
    logp, ids = torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    q, cache = torch.zeros(2, 1, 16), torch.zeros(2, 1, 4, 16).to(torch.float8_e4m3fn)
    sc, off = torch.zeros(2, 1, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    gq = q.clone().requires_grad_()
    tail = (cache, cache, sc, sc, t[:, None], t, off)
    calls = [lambda: lm.mca_distill(g, logp, ids), lambda: lm.mca_distill(z, logp.clone().requires_grad_(), ids),
             lambda: lm.mca_distill_grad(z, logp, ids, f, None, f, out=g), lambda: lm.mca_distill_grad(z, logp, ids, f.clone().requires_grad_(), None, f),
             lambda: lm.mca_verify_drafts(g, None, t, t, off, t, 1, f, f), lambda: lm.mca_verify_drafts(z, g, t, t, off, t, 1, f, f),
             lambda: lm.mca_cache8_append(gq, q, *tail), lambda: lm.mca_cache8_read(q, gq, *tail),
             lambda: lm.mca_tree_attention8(gq, q, q, *tail, t, 1), lambda: lm.mca_tree_attention8(q, q, q, *tail, t, 1, out=gq)]
    for call in calls:
        with pytest.raises(mca.MCAError, match="requires grad"):
            call()
        with torch.no_grad(), pytest.raises(mca.MCAError, match="cpu"):
            call()
    for kw in (dict(max_nodes=2 ** 32 + 1), dict(n_req=2 ** 32 + 1), dict(max_nodes=-1)):
        with pytest.raises(mca.MCAError):
            lm.mca_verify_drafts_plan(z, None, **{**dict(n_req=2, max_nodes=3), **kw})
    with pytest.raises(mca.MCAError):
        lm.mca_distill_plan(z, 2 ** 32 + 1)
    with pytest.raises(mca.MCAError):
        lm.mca_tree_attention8_plan(q, cache, 2, 4, 1, max_len=2 ** 32)
    assert lm.mca_tree_attention8_plan(q, cache, 2, 4, 1) == 0 and lm.mca_distill_plan(z, 3) == 0
