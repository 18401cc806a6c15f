"""Refusals of the language-model operators: the C entry points validate before
anything is enqueued, so they run here with addresses that nothing reads."""
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


def tables_args(**kw):
    a = dict(old_len=P, new_len=P, n_req=4, block_size=16, table=P, table_stride=8, max_blocks=8, free_list=P,
             n_blocks=64, offsets=P, slots=P, max_tokens=10, status=P, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("kw,code,word", [
    (dict(n_req=0), mca.MCA_EINVAL, "n_req"),
    (dict(n_req=65536), mca.MCA_EINVAL, "n_req"),
    (dict(block_size=0), mca.MCA_EINVAL, "positive"),
    (dict(max_blocks=0), mca.MCA_EINVAL, "positive"),
    (dict(n_blocks=0), mca.MCA_EINVAL, "positive"),
    (dict(block_size=2 ** 30), mca.MCA_EUNSUPPORTED, "2^31"),
    (dict(n_blocks=2 ** 31 - 1), mca.MCA_EUNSUPPORTED, "2^31"),
    (dict(table_stride=7), mca.MCA_EINVAL, "table_stride"),
    (dict(max_tokens=-1), mca.MCA_EINVAL, "max_tokens"),
    (dict(max_tokens=2 ** 31), mca.MCA_EINVAL, "max_tokens"),
    (dict(status=None), mca.MCA_EINVAL, "NULL"),
    (dict(slots=None), mca.MCA_EINVAL, "NULL"),
    (dict(slots=P + 4), mca.MCA_EINVAL, "aligned"),
    (dict(table=P + 2), mca.MCA_EINVAL, "aligned"),
])
def test_block_tables_refuses(lib, kw, code, word):
    refused(lib, lib.mca_block_tables(*tables_args(**kw)), code, word)


def fill(struct, base, kw):
    a = struct()
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


APPEND = dict(dtype=1, n_kv_head=2, head_dim=32, block_size=16, n_blocks=8, n=5, n_src=5, k=P, v=P, k_row=64, k_head=32,
              v_row=64, v_head=32, k_cache=P, v_cache=P, slots=P)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=3), mca.MCA_EINVAL, "dtype"),
    (dict(n=-1), mca.MCA_EINVAL, "negative"),
    (dict(head_dim=0), mca.MCA_EINVAL, "positive"),
    (dict(n_blocks=0), mca.MCA_EINVAL, "positive"),
    (dict(head_dim=2 ** 24), mca.MCA_EUNSUPPORTED, "2^24"),
    (dict(n=2 ** 24), mca.MCA_EUNSUPPORTED, "rows"),
    (dict(k_row=-1), mca.MCA_EINVAL, "strides"),
    (dict(v_cache=None), mca.MCA_EINVAL, "NULL"),
    (dict(k=P + 1), mca.MCA_EINVAL, "aligned"),
    (dict(slots=P + 4), mca.MCA_EINVAL, "aligned"),
])
def test_cache_append_refuses(lib, kw, code, word):
    refused(lib, lib.mca_cache_append(ctypes.byref(fill(mca.mca_cache_append_args, APPEND, kw)), None), code, word)


ATTENTION = dict(dtype=1, n_req=3, n_head=8, n_kv_head=2, head_dim=64, block_size=16, n_blocks=40, max_blocks=1000,
                 max_nodes=4, max_len=16000, scale=0.125, n_rows=12, table_stride=1000, q=P, k=P, v=P, q_row=512, q_head=64,
                 k_row=128, k_head=64, v_row=128, v_head=64, out_row=512, out_head=64, k_cache=P, v_cache=P, table=P,
                 lengths=P, offsets=P, parents=P, out=P, lse=P, workspace=P, workspace_bytes=1 << 40)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=-1), mca.MCA_EINVAL, "dtype"),
    (dict(n_req=-1), mca.MCA_EINVAL, "n_req"),
    (dict(n_req=65536), mca.MCA_EINVAL, "n_req"),
    (dict(n_head=7), mca.MCA_EINVAL, "multiple"),
    (dict(n_kv_head=0), mca.MCA_EINVAL, "multiple"),
    (dict(head_dim=264), mca.MCA_EUNSUPPORTED, "256"),
    (dict(head_dim=36), mca.MCA_EUNSUPPORTED, "16 bytes"),
    (dict(dtype=0, head_dim=30), mca.MCA_EUNSUPPORTED, "16 bytes"),
    (dict(max_nodes=0), mca.MCA_EINVAL, "max_nodes"),
    (dict(max_nodes=129), mca.MCA_EINVAL, "max_nodes"),
    (dict(max_len=-1), mca.MCA_EINVAL, "max_len"),
    (dict(max_len=2 ** 30 + 1), mca.MCA_EUNSUPPORTED, "2^30"),
    (dict(max_blocks=2 ** 27, table_stride=2 ** 27), mca.MCA_EUNSUPPORTED, "2^31"),
    (dict(block_size=0), mca.MCA_EINVAL, "positive"),
    (dict(n_blocks=2 ** 27, block_size=16), mca.MCA_EUNSUPPORTED, "2^31"),
    (dict(n_req=65535, max_nodes=128, n_head=64, n_kv_head=2), mca.MCA_EUNSUPPORTED, "too many"),
    (dict(scale=float("nan")), mca.MCA_EINVAL, "scale"),
    (dict(table_stride=999), mca.MCA_EINVAL, "table_stride"),
    (dict(q_row=-512), mca.MCA_EINVAL, "strides"),
    (dict(k_row=132), mca.MCA_EINVAL, "16 bytes"),
    (dict(v=P + 8), mca.MCA_EINVAL, "aligned"),
    (dict(parents=None), mca.MCA_EINVAL, "NULL"),
    (dict(lengths=P + 2), mca.MCA_EINVAL, "aligned"),
    (dict(workspace=None), mca.MCA_EINVAL, "workspace"),
    (dict(workspace=P + 16), mca.MCA_EINVAL, "workspace"),
    (dict(workspace_bytes=16), mca.MCA_ENOSPACE, "workspace"),
])
def test_tree_attention_refuses(lib, kw, code, word):
    a = fill(mca.mca_tree_attention_args, ATTENTION, kw)
    refused(lib, lib.mca_tree_attention(ctypes.byref(a), None), code, word)


LOGPROBS = dict(dtype=1, n_top=5, token_bytes=8, n_rows=2, n_vocab=500000, logits_row=500000, logits=P, tokens=P, logprob=P,
                entropy=P, lse=P, top_logprob=P, top_id=P, workspace=P, workspace_bytes=1 << 30)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=9), mca.MCA_EINVAL, "dtype"),
    (dict(n_rows=-1), mca.MCA_EINVAL, "n_rows"),
    (dict(n_vocab=0), mca.MCA_EINVAL, "n_vocab"),
    (dict(n_top=33), mca.MCA_EINVAL, "n_top"),
    (dict(n_top=-1), mca.MCA_EINVAL, "n_top"),
    (dict(n_top=9, n_vocab=8), mca.MCA_EINVAL, "n_top"),
    (dict(n_rows=2 ** 24), mca.MCA_EUNSUPPORTED, "rows"),
    (dict(n_vocab=2 ** 30 + 1, logits_row=2 ** 31), mca.MCA_EUNSUPPORTED, "n_vocab"),
    (dict(token_bytes=2), mca.MCA_EINVAL, "token_bytes"),
    (dict(logits_row=499999), mca.MCA_EINVAL, "logits_row"),
    (dict(top_id=None), mca.MCA_EINVAL, "NULL"),
    (dict(logits=P + 1), mca.MCA_EINVAL, "aligned"),
    (dict(tokens=P + 4), mca.MCA_EINVAL, "aligned"),
    (dict(workspace_bytes=8), mca.MCA_ENOSPACE, "workspace"),
    (dict(workspace=None), mca.MCA_EINVAL, "workspace"),
])
def test_token_logprobs_refuses(lib, kw, code, word):
    a = fill(mca.mca_token_logprobs_args, LOGPROBS, kw)
    refused(lib, lib.mca_token_logprobs(ctypes.byref(a), None), code, word)


GRAD = dict(dtype=1, token_bytes=4, n_rows=2, n_vocab=100, logits_row=100, grad_row=104, logits=P, tokens=P, lse=P,
            entropy=P, grad_logprob=P, grad_entropy=P, grad=2 * P)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=9), mca.MCA_EINVAL, "dtype"),
    (dict(n_rows=-1), mca.MCA_EINVAL, "n_rows"),
    (dict(n_rows=2 ** 24), mca.MCA_EUNSUPPORTED, "rows"),
    (dict(grad_row=99), mca.MCA_EINVAL, "grad_row"),
    (dict(token_bytes=0), mca.MCA_EINVAL, "token_bytes"),
    (dict(grad=None), mca.MCA_EINVAL, "NULL"),
    (dict(entropy=None), mca.MCA_EINVAL, "NULL"),
    (dict(grad=P), mca.MCA_EINVAL, "stride"),
    (dict(lse=P + 1), mca.MCA_EINVAL, "aligned"),
])
def test_token_logprobs_grad_refuses(lib, kw, code, word):
    a = fill(mca.mca_token_logprobs_grad_args, GRAD, kw)
    refused(lib, lib.mca_token_logprobs_grad(ctypes.byref(a), None), code, word)


def test_calls_without_rows_enqueue_nothing(lib):
    for call, a in [(lib.mca_cache_append, fill(mca.mca_cache_append_args, APPEND, dict(n=0, k=None))),
                    (lib.mca_tree_attention, fill(mca.mca_tree_attention_args, ATTENTION, dict(n_rows=0, q=None))),
                    (lib.mca_tree_attention, fill(mca.mca_tree_attention_args, ATTENTION, dict(n_req=0))),
                    (lib.mca_token_logprobs, fill(mca.mca_token_logprobs_args, LOGPROBS, dict(n_rows=0, logits=None))),
                    (lib.mca_token_logprobs_grad, fill(mca.mca_token_logprobs_grad_args, GRAD, dict(n_rows=0)))]:
        assert call(ctypes.byref(a), None) == mca.MCA_OK


def test_plans_without_requests_or_rows(lib):
    n = ctypes.c_size_t(7)
    for kw in (dict(n_req=0), dict(n_req=0, max_nodes=128), dict(n_rows=0), dict(max_len=0, max_blocks=0)):
        a = fill(mca.mca_tree_attention_args, ATTENTION, kw)
        assert lib.mca_tree_attention_plan(ctypes.byref(a), ctypes.byref(n)) == mca.MCA_OK
    a = fill(mca.mca_token_logprobs_args, LOGPROBS, dict(n_rows=0))
    assert lib.mca_token_logprobs_plan(ctypes.byref(a), ctypes.byref(n)) == mca.MCA_OK and n.value == 0


def test_null_arguments(lib):
    n = ctypes.c_size_t()
    for call, args in [(lib.mca_cache_append, (None, None)), (lib.mca_tree_attention, (None, None)),
                       (lib.mca_token_logprobs, (None, None)), (lib.mca_token_logprobs_grad, (None, None)),
                       (lib.mca_tree_attention_plan, (None, ctypes.byref(n))),
                       (lib.mca_token_logprobs_plan, (None, ctypes.byref(n))),
                       (lib.mca_extend, (None, None)), (lib.mca_extend_plan, (None, None, ctypes.byref(n)))]:
        assert call(*args) == mca.MCA_EINVAL


def test_plans(lib):
    """Short contexts and many rows need no workspace; a long one on few rows is split."""
    n = ctypes.c_size_t()
    a = fill(mca.mca_tree_attention_args, ATTENTION, dict(max_len=100))
    assert lib.mca_tree_attention_plan(ctypes.byref(a), ctypes.byref(n)) == 0 and n.value == 0
    a = fill(mca.mca_tree_attention_args, ATTENTION, dict())
    assert lib.mca_tree_attention_plan(ctypes.byref(a), ctypes.byref(n)) == 0
    assert n.value % (12 * 8 * 65 * 4) == 0 and n.value > 12 * 8 * 65 * 4
    b = fill(mca.mca_token_logprobs_args, LOGPROBS, dict(n_rows=5000))
    assert lib.mca_token_logprobs_plan(ctypes.byref(b), ctypes.byref(n)) == 0 and n.value == 0
    b = fill(mca.mca_token_logprobs_args, LOGPROBS, dict())
    assert lib.mca_token_logprobs_plan(ctypes.byref(b), ctypes.byref(n)) == 0 and n.value > 0
    assert lm.mca_token_logprobs_plan(torch.empty(2, 500000, dtype=torch.bfloat16), 5) == n.value


def test_tensors_without_a_gpu_are_refused():
    z = torch.zeros(2, 5)
    with pytest.raises(mca.MCAError):
        lm.mca_token_logprobs(z, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(mca.MCAError):
        lm.mca_cache_append(z[:, None], z[:, None], torch.zeros(2, 1, 4, 5), torch.zeros(2, 1, 4, 5),
                            torch.zeros(2, dtype=torch.int64))
    with pytest.raises(mca.MCAError):
        lm.mca_token_logprobs_plan(z.double(), 1)
