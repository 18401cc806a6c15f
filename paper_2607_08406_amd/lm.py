"""ctypes binding of the language-model operators (include/mca_lm.h): same names,
argument marshalling only.

Tensors pass as they are: their strides go to the library, and what it does not
take is refused, not copied.  The work goes on the current stream of the tensors'
device, and workspaces come from PyTorch's allocator on that stream unless one is
given.  Nothing is synchronised.  No call records a graph for autograd: while
gradients are recorded, tensors that require one are refused; given tensors that a
call writes count as changed in place.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch
from torch import is_grad_enabled
from torch._C import _cuda_getCurrentRawStream as _raw_stream, _increment_version as increment_version

from . import mca
from .mca import (MCA_EDEVICE, MCA_EINVAL, MCAError, _check, load_library, mca_cache_append_args, mca_extend_args,
                  mca_token_logprobs_args, mca_token_logprobs_grad_args, mca_tree_attention_args)

MCA_TYPE_F32, MCA_TYPE_BF16, MCA_TYPE_F16 = 0, 1, 2
MCA_MAX_NODES, MCA_MAX_TOP, MCA_MAX_REQ = 128, 32, 65535
MCA_TABLES_OK, MCA_TABLES_EXHAUSTED, MCA_TABLES_LENGTH, MCA_TABLES_SLOTS = 0, 1, 2, 3

_TYPES = {torch.float32: MCA_TYPE_F32, torch.bfloat16: MCA_TYPE_BF16, torch.float16: MCA_TYPE_F16}


def _refuse(msg: str):
    raise MCAError(MCA_EINVAL, msg)


def _type(t: torch.Tensor) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        _refuse(f"{t.dtype} values: the operators take float32, bfloat16 and float16")
    return code


def _check_all(device, dtype, dim, **tensors):
    """Each tensor is on that device, of that type and number of dimensions, the last one contiguous."""
    for what, t in tensors.items():
        if t.device != device:
            _refuse(f"{what} is on {t.device}, not {device}")
        if t.dtype != dtype:
            _refuse(f"{what} holds {t.dtype}, not {dtype}")
        if t.dim() != dim:
            _refuse(f"{what} has {t.dim()} dimensions, not {dim}")
        if t.stride(-1) != 1 and t.size(-1) > 1:
            _refuse(f"{what} is not contiguous in its last dimension")


def _flat(device, dtype, what, t, size):
    if t.dtype is not dtype or t.dim() != 1 or t.device != device or not t.is_contiguous():
        _check_all(device, dtype, 1, **{what: t})
    if t.numel() != size:
        _refuse(f"{what} has {t.numel()} entries, not {size}")


def _rows(device, dtype, what, t, shape):
    """The strides of a tensor of that shape, whose last dimension is contiguous."""
    if t.dtype is not dtype or t.device != device or t.shape != shape:
        _check_all(device, dtype, len(shape), **{what: t})
        _refuse(f"{what} has shape {tuple(t.shape)}, not {tuple(shape)}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        _refuse(f"{what} is not contiguous in its last dimension")
    return s


def _whole(device, dtype, what, t, shape):
    if t.dtype is not dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        _check_all(device, dtype, len(shape), **{what: t})
        _refuse(f"{what} is not a contiguous tensor of shape {tuple(shape)}")


def _int32(**numbers):
    """The numbers go to the library in 32 bits, which ctypes would cut them to."""
    for what, x in numbers.items():
        if not 0 <= x < 1 << 31:
            _refuse(f"{what} is {x}: out of range [0, 2^31)")


def _no_graph(**tensors):
    what = next(what for what, t in tensors.items() if t is not None and t.requires_grad)
    _refuse(f"{what} requires grad, but the call records no graph: detach it, or call under torch.no_grad()")


def _gpu(t: torch.Tensor) -> torch.device:
    if not t.is_cuda:
        raise MCAError(MCA_EDEVICE, f"a tensor on {t.device}: the operators run only on the GPU")
    return t.device


def _run(device, call, *args):
    # the raw handle: a Stream object would cost as much host time as the launch
    index = device.index
    if torch.cuda.current_device() == index:
        rc = call(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            rc = call(*args, _raw_stream(index))
    if rc:
        _check(rc)


def _room(device, nbytes, workspace):
    if workspace is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    _flat(device, torch.uint8, "workspace", workspace, workspace.numel())
    return workspace


# ---------------------------------------------------------------------------
# the cache
# ---------------------------------------------------------------------------

def mca_block_tables(old_len, new_len, table, free_list, block_size: int, offsets, slots, status):
    """Update table [n_req, max_blocks] and free_list [n_blocks] for requests that go from old_len to
    new_len [n_req] tokens; offsets [n_req + 1], slots [max_tokens] (int64) and status [4] are written."""
    _int32(block_size=block_size)
    dev, i32 = _gpu(table), torch.int32
    _check_all(dev, i32, 2, table=table)
    n, width = table.shape
    _flat(dev, i32, "old_len", old_len, n)
    _flat(dev, i32, "new_len", new_len, n)
    _flat(dev, i32, "free_list", free_list, free_list.numel())
    _flat(dev, i32, "offsets", offsets, n + 1)
    _flat(dev, torch.int64, "slots", slots, slots.numel())
    _flat(dev, i32, "status", status, 4)
    _run(dev, load_library().mca_block_tables, old_len.data_ptr(), new_len.data_ptr(), n, block_size, table.data_ptr(),
         table.stride(0) if n > 1 else width, width, free_list.data_ptr(), free_list.numel(),
         offsets.data_ptr(), slots.data_ptr(), slots.numel(), status.data_ptr())
    increment_version((table, free_list, offsets, slots, status))


def mca_cache_append(k, v, k_cache, v_cache, slots, rows=None):
    """Row i (rows[i] with rows) of k and v [n_src, n_kv_head, head_dim] into slot slots[i] of the caches
    [n_blocks, n_kv_head, block_size, head_dim]."""
    if is_grad_enabled() and (k.requires_grad or v.requires_grad or k_cache.requires_grad or v_cache.requires_grad):
        _no_graph(k=k, v=v, k_cache=k_cache, v_cache=v_cache)
    dev, dt = _gpu(k_cache), k_cache.dtype
    a = mca_cache_append_args()
    a.dtype = _type(k_cache)
    if k_cache.dim() != 4:
        _refuse("k_cache has 4 dimensions")
    shape = k_cache.shape
    _whole(dev, dt, "k_cache", k_cache, shape)
    _whole(dev, dt, "v_cache", v_cache, shape)
    a.n_blocks, a.n_kv_head, a.block_size, a.head_dim = shape
    n, n_src = slots.numel(), k.shape[0] if k.dim() else 0
    src = (n_src, shape[1], shape[3])
    a.k_row, a.k_head, _ = _rows(dev, dt, "k", k, src)
    a.v_row, a.v_head, _ = _rows(dev, dt, "v", v, src)
    _flat(dev, torch.int64, "slots", slots, n)
    a.n, a.n_src = n, n_src
    if rows is not None:
        _flat(dev, torch.int32, "rows", rows, n)
        a.rows = rows.data_ptr()
    elif n != n_src:
        _refuse("without rows, slots has an entry for each row of k")
    a.k, a.v, a.k_cache, a.v_cache = k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr()
    a.slots = slots.data_ptr()
    _run(dev, load_library().mca_cache_append, ctypes.byref(a))
    increment_version((k_cache, v_cache))


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def _attention_args(q, k, v, k_cache, v_cache, table, lengths, offsets, parents, max_nodes, max_len, scale, out, lse):
    dev, dt, i32 = _gpu(q), q.dtype, torch.int32
    a = mca_tree_attention_args()
    a.dtype = _type(q)
    if q.dim() != 3 or k_cache.dim() != 4 or table.dim() != 2:
        _refuse("q has 3 dimensions, k_cache 4, table 2")
    shape, cache = q.shape, k_cache.shape
    n, n_head, dim = shape
    n_blocks, n_kv_head, block_size, _ = cache
    if cache[3] != dim:
        _refuse("q and the caches must agree in head_dim")
    a.q_row, a.q_head, _ = _rows(dev, dt, "q", q, shape)
    a.k_row, a.k_head, _ = _rows(dev, dt, "k", k, (n, n_kv_head, dim))
    a.v_row, a.v_head, _ = _rows(dev, dt, "v", v, (n, n_kv_head, dim))
    a.out_row, a.out_head, _ = _rows(dev, dt, "out", out, shape)
    _whole(dev, dt, "k_cache", k_cache, cache)
    _whole(dev, dt, "v_cache", v_cache, cache)
    n_req, max_blocks = table.shape
    stride = _rows(dev, i32, "table", table, table.shape)[0]
    _flat(dev, i32, "lengths", lengths, n_req)
    _flat(dev, i32, "offsets", offsets, n_req + 1)
    _flat(dev, i32, "parents", parents, n)
    if lse is not None:
        _whole(dev, torch.float32, "lse", lse, shape[:2])
        a.lse = lse.data_ptr()
    a.n_rows, a.n_head, a.head_dim = n, n_head, dim
    a.n_blocks, a.n_kv_head, a.block_size = n_blocks, n_kv_head, block_size
    a.n_req, a.max_blocks, a.max_nodes = n_req, max_blocks, max_nodes
    if max_len is None:
        max_len = max_blocks * block_size
    if (max_nodes | max_len) >> 31:
        _int32(max_nodes=max_nodes, max_len=max_len)
    a.max_len = max_len
    a.scale = dim ** -0.5 if scale is None else scale
    a.table_stride = stride if n_req > 1 else max_blocks
    a.q, a.k, a.v, a.out = q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr()
    a.k_cache, a.v_cache = k_cache.data_ptr(), v_cache.data_ptr()
    a.table, a.lengths = table.data_ptr(), lengths.data_ptr()
    a.offsets, a.parents = offsets.data_ptr(), parents.data_ptr()
    return dev, a


def mca_tree_attention_plan(q, k_cache, n_req: int, max_blocks: int, max_nodes: int, max_len: Optional[int] = None) -> int:
    """Workspace bytes of mca_tree_attention on tensors of these shapes."""
    a = mca_tree_attention_args()
    a.dtype = _type(q)
    a.n_rows, a.n_head, a.head_dim = q.shape
    a.n_blocks, a.n_kv_head, a.block_size, _ = k_cache.shape
    if max_len is None:
        max_len = max_blocks * a.block_size
    _int32(n_req=n_req, max_blocks=max_blocks, max_nodes=max_nodes, max_len=max_len)
    a.n_req, a.max_blocks, a.max_nodes, a.max_len = n_req, max_blocks, max_nodes, max_len
    return _plan(a, load_library().mca_tree_attention_plan)


def _plan(a, call) -> int:
    n = ctypes.c_size_t(0)
    _check(call(ctypes.byref(a), ctypes.byref(n)))
    return n.value


def mca_tree_attention(q, k, v, k_cache, v_cache, table, lengths, offsets, parents, max_nodes: int,
                       max_len: Optional[int] = None, scale: Optional[float] = None, out=None, lse=None,
                       workspace=None):
    """Attention of drafted nodes over the cache and their ancestors; returns (out, lse).

    q [n_rows, n_head, head_dim], k and v [n_rows, n_kv_head, head_dim]; request r has rows offsets[r] ..
    offsets[r + 1] - 1 and lengths[r] <= max_len cached tokens (default: what its table holds).  scale defaults to
    1 / sqrt(head_dim).  Rows of a given out and lse behind the last request stay as they were; those of new ones
    are zero.
    """
    if is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or k_cache.requires_grad or
                              v_cache.requires_grad or (out is not None and out.requires_grad) or
                              (lse is not None and lse.requires_grad)):
        _no_graph(q=q, k=k, v=v, k_cache=k_cache, v_cache=v_cache, out=out, lse=lse)
    if out is None:
        out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.zeros(q.shape[:2], dtype=torch.float32, device=q.device)
    dev, a = _attention_args(q, k, v, k_cache, v_cache, table, lengths, offsets, parents, max_nodes, max_len, scale,
                             out, lse)
    lib = load_library()
    nbytes = _plan(a, lib.mca_tree_attention_plan)
    if nbytes:
        room = _room(dev, nbytes, workspace)
        a.workspace, a.workspace_bytes = room.data_ptr(), room.numel()
    _run(dev, lib.mca_tree_attention, ctypes.byref(a))
    increment_version((out, lse))
    return out, lse


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------

class TokenLogprobs(NamedTuple):
    logprob: torch.Tensor      # [n_rows] of the given tokens
    entropy: torch.Tensor      # [n_rows]
    lse: torch.Tensor          # [n_rows]
    top_logprob: torch.Tensor  # [n_rows, n_top]
    top_id: torch.Tensor       # [n_rows, n_top] int32


def _logits(logits, tokens):
    """The logits' device and row stride."""
    dev = _gpu(logits)
    if logits.dim() != 2:
        _refuse("logits has 2 dimensions")
    row = _rows(dev, logits.dtype, "logits", logits, logits.shape)[0]
    if tokens.dtype is not torch.int32 and tokens.dtype is not torch.int64:
        _refuse("tokens must be int32 or int64")
    n, n_vocab = logits.shape
    _flat(dev, tokens.dtype, "tokens", tokens, n)
    return dev, row if n > 1 else n_vocab


def mca_token_logprobs_plan(logits, n_top: int = 0) -> int:
    """Workspace bytes of mca_token_logprobs on logits of this shape."""
    _int32(n_top=n_top)
    a = mca_token_logprobs_args()
    a.dtype, a.n_top = _type(logits), n_top
    a.n_rows, a.n_vocab = logits.shape
    return _plan(a, load_library().mca_token_logprobs_plan)


def mca_token_logprobs(logits, tokens, n_top: int = 0, workspace=None) -> TokenLogprobs:
    """Log probabilities of tokens [n_rows] under logits [n_rows, n_vocab], entropies and the n_top alternatives.

    Their gradient is mca_token_logprobs_grad.
    """
    if logits.requires_grad and is_grad_enabled():
        _no_graph(logits=logits)
    dev, row = _logits(logits, tokens)
    if n_top >> 31:
        _int32(n_top=n_top)
    a = mca_token_logprobs_args()
    a.dtype, a.n_top, a.token_bytes = _type(logits), n_top, tokens.element_size()
    n, a.n_vocab = logits.shape
    a.n_rows, a.logits_row = n, row
    lib = load_library()
    nbytes = _plan(a, lib.mca_token_logprobs_plan)
    logprob, entropy, lse = torch.empty((3, n), dtype=torch.float32, device=dev).unbind()
    top = torch.empty((n, n_top), dtype=torch.float32, device=dev)
    ids = torch.empty((n, n_top), dtype=torch.int32, device=dev)
    a.logits, a.tokens = logits.data_ptr(), tokens.data_ptr()
    a.logprob, a.entropy, a.lse = logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr()
    a.top_logprob, a.top_id = top.data_ptr(), ids.data_ptr()
    if nbytes:
        room = _room(dev, nbytes, workspace)
        a.workspace, a.workspace_bytes = room.data_ptr(), room.numel()
    _run(dev, lib.mca_token_logprobs, ctypes.byref(a))
    return TokenLogprobs(logprob, entropy, lse, top, ids)


def mca_token_logprobs_grad(logits, tokens, lse, entropy, grad_logprob=None, grad_entropy=None, out=None):
    """Gradient with respect to the logits of sum grad_logprob * logprob + grad_entropy * entropy; out may be logits.

    entropy may be None without grad_entropy.  A new gradient is contiguous; logits whose rows lie further apart than
    n_vocab are served several times faster with an out whose rows lie as far apart.
    """
    if is_grad_enabled() and (logits.requires_grad or lse.requires_grad or
                              (entropy is not None and entropy.requires_grad) or
                              (grad_logprob is not None and grad_logprob.requires_grad) or
                              (grad_entropy is not None and grad_entropy.requires_grad) or
                              (out is not None and out.requires_grad)):
        _no_graph(logits=logits, lse=lse, entropy=entropy, grad_logprob=grad_logprob, grad_entropy=grad_entropy, out=out)
    dev, row = _logits(logits, tokens)
    n, f32 = logits.shape[0], torch.float32
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    grad_row = _rows(dev, logits.dtype, "out", out, logits.shape)[0]
    a = mca_token_logprobs_grad_args()
    a.dtype, a.token_bytes = _type(logits), tokens.element_size()
    a.n_rows, a.n_vocab = logits.shape
    a.logits_row, a.grad_row = row, grad_row if n > 1 else out.shape[1]
    a.logits, a.tokens, a.grad = logits.data_ptr(), tokens.data_ptr(), out.data_ptr()
    _flat(dev, f32, "lse", lse, n)
    a.lse = lse.data_ptr()
    if grad_logprob is not None:
        _flat(dev, f32, "grad_logprob", grad_logprob, n)
        a.grad_logprob = grad_logprob.data_ptr()
    if grad_entropy is not None:
        _flat(dev, f32, "grad_entropy", grad_entropy, n)
        if entropy is None:
            _refuse("grad_entropy takes the entropy")
        _flat(dev, f32, "entropy", entropy, n)
        a.grad_entropy, a.entropy = grad_entropy.data_ptr(), entropy.data_ptr()
    _run(dev, load_library().mca_token_logprobs_grad, ctypes.byref(a))
    increment_version((out,))
    return out


# ---------------------------------------------------------------------------
# the committed net of a Transformer context
# ---------------------------------------------------------------------------

def _extend_args(dev, desc, tokens, parents, offsets, lengths, table, k_cache, v_cache, max_nodes, max_len, qkv, logits):
    i32, f32 = torch.int32, torch.float32
    H = desc.n_head
    a = mca_extend_args()
    n = tokens.numel()
    _flat(dev, i32, "tokens", tokens, n)
    _check_all(dev, i32, 2, table=table)
    R = table.shape[0]
    _flat(dev, i32, "parents", parents, n)
    _flat(dev, i32, "offsets", offsets, R + 1)
    _flat(dev, i32, "lengths", lengths, R)
    if k_cache.dim() != 5 or k_cache.shape[0] != desc.n_block or k_cache.shape[2] != H or k_cache.shape[4] != 32:
        _refuse(f"k_cache must be [{desc.n_block}, n_blocks, {H}, block_size, 32]")
    _whole(dev, f32, "k_cache", k_cache, k_cache.shape)
    _whole(dev, f32, "v_cache", v_cache, k_cache.shape)
    _whole(dev, f32, "qkv", qkv, (desc.n_block, n, 3, H, 32))
    logits_row = _rows(dev, f32, "logits", logits, (n, desc.vocab))[0]
    a.n_req, a.n_rows = R, n
    a.n_blocks, a.block_size, a.max_blocks = k_cache.shape[1], k_cache.shape[3], table.shape[1]
    if max_len is None:
        max_len = a.max_blocks * a.block_size
    _int32(max_nodes=max_nodes, max_len=max_len)
    a.max_nodes, a.max_len = max_nodes, max_len
    a.table_stride = table.stride(0) if R > 1 else a.max_blocks
    a.cache_layer = k_cache.stride(0) if desc.n_block > 1 else 0
    a.logits_row = logits_row if n > 1 else desc.vocab
    a.tokens, a.parents, a.offsets = tokens.data_ptr(), parents.data_ptr(), offsets.data_ptr()
    a.lengths, a.table = lengths.data_ptr(), table.data_ptr()
    a.k_cache, a.v_cache = k_cache.data_ptr(), v_cache.data_ptr()
    a.qkv, a.logits = qkv.data_ptr(), logits.data_ptr()
    return a


def mca_extend(ctx: "mca.TransformerContext", tokens, parents, offsets, lengths, table, k_cache, v_cache, max_nodes: int,
               max_len: Optional[int] = None, qkv=None, logits=None, workspace=None):
    """The context's committed net on drafted nodes; returns (logits [n_rows, vocab], qkv [n_block, n_rows, 3, n_head, 32]).

    The work goes on the context's stream.  Where that is not the current one, the caller orders the two (inputs
    before the call, results after it); the memory of the tensors stays theirs until both streams are done with it.
    """
    if is_grad_enabled() and any(t is not None and t.requires_grad for t in (k_cache, v_cache, qkv, logits)):
        _no_graph(k_cache=k_cache, v_cache=v_cache, qkv=qkv, logits=logits)
    # the context's own device: its name may lack the index
    dev, desc = ctx.workspace.device, ctx.desc
    given = dict(tokens=tokens, parents=parents, offsets=offsets, lengths=lengths, table=table, k_cache=k_cache,
                 v_cache=v_cache, qkv=qkv, logits=logits)
    for what, t in given.items():
        if t is not None and t.device != dev:
            _refuse(f"{what} is on {t.device}, not {dev}")
    n, caller = tokens.numel(), torch.cuda.current_stream(dev)
    with torch.cuda.device(dev), torch.cuda.stream(ctx.stream):
        if qkv is None:
            qkv = torch.empty((desc.n_block, n, 3, desc.n_head, 32), dtype=torch.float32, device=dev)
        if logits is None:
            logits = torch.zeros((n, desc.vocab), dtype=torch.float32, device=dev)
        a = _extend_args(dev, desc, tokens, parents, offsets, lengths, table, k_cache, v_cache, max_nodes, max_len, qkv,
                         logits)
        lib = load_library()
        nbytes = ctypes.c_size_t(0)
        _check(lib.mca_extend_plan(ctx.ctx, ctypes.byref(a), ctypes.byref(nbytes)), ctx.ctx)
        room = _room(dev, nbytes.value, workspace)
        a.workspace, a.workspace_bytes = room.data_ptr(), room.numel()
        _check(lib.mca_extend(ctx.ctx, ctypes.byref(a)), ctx.ctx)
    increment_version((qkv, logits))
    if caller != ctx.stream:
        for t in given.values():
            if t is not None:
                t.record_stream(ctx.stream)
        if workspace is not None:
            workspace.record_stream(ctx.stream)
        for what, t in (("qkv", qkv), ("logits", logits)):
            if given[what] is None:
                t.record_stream(caller)
    return logits, qkv
