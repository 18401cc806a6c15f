"""What the binding of the language-model operators refuses before it calls the library."""
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
