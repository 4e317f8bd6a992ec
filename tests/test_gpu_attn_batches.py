"""Grouped attention over batches of more sequences than a wave holds boundaries of,
and of none: the order of tiles, the parts of keys and of rows, and what joins them."""
import itertools

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_queries_against_a_cache(gpu, dtype):
    """Nothing to do, and nothing refused: with the workspace that the call makes and with a given one."""
    cu = [torch.tensor(c, dtype=torch.int32, device="cuda") for c in ([0, 0], [0, 5])]
    q = torch.empty((0, 4, 64), dtype=dtype, device="cuda")
    k = torch.randn((5, 2, 64), device="cuda").to(dtype)
    ws = gpu.new_grouped_attn_workspace(1, 4, 2, 64, 0, 0, 5, backward=True)
    for workspace in (None, ws):
        out, lse, st = gpu.dora_grouped_attn(q, k, k, cu[0], 0, cu_k=cu[1], workspace=workspace)
        assert out.shape == (0, 4, 64) and lse.shape == (0, 4) and int(st) == 0
        dq, dk, dv, st = gpu.dora_grouped_attn_backward(q, q, k, k, out, lse, cu[0], 0, cu_k=cu[1], workspace=workspace)
        assert int(st) == 0 and dq.shape == (0, 4, 64) and bool((dk == 0).all()) and bool((dv == 0).all())
    # every sequence longer than it was said to be: reported and skipped
    q = torch.randn((6, 4, 64), device="cuda").to(dtype)
    out = torch.full_like(q, 5.0)
    cq, ck = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in ([0, 2, 4, 6], [0, 3, 4, 5]))
    _, _, st = gpu.dora_grouped_attn(q, k, k, cq, 0, cu_k=ck, out=out)
    assert int(st) == gpu.DORA_DEV_CU_SEQLENS and bool((out == 5.0).all())
