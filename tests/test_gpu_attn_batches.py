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


def cu_of(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def make(nq, nk, H, Hk, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    cu_q, cu_k = cu_of(nq), cu_of(nk)
    t = {n: torch.randn((c[-1], h, D), generator=g).to(dtype) for n, c, h in (("q", cu_q, H), ("k", cu_k, Hk), ("v", cu_k, Hk),
                                                                               ("dout", cu_q, H))}
    return t, cu_q, cu_k


def forward(gpu, t, cu_q, cu_k, max_q, causal, what, **kw):
    d = {n: x.cuda() for n, x in t.items()}
    cq, ck = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in (cu_q, cu_k))
    out, lse, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], cq, max_q, cu_k=ck, causal=causal, **kw)
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal)
    assert int(st) == 0
    ref.check(out, want["out"], bound["out"], what + " out")
    ref.check(lse, want["lse"], bound["lse"], what + " lse")
    return d, cq, ck, out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [0, 300, 500])
def test_one_long_list_among_short_ones(gpu, dtype, at):
    """501 new tokens, one with 60000 keys, the others with one or none; the longest known and not."""
    nk = [1 if i % 7 else 0 for i in range(501)]
    nk[at] = 60000
    t, cu_q, cu_k = make([1] * 501, nk, 4, 2, 64, dtype, at)
    for max_k in (0, 60000):
        forward(gpu, t, cu_q, cu_k, 1, True, f"longest {max_k}", max_k=max_k)
