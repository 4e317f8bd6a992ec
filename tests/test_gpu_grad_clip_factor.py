"""dora_grad_clip's factor at the ends of its range: no limit, and factors far
below what fp32 holds.  Tolerances as in test_gpu_grad_clip.py."""
import numpy as np
import pytest
import torch

from policy_ref import HALF, U32
from gpu_util import widen

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("bad", [None, INF, -INF, float("nan")])
def test_no_limit_out_of_place(gpu, bad):
    """Without a limit the factor is 1 whatever the norm: out gets the gradients."""
    g = torch.Generator("cuda").manual_seed(1)
    grads = [torch.randn(n, generator=g, device="cuda").to(t) for n, t in ((1000, torch.float32), (70001, torch.bfloat16),
                                                                          (0, torch.float32), (5, torch.bfloat16))]
    if bad is not None:
        grads[1][3] = bad
    out = [torch.full_like(t, 9.0) for t in grads]
    got, norm = gpu.dora_grad_clip(grads, INF, out=out)
    for a, b in zip(got, grads):
        assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    _, only = gpu.dora_grad_clip(grads, INF)
    assert torch.equal(norm.nan_to_num(7.0), only.nan_to_num(7.0))
    keep = [t.clone() for t in grads]
    gpu.dora_grad_clip(grads, INF, out=grads)                  # its own inputs: nothing to write
    for a, b in zip(grads, keep):
        assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


def test_no_limit_refuses_like_a_limit(gpu):
    g = torch.randn(10, device="cuda")
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([g], INF, out=[g[:5].clone()])
    assert e.value.code == gpu.DORA_ERR_SHAPE
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([g[:5], g[5:]], INF, out=[g[1:6], torch.empty_like(g[5:])])
    assert e.value.code == gpu.DORA_ERR_OVERLAP
    gpu.dora_grad_clip([g, g], INF)                            # only read
