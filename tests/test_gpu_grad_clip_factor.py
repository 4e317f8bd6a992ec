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


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1e-10, 1e-19, 1e-22, 1e-30, 1e-38, 1e-40, 1e-44, 0.0])
def test_small_factors(gpu, dtype, max_norm, in_place):
    """Gradients near fp32's limit under a small limit: a factor down to 2^-277.
    A subnormal result is a whole number of 2^-149 (bf16: 2^-133), off by half a
    step of that for each of its up to three roundings."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator("cuda").manual_seed(2)
    grads = [(3e38 * (2 * torch.rand(n, generator=g, device="cuda") - 1)).to(t) for n in (7, 3000, 20001)]
    ref = [widen(x) for x in grads]
    limit = float(np.float32(max_norm))
    norm = np.sqrt(sum((x ** 2).sum() for x in ref))
    c = limit / (norm + float(np.float32(1e-6)))
    got, _ = gpu.dora_grad_clip(grads, max_norm, out=None if in_place else [torch.empty_like(x) for x in grads])
    step = 2.0 ** (-149 if dtype == "f32" else -133)
    for x, w in zip(got, ref):
        w = w * c
        assert np.all(np.abs(widen(x) - w) <= (2.01 * U32 + HALF[dtype]) * np.abs(w) + 1.5 * step)
