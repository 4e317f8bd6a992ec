"""GPU parity of dora_grad_clip with numpy in 64 bits.

The squares are added in 64 bits: the norm is within u = 2^-24 of its storage
in fp32.  An output is the gradient times the factor (rounded to fp32: u) in
fp32 (u), rounded once to its type."""
import numpy as np
import pytest
import torch

import policy_ref as P
from gpu_util import to_dev, widen

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(sizes, dtypes, seed=0, scale=1.0):
    rng = np.random.default_rng([seed, len(sizes)])
    return [torch.from_numpy((scale * rng.standard_normal(n)).astype(np.float32)).to(DT[d]).cuda()
            for n, d in zip(sizes, dtypes)]


def check(dora, grads, max_norm, in_place=False, **kw):
    ref = [widen(g) for g in grads]
    want, norm = P.clip(ref, float(np.float32(max_norm)))
    keep = [g.clone() for g in grads]
    out = None if in_place else [torch.full_like(g, 9.0) for g in grads]
    got, gn = dora.dora_grad_clip(grads, max_norm, out=out, **kw)
    torch.cuda.synchronize()
    u = P.U32
    assert gn.shape == (1,)
    if norm > np.finfo(np.float32).max:      # not to be held in fp32; the factor is formed before it is stored there
        assert float(gn) == np.inf
    else:
        assert abs(float(gn) - norm) <= u * norm * (1 + 1e-6)
    for g, w, k, src in zip(got, want, keep, grads):
        half = P.HALF["bf16" if g.dtype == torch.bfloat16 else "f32"]
        e = np.abs(widen(g) - w)
        assert np.all(e <= (2.01 * u + half) * np.abs(w) + 1e-38), e.max()   # 1e-38: subnormal results
        if not in_place:
            assert torch.equal(src, k)
    return got, gn


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[1], [7], [8], [0, 1, 0], [16383], [16384], [16385], [100000, 3, 0, 40001],
                                   [3000001], [1] * 95, [5] * 96, [13] * 97, list(range(300))])
def test_sizes(gpu, sizes, dtype, in_place):
    check(gpu, make(sizes, [dtype] * len(sizes), seed=1), 0.5, in_place)


def test_mixed_types_and_shapes(gpu):
    rng = np.random.default_rng(2)
    sizes = rng.integers(1, 5000, 150)
    grads = make(sizes, [("f32", "bf16")[i % 2] for i in range(150)], seed=2)
    grads[3] = torch.randn((7, 11, 13), device="cuda")
    grads[4] = torch.tensor(2.5, device="cuda")          # no dimension
    check(gpu, grads, 1.0)
    check(gpu, grads, 1.0, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lead", [1, 2, 3, 5, 7])
def test_unaligned_views(gpu, dtype, lead):
    """Views of one buffer at every offset, neighbours untouched."""
    sizes = [1, 2, 3, 15, 16, 17, 31, 33, 4097, 20001, 8, 9]
    flat = torch.randn(sum(sizes) + lead + 3, device="cuda").to(DT[dtype])
    keep = flat.clone()
    grads = list(flat[lead:lead + sum(sizes)].split(sizes))
    room = torch.full((flat.numel() + 4,), 9.0, device="cuda").to(DT[dtype])
    out = list(room[lead + 1:lead + 1 + sum(sizes)].split(sizes))     # shifted against the gradients
    want, _ = gpu.dora_grad_clip([g.clone() for g in grads], 0.25, out=[torch.empty_like(g) for g in grads])
    got, _ = gpu.dora_grad_clip(grads, 0.25, out=out)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert bool((room[:lead + 1] == 9).all()) and bool((room[lead + 1 + sum(sizes):] == 9).all())
    assert torch.equal(flat, keep)
    gpu.dora_grad_clip(grads, 0.25)
    for a, b in zip(grads, want):
        assert torch.equal(a, b)
    assert torch.equal(flat[:lead], keep[:lead]) and torch.equal(flat[lead + sum(sizes):], keep[lead + sum(sizes):])


@pytest.mark.parametrize("in_place", [False, True])
def test_nothing_to_clip(gpu, in_place):
    """Below the limit the gradients come out to the last bit."""
    grads = make([1000, 70000], ["f32", "bf16"], seed=3, scale=1e-3)
    keep = [g.clone() for g in grads]
    got, _ = check(gpu, grads, 1e9, in_place)
    for a, b in zip(got, keep):
        assert torch.equal(a, b)


def test_norm_only(gpu):
    grads = make([1000, 70000, 0, 5], ["f32", "bf16", "f32", "bf16"], seed=4)
    keep = [g.clone() for g in grads]
    _, n = gpu.dora_grad_clip(grads, float("inf"))
    norm = P.clip([widen(g) for g in grads], 1.0)[1]
    assert abs(float(n) - norm) <= P.U32 * norm * (1 + 1e-6)
    for a, b in zip(grads, keep):
        assert torch.equal(a, b)


def test_zero_and_empty(gpu):
    for grads in ([torch.zeros(5, device="cuda")], [torch.empty(0, device="cuda")], [torch.empty(0, device="cuda")] * 200):
        out, n = gpu.dora_grad_clip(grads, 0.0, eps=0.0)
        assert float(n) == 0.0 and not any(bool(g.any()) for g in out)


@pytest.mark.parametrize("big", [1e30, 3e38, 1e-30, 1e-38])
def test_squares_past_fp32(gpu, big):
    grads = [torch.full((300,), big, device="cuda"), torch.full((4,), big / 2, device="cuda")]
    check(gpu, grads, 1.0)


def test_nan_and_infinity(gpu):
    g = [torch.ones(10, device="cuda"), torch.ones(10, device="cuda", dtype=torch.bfloat16)]
    g[1][3] = float("inf")
    out, n = gpu.dora_grad_clip(g, 1.0, out=[torch.empty_like(t) for t in g])
    assert float(n) == float("inf") and not bool(out[0].any()) and bool(torch.isnan(out[1][3])) and not bool(out[1][:3].any())
    g[1][3] = float("nan")
    out, n = gpu.dora_grad_clip(g, 1.0, out=[torch.empty_like(t) for t in g])
    assert bool(torch.isnan(n).all()) and all(bool(torch.isnan(t).all()) for t in out)


def test_large_tensor(gpu):
    """More than 2^32 bytes in one tensor, and more chunks than workgroups."""
    n = (1 << 31) + 77
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    g[-1] = 100.0
    out, norm = gpu.dora_grad_clip([g, torch.ones(3, device="cuda")], 1.0)
    want = np.sqrt(0.25 * (n - 1) + 1e4 + 3)
    assert abs(float(norm) - want) <= P.U32 * want * 1.01
    c = 1 / (want + 1e-6)
    tail = out[0][-5:].double().cpu().numpy()
    assert np.all(np.abs(tail - c * np.array([.5, .5, .5, .5, 100])) <= P.HALF["bf16"] * 1.01 * c * np.array([.5, .5, .5, .5, 100]))
    head = out[0][0]
    assert bool((out[0][:-1] == head).all())


def test_repeats_to_the_last_bit(gpu):
    grads = make([100003] * 30 + [17] * 130, ["f32", "bf16"] * 80, seed=5)
    a = gpu.dora_grad_clip(grads, 0.5, out=[torch.empty_like(g) for g in grads])
    ws = torch.randint(0, 255, (gpu.dora_grad_clip_workspace_size(160),), dtype=torch.uint8, device="cuda")
    b = gpu.dora_grad_clip(grads, 0.5, out=[torch.empty_like(g) for g in grads], workspace=ws)
    assert torch.equal(a[1], b[1]) and all(torch.equal(x, y) for x, y in zip(a[0], b[0]))


def test_same_input_twice_out_of_place(gpu):
    g = torch.randn(1000, device="cuda")
    check(gpu, [g, g], 0.5)


def test_refusals(gpu):
    g = torch.randn(10, device="cuda")
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([g, g], 1.0)
    assert e.value.code == gpu.DORA_ERR_OVERLAP
    with pytest.raises(ValueError, match=r"grads\[1\] must be contiguous"):
        gpu.dora_grad_clip([g, torch.zeros((4, 4), device="cuda").t()], 1.0)
    with pytest.raises(ValueError, match=r"grads\[1\] must be on the GPU"):
        gpu.dora_grad_clip([g, torch.zeros(4)], 1.0)
    with pytest.raises(TypeError, match="dtype"):
        gpu.dora_grad_clip([g.half()], 1.0)
    with pytest.raises(ValueError, match="for each"):
        gpu.dora_grad_clip([g], 1.0, out=[])
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([g], 1.0, out=[g[:5].clone()])
    assert e.value.code == gpu.DORA_ERR_SHAPE
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([g], -1.0)
    assert e.value.code == gpu.DORA_ERR_SHAPE
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([g] * 200, 1.0, workspace=gpu.new_grad_clip_workspace(200)[:-1], out=[g.clone() for _ in range(200)])
    assert e.value.code == gpu.DORA_ERR_WORKSPACE
    # by ctypes, as where the native marshalling is not built
    spans, device = gpu._spans((t for t in [g, g.bfloat16()]), "grads")
    assert [s.numel for s in spans] == [10, 10] and [s.dtype for s in spans] == [0, 1] and spans[0].data == g.data_ptr()
