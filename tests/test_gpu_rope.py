"""Rotary positions against the 64-bit reference, element by element."""
import itertools

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def inputs(T, H, D, R, axes, far, dtype, seed, Hk=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, H + Hk, D), generator=g).to(dtype)
    pos = torch.randint(-far, far + 1, (T, axes), generator=g, dtype=torch.int32)
    freq = torch.rand(R // 2, generator=g, dtype=torch.float64)
    return x, pos, freq


@pytest.mark.parametrize("dtype,interleaved,inverse", itertools.product(DTYPES, (False, True), (False, True)))
@pytest.mark.parametrize("T,H,Hk,D,R,axes,far", [
    (1, 1, 0, 2, 2, 1, 3), (1, 32, 8, 128, 128, 1, 2 ** 31 - 1), (7, 3, 0, 20, 12, 3, 100), (13, 5, 1, 64, 64, 2, 14),
    (300, 12, 12, 64, 32, 1, 577), (37, 4, 2, 96, 40, 4, 9), (5, 2, 1, 1024, 1024, 1, 10 ** 6), (4099, 2, 1, 32, 16, 1, 8192),
    (3, 200, 200, 33, 18, 1, 50)])
def test_rope(gpu, T, H, Hk, D, R, axes, far, dtype, interleaved, inverse):
    x, pos, freq = inputs(T, H, D, R, axes, min(far, 2 ** 31 - 2), dtype, T + D, Hk)
    q = x[:, :H].cuda()
    k = x[:, H:].cuda() if Hk else None
    scale = 1.25
    qo, ko = gpu.dora_rope(q, pos.cuda() if axes > 1 else pos[:, 0].contiguous().cuda(), freq.cuda(), k=k,
                           interleaved=interleaved, inverse=inverse, scale=scale)
    want, bound = ref.rope(x, pos, freq, interleaved, inverse, scale)
    ref.check(qo, want[:, :H], bound[:, :H], "q")
    assert (ko is None) == (Hk == 0)
    if Hk:
        ref.check(ko, want[:, H:], bound[:, H:], "k")


@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(gpu, dtype):
    """Slices of one product, heads before rows, odd addresses, in place; what lies between stays."""
    T, H, Hk, D, R = 33, 4, 2, 64, 48
    x, pos, freq = inputs(T, H, D, R, 1, 500, dtype, 5, Hk)
    want, bound = ref.rope(x, pos, freq, False, False, 1.0)
    p, f = pos[:, 0].contiguous().cuda(), freq.cuda()
    fused = torch.full((T, H + 2 * Hk + 1, D), 7.0, dtype=dtype, device="cuda")
    fused[:, :H + Hk] = x.cuda()
    gpu.dora_rope(fused[:, :H], p, f, k=fused[:, H:H + Hk], q_out=fused[:, :H], k_out=fused[:, H:H + Hk])
    ref.check(fused[:, :H + Hk], want, bound, "in place")
    assert bool((fused[:, H + Hk:] == 7.0).all())
    turned = torch.empty((H, T, D), dtype=dtype, device="cuda").transpose(0, 1)
    gpu.dora_rope(x[:, :H].cuda().transpose(0, 1).contiguous().transpose(0, 1), p, f, q_out=turned)
    ref.check(turned, want[:, :H], bound[:, :H], "heads first")
    odd = torch.full((T * (H * (D + 1) + 3) + 1,), 7.0, dtype=dtype, device="cuda")
    view = odd[1:].as_strided((T, H, D), (H * (D + 1) + 3, D + 1, 1), 1)
    view.copy_(x[:, :H].cuda())
    out = torch.full_like(odd, 9.0)
    gpu.dora_rope(view, p, f, q_out=out.as_strided(view.shape, view.stride(), 1))
    ref.check(out.as_strided(view.shape, view.stride(), 1), want[:, :H], bound[:, :H], "odd strides")
    rest = torch.ones_like(out, dtype=torch.bool)
    rest.as_strided(view.shape, view.stride(), 1).fill_(False)
    assert bool((out[rest] == 9.0).all())
    wide = x[:, :1].cuda().expand(T, 3, D)                     # one head read three times
    got, _ = gpu.dora_rope(wide, p, f)
    ref.check(got, want[:, :1].expand(T, 3, D), bound[:, :1].expand(T, 3, D), "broadcast head")


def test_special_values_and_zero_rows(gpu):
    x = torch.tensor([float("inf"), 1.0, float("nan"), 2.0, 3.0, float("-inf")], device="cuda").view(1, 1, 6)
    freq = torch.tensor([0.5, 0.25], dtype=torch.float64, device="cuda")
    y, _ = gpu.dora_rope(x, torch.tensor([0], dtype=torch.int32, device="cuda"), freq, interleaved=True)
    y = y.flatten().tolist()
    assert y[0] == float("inf") and y[1] != y[1] and y[2] != y[2] and y[3] != y[3]
    assert y[4] == 3.0 and y[5] == float("-inf")                     # copied
    none = torch.empty((0, 2, 8), device="cuda")
    out, _ = gpu.dora_rope(none, torch.empty(0, dtype=torch.int32, device="cuda"), freq)
    assert out.shape == (0, 2, 8)


def test_long_offsets(gpu):
    """Rows further apart than 2^31 elements."""
    T, D = 3, 64
    big = torch.empty(2 * (1 << 31) + D, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((T, 1, D), (1 << 31, D, 1))
    x, pos, freq = inputs(T, 1, D, D, 1, 1000, torch.bfloat16, 3)
    view.copy_(x.cuda())
    gpu.dora_rope(view, pos[:, 0].contiguous().cuda(), freq.cuda(), q_out=view)
    want, bound = ref.rope(x, pos, freq, False, False, 1.0)
    ref.check(view, want, bound, "far rows")


def test_stream_and_versions(gpu):
    x, pos, freq = inputs(64, 4, 64, 64, 1, 100, torch.float32, 9)
    q, p, f = x.cuda(), pos[:, 0].contiguous().cuda(), freq.cuda()
    want, _ = gpu.dora_rope(q, p, f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = gpu.dora_rope(q, p, f, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    before = q._version
    gpu.dora_rope(q, p, f, q_out=q)
    assert q._version > before


def test_frequencies(gpu):
    f = gpu.rope_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and f[0] == 1.0 and abs(float(f[1]) - 10000 ** (-1 / 32)) < 1e-15
    assert torch.allclose(gpu.rope_frequencies(64, factor=4.0, device="cpu"), f / 4)
    g = gpu.rope_frequencies(64, factor=4.0, trained=4096, device="cpu")
    turns = 4096 * f / (2 * torch.pi)
    assert torch.equal(g[turns > 32], f[turns > 32]) and torch.allclose(g[turns < 1], f[turns < 1] / 4)
    assert bool(((g >= f / 4) & (g <= f)).all())
    with pytest.raises(ValueError):
        gpu.rope_frequencies(7)
