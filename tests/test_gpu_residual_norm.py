"""The norms between two branches, forward and backward, against the 64-bit
reference, element by element."""
import itertools

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def inputs(T, C, dtype, kind, scale, gate, post, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)

    def rows(s=1.0):
        return (offset + s * torch.randn((T, C), generator=g)).to(dtype)
    t = dict(x=rows(2.0), a=rows(), dy=rows(), dh=rows())
    p = {"gamma": 1 + 0.1 * torch.randn(C, generator=g)}
    layer = kind == "layer"
    p["beta"] = 0.1 * torch.randn(C, generator=g) if layer else None
    p["scale"] = 0.5 + 0.1 * torch.randn(C, generator=g) if scale else None
    p["gate"] = (torch.rand(T, generator=g) >= 0.2).float() * 1.25 if gate else None
    p["post_gamma"] = 1 + 0.1 * torch.randn(C, generator=g) if post else None
    p["post_beta"] = 0.1 * torch.randn(C, generator=g) if post and layer else None
    return t, p


def cuda(d):
    return {n: None if t is None else t.cuda() for n, t in d.items()}


def compare_grads(got, want, bound, p, what=""):
    for n in got._fields:
        t = getattr(got, n)
        name = n[1:]
        if name in p and p[name] is None:
            assert t is None, n
            continue
        if t is not None:
            ref.check(t, want[n], bound[n], f"{what} {n}")


# widths on both sides of every change of lanes and pieces (16-byte pieces: 8 bf16, 4 fp32)
WIDTHS = [8, 16, 120, 128, 136, 256, 264, 504, 512, 520, 768, 1024, 1032, 2048, 2056, 4088, 4096, 4104, 8192]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(gpu, C, dtype):
    for i, (kind, scale, gate, post) in enumerate((("layer", True, True, True), ("rms", False, True, True),
                                                   ("layer", True, False, False), ("rms", False, False, False))):
        T = (5, 1, 19, 3)[i]
        t, p = inputs(T, C, dtype, kind, scale, gate, post, C + i)
        d, q = cuda(t), cuda(p)
        h, y = gpu.dora_residual_norm(d["x"], d["a"], kind=kind, **q)
        want, bound = ref.residual_norm(t["x"], t["a"], p, kind)
        ref.check(h, want["h"], bound["h"], f"h {i}")
        ref.check(y, want["y"], bound["y"], f"y {i}")
        got = gpu.dora_residual_norm_backward(d["dy"], h, d["a"], dh=d["dh"], kind=kind, **q)
        want, bound = ref.residual_norm_backward(t["dy"], t["dh"], h.cpu(), t["a"], p, kind)
        compare_grads(got, want, bound, p, f"{i}")
        if not (scale or gate or post):
            assert got.da is got.dx


@pytest.mark.parametrize("dtype,kind,scale,gate,post", itertools.product(DTYPES, ("layer", "rms"), (False, True),
                                                                         (False, True), (False, True)))
def test_many_rows(gpu, dtype, kind, scale, gate, post):
    """More rows than the GPU holds, more than a row's workgroups take at once."""
    T, C = 9001, 136
    t, p = inputs(T, C, dtype, kind, scale, gate, post, 7)
    d, q = cuda(t), cuda(p)
    h, y = gpu.dora_residual_norm(d["x"], d["a"], kind=kind, **q)
    want, bound = ref.residual_norm(t["x"], t["a"], p, kind)
    ref.check(h, want["h"], bound["h"], "h")
    ref.check(y, want["y"], bound["y"], "y")
    got = gpu.dora_residual_norm_backward(d["dy"], h, d["a"], dh=d["dh"], kind=kind, **q)
    again = gpu.dora_residual_norm_backward(d["dy"], h, d["a"], dh=d["dh"], kind=kind, **q)
    want, bound = ref.residual_norm_backward(t["dy"], t["dh"], h.cpu(), t["a"], p, kind)
    compare_grads(got, want, bound, p)
    for x, z in zip(got, again):
        assert x is None and z is None or torch.equal(x, z)


@pytest.mark.parametrize("T,C", [(2, 8192), (1500, 4096), (700, 1024), (3000, 512), (5, 16)])
def test_each_row_counts_once(gpu, T, C):
    """Sums over rows of 1s are exact whatever their order."""
    one = torch.ones((T, C), device="cuda")
    h = torch.cat([torch.ones((T, C // 2)), -torch.ones((T, C // 2))], 1).cuda()     # normed: itself, eps 0
    w = torch.ones(C, device="cuda")
    got = gpu.dora_residual_norm_backward(one, h, one, w, w, scale=w, gate=torch.ones(T, device="cuda"), dh=one,
                                          kind="layer", eps=0.0)
    assert bool((got.dbeta == T).all()) and bool((got.dgamma == T * h[0]).all())
    assert bool((got.dx == 1).all()) and bool((got.dscale == T).all()) and bool((got.dgate == C).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_partial_calls(gpu, dtype):
    """Only dy, only dh, no branch, no bias."""
    T, C = 33, 776
    t, p = inputs(T, C, dtype, "layer", True, True, True, 3)
    d, q = cuda(t), cuda(p)
    for dy, dh in (("dy", None), (None, "dh")):
        want, bound = ref.residual_norm_backward(t.get(dy), t.get(dh), t["x"], t["a"], p)
        got = gpu.dora_residual_norm_backward(d.get(dy), d["x"], d["a"], dh=d.get(dh), **q)
        compare_grads(got, want, bound, p, f"{dy} {dh}")
    just = {"gamma": p["gamma"], "beta": None}
    h, y = gpu.dora_residual_norm(d["x"], None, q["gamma"])
    want, bound = ref.residual_norm(t["x"], None, just)
    assert h is d["x"]
    ref.check(y, want["y"], bound["y"], "y")
    got = gpu.dora_residual_norm_backward(d["dy"], d["x"], None, q["gamma"])
    want, bound = ref.residual_norm_backward(t["dy"], None, t["x"], None, just)
    ref.check(got.dx, want["dx"], bound["dx"], "dx")
    ref.check(got.dgamma, want["dgamma"], bound["dgamma"], "dgamma")
    assert got.da is None and got.dbeta is None


@pytest.mark.parametrize("dtype", DTYPES)
def test_far_means(gpu, dtype):
    """Rows whose mean is far from 0 against their spread."""
    t, p = inputs(40, 1024, dtype, "layer", True, False, True, 4, offset=300.0 if dtype == torch.float32 else 10.0)
    d, q = cuda(t), cuda(p)
    h, y = gpu.dora_residual_norm(d["x"], d["a"], **q)
    want, bound = ref.residual_norm(t["x"], t["a"], p)
    ref.check(h, want["h"], bound["h"], "h")
    ref.check(y, want["y"], bound["y"], "y")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,C", [(50, 264), (700, 8192), (3000, 128)])
def test_in_place_and_strided(gpu, dtype, T, C):
    t, p = inputs(T, C, dtype, "layer", True, True, True, 6)
    d, q = cuda(t), cuda(p)
    h, y = gpu.dora_residual_norm(d["x"], d["a"], **q)
    g = gpu.dora_residual_norm_backward(d["dy"], h, d["a"], dh=d["dh"], **q)
    x, a = d["x"].clone(), d["a"].clone()
    gpu.dora_residual_norm(x, a, h_out=x, y_out=a, **q)
    assert torch.equal(x, h) and torch.equal(a, y)
    dy, dh = d["dy"].clone(), d["dh"].clone()
    g2 = gpu.dora_residual_norm_backward(dy, h, d["a"], dh=dh, dx=dh, da=dy, **q)
    assert torch.equal(dh, g.dx) and torch.equal(dy, g.da) and torch.equal(g2.dgamma, g.dgamma)
    a = d["a"].clone()
    hh = h.clone()
    gpu.dora_residual_norm_backward(d["dy"], hh, a, dh=d["dh"], dx=a, da=hh, **q)
    assert torch.equal(a, g.dx) and torch.equal(hh, g.da)
    wide = torch.full((T, 4 * C + 8), 7.0, dtype=dtype, device="cuda")
    parts = [wide[:, i * C:(i + 1) * C] for i in range(4)]
    parts[0].copy_(d["x"]), parts[1].copy_(d["a"])
    gpu.dora_residual_norm(parts[0], parts[1], h_out=parts[2], y_out=parts[3], **q)
    assert torch.equal(parts[2], h) and torch.equal(parts[3], y) and bool((wide[:, 4 * C:] == 7.0).all())
    one = d["x"][:1].expand(T, C)                                                     # one row read again and again
    got, _ = gpu.dora_residual_norm(one, d["a"], **q)
    want, bound = ref.residual_norm(t["x"][:1].expand(T, C), t["a"], p)
    ref.check(got, want["h"], bound["h"], "broadcast rows")


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_that_do_not_count(gpu, dtype):
    """A dropped row's branch; NaN and infinity stay in their row; a row of zeros."""
    T, C = 12, 264
    t, p = inputs(T, C, dtype, "rms", True, True, True, 8)
    p["gate"] = torch.ones(T)
    p["gate"][3] = 0.0
    t["a"][3] = float("nan")
    t["a"][3, 5] = float("inf")
    t["x"][6] = 0.0
    d, q = cuda(t), cuda(p)
    h, y = gpu.dora_residual_norm(d["x"], d["a"], kind="rms", **q)
    assert torch.equal(h[3], d["x"][3])
    ok = torch.ones(T, dtype=torch.bool)
    clean = t["a"].clone()
    clean[3] = 0.0
    want, bound = ref.residual_norm(t["x"], clean, p, "rms")
    ref.check(h, want["h"], bound["h"], "h")
    ref.check(y, want["y"], bound["y"], "y")
    got = gpu.dora_residual_norm_backward(d["dy"], h, d["a"], dh=d["dh"], kind="rms", **q)
    want, bound = ref.residual_norm_backward(t["dy"], t["dh"], h.cpu(), clean, p, "rms")
    assert bool((got.da[3] == 0).all())
    for n in ("dx", "da", "dscale", "dgamma", "dpost_gamma"):
        ref.check(getattr(got, n), want[n], bound[n], n)
    ok[3] = False
    ref.check(got.dgate.cpu()[ok], want["dgate"][ok], bound["dgate"][ok], "dgate")
    t["x"][9, 1] = float("nan")
    h, y = gpu.dora_residual_norm(t["x"].cuda(), d["a"], kind="rms", **q)
    rest = torch.arange(T) != 9
    assert bool(torch.isnan(y[9]).all()) and not bool(torch.isnan(y.cpu()[rest]).any())


def test_zero_rows(gpu):
    C = 64
    none, w = torch.empty((0, C), device="cuda"), torch.ones(C, device="cuda")
    h, y = gpu.dora_residual_norm(none, none.clone(), w)
    assert h.shape == y.shape == (0, C)
    got = gpu.dora_residual_norm_backward(none, none, none, w, w, scale=w)
    assert bool((got.dgamma == 0).all()) and bool((got.dbeta == 0).all()) and bool((got.dscale == 0).all())


def test_stream_and_versions(gpu):
    t, p = inputs(300, 768, torch.bfloat16, "layer", True, True, False, 10)
    d, q = cuda(t), cuda(p)
    h, y = gpu.dora_residual_norm(d["x"], d["a"], **q)
    g = gpu.dora_residual_norm_backward(d["dy"], h, d["a"], **q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h2, y2 = gpu.dora_residual_norm(d["x"], d["a"], stream=side, **q)
    g2 = gpu.dora_residual_norm_backward(d["dy"], h2, d["a"], stream=side, **q)
    side.synchronize()
    assert torch.equal(h, h2) and torch.equal(y, y2)
    assert all(a is None or torch.equal(a, b) for a, b in zip(g, g2))
    before = d["x"]._version
    gpu.dora_residual_norm(d["x"], d["a"], h_out=d["x"], **q)
    assert d["x"]._version > before
