"""GPU parity of dora_pl_policy_loss with the formula in 64 bits, its sums
formed from scratch at every step (policy_ref.pl).

The kernel works in 64 bits and rounds its results to fp32: u = 2^-24 relative
of the log-probability and of each gradient, plus 64-bit rounding (sums of up
to 2047 terms, 1e-12 of the sizes involved)."""
import numpy as np
import pytest
import torch

import policy_ref as P
from gpu_util import cu_of, to_dev

pytestmark = pytest.mark.gpu


def make(lens, N=None, packed=False, seed=0, spread=2.0, frac=0.6, ks=None, ref=True, low=0.2, high=0.28):
    rng = np.random.default_rng([seed, len(lens), int(max(lens))])
    cu = cu_of(lens)
    s = (spread * rng.standard_normal(int(cu[-1]))).astype(np.float32)
    segs = [(int(cu[b]), int(n)) for b, n in enumerate(lens)]
    order, k = [], []
    for b, (off, n) in enumerate(segs):
        kb = int(ks[b]) if ks is not None else int(rng.integers(0, int(frac * (n - 1)) + 1))
        key = s[off + 1:off + n] + spread * rng.gumbel(size=n - 1)
        order.append(1 + np.argsort(-key)[:kb])
        k.append(kb)
    order, cuo = np.concatenate(order).astype(np.int32), cu_of(k)
    h = dict(s=s, order=order, cuo=cuo, cu=cu if packed else None, N=int(max(lens)), segs=segs, low=low, high=high)
    B = len(lens)
    z = np.zeros(B)
    lp = P.pl(s.astype(np.float64), order, cuo, z, z, segments=segs)[1]
    h["old"] = P.off_border(lp, 0.3 * rng.standard_normal(B), low, high)
    h["A"] = rng.standard_normal(B).astype(np.float32)
    h["ref"] = (lp + 0.3 * rng.standard_normal(B)).astype(np.float32) if ref else None
    h["weight"] = None
    return h


def run(dora, h, kl=0.0, **kw):
    s = to_dev(h["s"]) if h["cu"] is not None else to_dev(h["s"]).view(len(h["segs"]), -1)
    order = h["order"] if len(h["order"]) else np.zeros(1, np.int32)
    dev = lambda a: None if a is None else to_dev(a)
    out = dora.dora_pl_policy_loss(s if "scores" not in kw else kw.pop("scores"), dev(order), dev(h["cuo"]), dev(h["old"]),
                                   dev(h["A"]), ref_logprob=dev(h["ref"]), weight=dev(h["weight"]), cu_in=dev(h["cu"]),
                                   N=h["N"], clip_low=h["low"], clip_high=h["high"],
                                   kl_coef=kl if h["ref"] is not None else 0.0, **kw)
    torch.cuda.synchronize()
    return out


def check(dora, h, kl=0.05, **kw):
    f32 = lambda v: float(np.float32(v))
    g, lp, stats, scale = P.pl(h["s"].astype(np.float64), h["order"], h["cuo"], h["old"].astype(np.float64),
                               h["A"].astype(np.float64), None if h["ref"] is None else h["ref"].astype(np.float64),
                               h["weight"], h["segs"], f32(h["low"]), f32(h["high"]),
                               f32(kl) if h["ref"] is not None else 0.0)
    ds, glp, st, flag = run(dora, h, kl, **kw)
    assert int(flag.item()) == 0
    u = P.U32
    size = np.array([np.abs(h["s"][o:o + n]).max() * (n + 1) for o, n in h["segs"]])   # the sums' size
    lim = u * np.abs(lp) + 1e-12 * size
    got = glp.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - lp) <= lim), np.abs(got - lp).max()
    got = ds.cpu().numpy().astype(np.float64).reshape(-1)
    for b, (o, n) in enumerate(h["segs"]):
        sl = slice(o, o + n)
        # dscores is slope times a difference, 1 - exp(s_j) sum 1 / S: its two sides are up to the number of draws, each
        # with a few 2^-53 of itself (1 - x (1 / x) is 2^-53, not 0), so the error scales with slope, not with what is left
        w = 1.0 if h["weight"] is None else float(h["weight"][b])
        pull = w * (abs(float(h["A"][b])) * np.exp(lp[b] - float(h["old"][b])) +
                    (0.0 if h["ref"] is None else kl * (1 + np.exp(float(h["ref"][b]) - lp[b])))) if w else 0.0
        assert np.all(np.abs(got[sl] - g[sl]) <= u * np.abs(g[sl]) + 1e-11 * (1 + size[b]) * pull + 1e-38), b
    got = st.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - stats) <= u * np.abs(stats) + 1e-11 * (1 + size.max()) * scale + 1e-30), (got, stats)
    return ds, glp, st


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B,N", [(1, 1), (3, 2), (4, 3), (9, 17), (5, 64), (5, 65), (7, 197), (6, 257), (5, 258), (4, 577),
                                 (2, 1025), (3, 2048)])
def test_sizes(gpu, B, N, packed):
    lens = np.full(B, N)
    if packed and B > 1:
        lens = np.random.default_rng(N).integers(1, N + 1, B)
        lens[0] = N
    check(gpu, make(lens, packed=packed, seed=1))


@pytest.mark.parametrize("B,N", [(1100, 130), (1030, 321), (1025, 800)])
def test_many_images(gpu, B, N):
    """Batches and lengths that take workgroups of other widths."""
    lens = np.random.default_rng(B).integers(1, N + 1, B)
    lens[7] = N
    check(gpu, make(lens, packed=True, seed=12, frac=0.15))


@pytest.mark.parametrize("N", [2, 5, 197, 258, 2048])
def test_no_draw_one_and_all(gpu, N):
    h = make([N] * 3, ks=[0, 1, N - 1], seed=2)
    ds, lp, _ = check(gpu, h)
    assert not bool(ds[0].any()) and float(lp[0]) == 0.0
    assert not bool(ds[:, 0].any())                       # CLS


def test_no_reference(gpu):
    check(gpu, make([50] * 4, seed=3, ref=False), kl=0.0)


@pytest.mark.parametrize("spread", [1e-3, 30.0, 3000.0, 1e6])
def test_scores_far_apart(gpu, spread):
    """Tokens a thousand and more below the largest, drawn late: their own
    shares, no division of zero by zero."""
    h = make([60] * 4, ks=[59, 30, 58, 1], seed=4, spread=spread)
    check(gpu, h)
    h = make([200] * 3, ks=[199, 100, 3], seed=5, spread=spread)
    h["s"][100:140] = h["s"][100]                         # equal scores
    lp = P.pl(h["s"].astype(np.float64), h["order"], h["cuo"], np.zeros(3), np.zeros(3), segments=h["segs"])[1]
    h["old"], h["ref"] = (lp - 0.1).astype(np.float32), (lp + 0.1).astype(np.float32)
    if np.abs(lp).max() * P.U32 < 0.01:                   # else the stored old one is no longer off the border
        check(gpu, h)


@pytest.mark.parametrize("spread", [2.0, 3000.0])
@pytest.mark.parametrize("n,masked", [(2, 1), (40, 7), (200, 400), (700, 1300)])
def test_masked_scores(gpu, n, masked, spread):
    """Scores of -inf that no draw takes are as if the tokens were not there."""
    want = make([n] * 3, ks=[n - 1, n // 2, 0], seed=8, spread=spread, ref=False)
    g, lp, _, _ = P.pl(want["s"].astype(np.float64), want["order"], want["cuo"], want["old"].astype(np.float64),
                       want["A"].astype(np.float64), segments=want["segs"], low=float(np.float32(want["low"])),
                       high=float(np.float32(want["high"])))
    N = n + masked
    h = dict(want, s=np.full(3 * N, -np.inf, np.float32), order=want["order"].copy(), N=N,
             segs=[(b * N, N) for b in range(3)])
    rng = np.random.default_rng(n)
    at = [1 + np.sort(rng.permutation(N - 1)[:n - 1]) for _ in range(3)]    # where each image's open tokens stand
    for b in range(3):
        h["s"][b * N + at[b]] = want["s"][b * n + 1:(b + 1) * n]
        sl = slice(want["cuo"][b], want["cuo"][b + 1])
        h["order"][sl] = at[b][want["order"][sl] - 1]
    ds, got, _, flag = run(gpu, h)
    assert int(flag.item()) == 0
    size = np.abs(want["s"]).max() * (n + 1)
    assert np.all(np.abs(got.cpu().numpy() - lp) <= P.U32 * np.abs(lp) + 1e-12 * size)
    ds = ds.cpu().numpy().astype(np.float64)
    for b in range(3):
        pull = abs(float(want["A"][b])) * np.exp(lp[b] - float(want["old"][b]))
        w = g[b * n + 1:(b + 1) * n]
        assert np.all(np.abs(ds[b, at[b]] - w) <= P.U32 * np.abs(w) + 1e-11 * (1 + size) * pull + 1e-38)
        ds[b, at[b]] = 0.0
    assert not ds.any()


def test_masked_score_drawn(gpu):
    """A draw of probability 0: log-probability -inf, ratio 0, gradient 0."""
    h = make([30] * 3, ks=[6, 6, 6], seed=9, ref=False)
    h["s"][h["order"][2]] = -np.inf                       # the first image's third draw
    h["A"][:] = [1.0, -1.0, 0.5]
    want = make([30] * 3, ks=[6, 6, 6], seed=9, ref=False)
    want["A"][:] = h["A"]
    clean = run(gpu, want)
    ds, lp, st, flag = run(gpu, h)
    assert int(flag.item()) == 0 and float(lp[0]) == -np.inf and not bool(ds[0].any())
    assert torch.equal(ds[1:], clean[0][1:]) and torch.equal(lp[1:], clean[1][1:]) and bool(st.isfinite().all())
    assert float(gpu.dora_pl_logprob(to_dev(h["s"]).view(3, 30), to_dev(h["order"]), to_dev(h["cuo"]))[0][0]) == -np.inf


def test_agrees_with_logprob(gpu):
    h = make([197] * 32, seed=6)
    lp, st = gpu.dora_pl_logprob(to_dev(h["s"]).view(32, 197), to_dev(h["order"]), to_dev(h["cuo"]))
    _, lp2, _, _ = run(gpu, h)
    # dora_pl_logprob: fp32 sums, at most (n + 16) u a term over k terms, and the terms' own size
    k = np.diff(h["cuo"])
    lim = P.U32 * (k * (197 + 40) + 8 * np.abs(lp2.cpu().numpy()))
    assert np.all((lp - lp2).abs().cpu().numpy() <= lim)


def test_padding_and_bad_images(gpu):
    h = make([40, 30, 20, 25, 33, 18, 22], packed=True, ks=[5, 6, 7, 8, 4, 3, 6], seed=7)
    h["weight"] = np.full(7, 0.25, np.float32)
    h["weight"][1] = 0.0
    want = check(gpu, h)
    c = h["cuo"]
    h["s"][h["segs"][1][0]:h["segs"][1][0] + 30] = np.nan      # padding: anything
    h["order"][c[1]] = 99
    h["old"][1] = h["A"][1] = h["ref"][1] = np.nan
    got = run(gpu, h, 0.05)
    assert int(got[3].item()) == 0 and float(got[1][1]) == 0.0
    for a, b in zip(got[:3], want):
        assert torch.equal(a, b)
    h["order"][c[2]] = h["order"][c[2] + 1]                     # twice the same
    h["order"][c[3]] = 0                                        # CLS
    h["order"][c[4] + 1] = 33                                   # past the end
    ds, lp, st, flag = run(gpu, h, 0.05)
    assert int(flag.item()) == gpu.DORA_DEV_KEEP_RANGE
    assert bool(torch.isnan(lp[2:5]).all()) and bool(torch.isfinite(lp[[0, 1, 5, 6]]).all())
    for b in (1, 2, 3, 4):
        o, n = h["segs"][b]
        assert not bool(ds[o:o + n].any())
    for b in (0, 5, 6):
        o, n = h["segs"][b]
        assert torch.equal(ds[o:o + n], want[0][o:o + n])
    assert float(st[5]) == 0.75


def test_bad_offsets(gpu):
    """Offsets of draws and of segments out of their ranges: reported, nothing
    outside the scores' extent is written."""
    h = make([20] * 4, packed=True, ks=[3, 3, 3, 3], seed=8)
    good = {k: np.copy(v) if isinstance(v, np.ndarray) else v for k, v in h.items()}
    h["cuo"] = np.array([0, 3, 30, 9, 12], np.int32)           # past the list's end, then back
    ds, lp, _, flag = run(gpu, h)
    assert int(flag.item()) == gpu.DORA_DEV_KEEP_RANGE and bool(torch.isnan(lp[1:3]).all())
    h = {**good, "cu": np.array([0, 20, 40, 95, 80], np.int32)}  # past the scores' end; then negative
    room = torch.full((80,), 5.0, device="cuda")
    ds, lp, _, flag = run(gpu, h, dscores=room)
    assert int(flag.item()) == gpu.DORA_DEV_CU_IN
    assert bool(torch.isnan(lp[2:]).all()) and bool((ds[40:] == 5).all()) and bool(torch.isfinite(lp[:2]).all())


def test_rows_behind_the_last_segment(gpu):
    h = make([12, 9], packed=True, ks=[4, 2], seed=9)
    want = run(gpu, h, 0.05)
    h["s"] = np.concatenate([h["s"], np.full(11, np.nan, np.float32)])
    room = torch.full((32,), 5.0, device="cuda")
    ds, lp, st, flag = run(gpu, h, 0.05, dscores=room)
    assert torch.equal(ds[:21], want[0]) and bool((ds[21:] == 5).all()) and torch.equal(lp, want[1])


def test_in_place_and_repeats(gpu):
    h = make([577] * 40, seed=10)
    want = run(gpu, h, 0.05)
    s = to_dev(h["s"]).view(40, 577)
    got = run(gpu, h, 0.05, scores=s, dscores=s)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)


def test_most_images(gpu):
    """As many images as a call takes, on draws that the library makes."""
    g = torch.Generator("cuda").manual_seed(1)
    s = torch.randn((8192, 30), generator=g, device="cuda")
    u = torch.rand((8192, 30), generator=g, device="cuda").clamp_(1e-6, 1 - 1e-6)
    k = torch.randint(0, 30, (8192,), generator=g, device="cuda", dtype=torch.int32)
    order, cuo, lp, st = gpu.dora_pl_sample(s, -torch.log(-torch.log(u)), k)
    one = torch.ones(8192, device="cuda")
    ds, lp2, stats, flag = gpu.dora_pl_policy_loss(s, order, cuo, lp, one)
    assert int(flag.item()) == 0 and float(stats[5]) == 8192
    # shifting all scores of an image changes nothing: gradients sum to zero (28 fp32 roundings of terms up to 30 in all)
    assert float(ds.sum(1).abs().max()) <= 1e-4
    assert abs(float(stats[1]) - 8192) <= 8192 * 30 * 70 * P.U32


def test_refusals(gpu):
    h = make([20] * 4, seed=11)
    s = to_dev(h["s"]).view(4, 20)
    with pytest.raises(gpu.DoraError) as e:
        run(gpu, {**h, "N": 20}, scores=s.new_zeros((4, 2049)))
    assert e.value.code == gpu.DORA_ERR_SHAPE
    with pytest.raises(ValueError, match="dense scores"):
        run(gpu, h, scores=s[:3])
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_pl_policy_loss(s, to_dev(h["order"]), to_dev(h["cuo"]), to_dev(h["old"]), to_dev(h["A"]), kl_coef=0.1)
    assert e.value.code == gpu.DORA_ERR_NULL
    with pytest.raises(ValueError, match="contiguous"):
        run(gpu, h, scores=torch.zeros((20, 4), device="cuda").t())
