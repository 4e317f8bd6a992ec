"""Ordered-draw loss with scores of any size: masks of a finite low value, and
images whose scores are all alike far from 0.  Only differences of scores
count, so a mask that no draw takes is a token that is not there, and equal
scores are a uniform draw wherever they lie.

The reference (policy_ref.pl) forms each step's differences to the largest score
left, exactly.  The kernel works in 64 bits on scores that count (those within
sight of a draw) of size |s|: 8 n |s| 2^-53 for log p (and its storage in fp32),
and twice that times the slope for a gradient; equal scores' differences are
exact, which leaves the sums' own roundings, n log n 2^-50."""
import numpy as np
import pytest

import policy_ref as P
from test_gpu_pl_policy import run

LOWEST = float(np.finfo(np.float32).min)
KL = 0.05


def image_set(images, low=0.2, high=0.28, seed=0):
    """images: (scores of the visual tokens, draws as positions from 1, size of the scores that count)."""
    rng = np.random.default_rng(seed)
    N = 1 + max(len(x) for x, _, _ in images)
    s = np.concatenate([np.concatenate([[7.0], x]).astype(np.float32) for x, _, _ in images])
    lens = [len(x) + 1 for x, _, _ in images]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cuo = np.concatenate([[0], np.cumsum([len(d) for _, d, _ in images])]).astype(np.int32)
    B = len(images)
    h = dict(s=s, order=np.concatenate([d for _, d, _ in images]).astype(np.int32), cuo=cuo, cu=cu, N=N,
             segs=[(int(cu[b]), lens[b]) for b in range(B)], low=low, high=high, weight=None)
    z = np.zeros(B)
    lp = P.pl(s.astype(np.float64), h["order"], cuo, z, z, segments=h["segs"])[1]
    h["old"] = P.off_border(lp, 0.3 * rng.standard_normal(B), low, high)
    h["A"] = rng.standard_normal(B).astype(np.float32)
    h["ref"] = (lp + 0.3 * rng.standard_normal(B)).astype(np.float32)
    lim = np.array([8 * len(x) * size * 2.0 ** -53 + len(x) * np.log(len(x) + 1) * 2.0 ** -50 for x, _, size in images])
    return h, lim


def compare(dora, h, lim):
    f = lambda v: float(np.float32(v))
    g, lp, stats, scale = P.pl(h["s"].astype(np.float64), h["order"], h["cuo"], h["old"].astype(np.float64),
                               h["A"].astype(np.float64), h["ref"].astype(np.float64), None, h["segs"], f(h["low"]),
                               f(h["high"]), f(KL))
    assert np.isfinite(g).all() and np.isfinite(lp).all() and np.isfinite(stats).all()
    ds, glp, st, flag = run(dora, h, KL)
    assert int(flag.item()) == 0
    u, ds = P.U32, ds.cpu().numpy().astype(np.float64)
    got = glp.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - lp) <= u * np.abs(lp) + lim), (got, lp)
    for b, (o, n) in enumerate(h["segs"]):
        pull = abs(float(h["A"][b])) * np.exp(lp[b] - float(h["old"][b])) + KL * (1 + np.exp(float(h["ref"][b]) - lp[b]))
        w = g[o:o + n]
        assert np.all(np.abs(ds[o:o + n] - w) <= u * np.abs(w) + 2 * pull * lim[b] + 1e-38), b
    assert np.all(np.abs(st.cpu().numpy() - stats) <= u * np.abs(stats) + 2 * lim.max() * scale + 1e-30)
    return ds


MASKS = [LOWEST, -1e38, -1e30, -1e20, -1e18, -1e9, -65504.0, -1e4]


@pytest.mark.gpu
@pytest.mark.parametrize("n", [20, 300, 2047])
@pytest.mark.parametrize("mask", MASKS)
def test_masked_by_a_low_value(gpu, mask, n):
    """Not drawn: as if absent, and without a gradient.  Images with nothing
    masked, one token left, and half of them."""
    rng = np.random.default_rng([n, int(np.log10(-mask))])
    images, masked = [], []
    for opened in (n, 1, n // 2, n // 2):
        x = 2 * rng.standard_normal(n)
        at = rng.permutation(n)
        x[at[opened:]] = mask
        take = 1 if opened == 1 else int(rng.integers(1, opened))
        key = x[at[:opened]] + rng.gumbel(size=opened)
        images.append((x, 1 + at[:opened][np.argsort(-key)[:take]], 10.0))
        masked.append(1 + at[opened:])
    h, lim = image_set(images, seed=n)
    ds = compare(gpu, h, lim)
    for b, (o, _) in enumerate(h["segs"]):
        assert not ds[o + masked[b]].any()


@pytest.mark.gpu
@pytest.mark.parametrize("mask", MASKS)
def test_draws_go_on_into_the_mask(gpu, mask):
    """All open tokens drawn, then some of the masked ones: uniform among these."""
    rng = np.random.default_rng(3)
    images = []
    for n, opened, more in ((50, 20, 10), (50, 1, 49), (200, 100, 1), (300, 299, 1)):
        x = 2 * rng.standard_normal(n)
        x[opened:] = mask
        images.append((x, 1 + np.concatenate([rng.permutation(opened), opened + rng.permutation(n - opened)[:more]]), 10.0))
    h, lim = image_set(images, seed=4)
    compare(gpu, h, lim)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [0.0, 3.25, -1e6, 1e6, 1.5e15, -1e18, 1e19, -1e30, 3e38, -LOWEST, LOWEST])
def test_all_alike(gpu, value):
    rng = np.random.default_rng(5)
    images = [(np.full(n, value), 1 + rng.permutation(n)[:k], 0.0)
              for n, k in ((1, 1), (2, 1), (30, 30), (64, 13), (65, 1), (500, 499), (2000, 700))]
    h, lim = image_set(images, seed=6)
    compare(gpu, h, lim)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [1e5, 8e6, -8e6])
def test_a_shift_counts_for_nothing(gpu, value):
    """Scores a few apart, all far from 0 (whole numbers, exact in fp32)."""
    rng = np.random.default_rng(7)
    images = []
    for n, k in ((40, 20), (300, 299), (1500, 800)):
        x = value + rng.integers(-6, 7, n)
        images.append((x, 1 + np.argsort(-(x + rng.gumbel(size=n)))[:k], 12.0))
    h, lim = image_set(images, seed=8)
    compare(gpu, h, lim)
