"""Equal removal scores among scores thousands apart, where the ordered-draw
loss keeps (value, exponent) pairs: joins at equal exponents, with the draws
ending before, inside and behind a block of equal scores.

Drawn from the highest score down, each draw's log-probability is minus the log
of the equal scores left, so log p stays small beside the scores and the ratio's
side of the clip is certain.  The kernel's terms are differences of 64-bit
numbers as large as the scores, each off by a few 2^-53 of them: over n terms
8 n |s| 2^-53, for log p (stored in fp32) and, times the slope, for a gradient
(twice: its slope and its own difference)."""
import numpy as np
import pytest

import policy_ref as P
from test_gpu_pl_policy import run

KL = 0.05


def case(spread, seed, n=200, low=0.2, high=0.28):
    rng = np.random.default_rng([seed, int(spread)])
    ends = [n - 1, 150, 120, 100, 3, 0]        # the block is at draws 80 .. 119: behind it, inside, before it
    s, order = [], []
    for k in ends:
        x = np.sort((spread * rng.standard_normal(n - 1)).astype(np.float32))[::-1].copy()
        x[80:120] = x[80]
        x[5:7] = x[5]                          # a pair as well
        at = rng.permutation(n - 1)            # where the scores stand
        one = np.empty(n, np.float32)
        one[0] = 9e9                           # CLS: not looked at
        one[1 + at] = x
        s.append(one)
        order.append(1 + at[:k])
    B = len(ends)
    cuo = np.concatenate([[0], np.cumsum(ends)]).astype(np.int32)
    h = dict(s=np.concatenate(s), order=np.concatenate(order).astype(np.int32), cuo=cuo, cu=None, N=n,
             segs=[(b * n, n) for b in range(B)], low=low, high=high, weight=None)
    z = np.zeros(B)
    lp = P.pl(h["s"].astype(np.float64), h["order"], cuo, z, z, segments=h["segs"])[1]
    h["old"] = P.off_border(lp, 0.3 * rng.standard_normal(B), low, high)
    h["A"] = rng.standard_normal(B).astype(np.float32)
    h["ref"] = (lp + 0.3 * rng.standard_normal(B)).astype(np.float32)
    return h, lp


def limit(h):
    visual = np.array([np.abs(h["s"][o + 1:o + n]).max() for o, n in h["segs"]])
    return 8 * h["N"] * visual * 2.0 ** -53


SPREADS = [300.0, 3000.0, 1e6]


@pytest.mark.parametrize("spread", SPREADS)
def test_the_case_is_certain(spread):
    """On the host: pairs are needed, the ties' share of log p is what the
    formula says, and the ratio stays off the clip's borders."""
    h, lp = case(spread, 1)
    want = -np.array([np.log(np.arange(1, 41)).sum() + np.log(2)] * 3 + [np.log(np.arange(21, 41)).sum() + np.log(2), 0, 0])
    assert np.all(lp <= want + 1e-9)           # other neighbours' shares come on top
    assert np.all(np.abs(lp) * P.U32 < 1e-4)   # what storing the old one in fp32 moves it by
    r = np.exp(lp - h["old"].astype(np.float64))
    for b, (o, n) in enumerate(h["segs"]):
        s = h["s"][o + 1:o + n].astype(np.float64)
        assert (s.max() - s.min()) / np.log(2) > 900
        assert min(abs(np.log(r[b]) - np.log(0.8)), abs(np.log(r[b]) - np.log(1.28))) > 10 * limit(h)[b]


@pytest.mark.gpu
@pytest.mark.parametrize("seed", [1, 2, 3])
@pytest.mark.parametrize("spread", SPREADS)
def test_equal_scores_among_distant_ones(gpu, spread, seed):
    h, _ = case(spread, seed)
    f = lambda v: float(np.float32(v))
    g, lp, stats, scale = P.pl(h["s"].astype(np.float64), h["order"], h["cuo"], h["old"].astype(np.float64),
                               h["A"].astype(np.float64), h["ref"].astype(np.float64), None, h["segs"], f(h["low"]),
                               f(h["high"]), f(KL))
    ds, glp, st, flag = run(gpu, h, KL)
    assert int(flag.item()) == 0
    u, lim = P.U32, limit(h)
    assert np.all(np.abs(glp.cpu().numpy() - lp) <= u * np.abs(lp) + lim)
    ds = ds.cpu().numpy().astype(np.float64)
    for b, (o, n) in enumerate(h["segs"]):
        pull = abs(float(h["A"][b])) * np.exp(lp[b] - float(h["old"][b])) + KL * (1 + np.exp(float(h["ref"][b]) - lp[b]))
        w = g[o:o + n]
        assert np.all(np.abs(ds[b] - w) <= u * np.abs(w) + 2 * pull * lim[b] + 1e-38), (b, np.abs(ds[b] - w).max())
    assert np.all(np.abs(st.cpu().numpy() - stats) <= u * np.abs(stats) + 2 * lim.max() * scale + 1e-30)
