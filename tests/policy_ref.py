"""The policy operators in plain 64-bit numpy, for the tests: each formula row
by row, without the package."""
import numpy as np

U32 = 2.0 ** -24     # half a step of fp32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def decision(logp, H, old, ref, A, w, low, high, kl_coef, ent):
    """Six terms and d loss / d logp of one decision."""
    with np.errstate(over="ignore", invalid="ignore"):
        r = np.exp(logp - old)
        held, free = np.clip(r, 1 - low, 1 + high) * A, r * A
        clipped = held < free
        gain = held if clipped else free
        slope = 0.0 if clipped else -free
        kl = 0.0
        if ref is not None:
            kl = np.expm1(ref - logp) - (ref - logp)
            if kl_coef:
                slope -= kl_coef * np.expm1(ref - logp)
        loss = (kl_coef * kl if kl_coef else 0.0) - gain - (ent * H if ent else 0.0)
    return np.array([w * loss, w * gain, w * kl, w * H, w * clipped, w]), w * slope


def softmax_row(x, a):
    """log-probability of a, entropy, log-probabilities of a row of open logits."""
    with np.errstate(divide="ignore", invalid="ignore"):
        m = x.max()
        lp = x - m
        lp = lp - np.log(np.exp(lp).sum())
        p = np.exp(lp)
        H = -np.where(p == 0, 0.0, p * lp).sum()
    return lp[a], H, lp


def policy(x, actions, old, A, ref=None, weight=None, legal=None, low=0.2, high=0.2, kl_coef=0.0, ent=0.0):
    """x: float64 [T, V].  Returns dlogits, logp, entropy, stats, and |terms|
    summed as the stats are (the scale of their rounding)."""
    T, V = x.shape
    g, lps, Hs = np.zeros((T, V)), np.zeros(T), np.zeros(T)
    stats, scale = np.zeros(6), np.zeros(6)
    for t in range(T):
        w = 1.0 if weight is None else float(weight[t])
        if w == 0.0:
            continue
        n = V if legal is None else int(legal[t])
        a = int(actions[t])
        if not (1 <= n <= V and 0 <= a < n) or np.all(x[t, :n] == -np.inf):
            lps[t] = Hs[t] = np.nan
            continue
        lps[t], Hs[t], lp = softmax_row(x[t, :n], a)
        terms, slope = decision(lps[t], Hs[t], float(old[t]), None if ref is None else float(ref[t]), float(A[t]), w,
                                low, high, kl_coef, ent)
        stats += terms
        scale += np.abs(terms)
        scale[0] += abs(terms[1]) + abs(kl_coef * terms[2]) + abs(ent * terms[3])
        p = np.exp(lp)
        with np.errstate(invalid="ignore"):
            g[t, :n] = -slope * p + (ent * w * np.where(p == 0, 0.0, p * (lp + Hs[t])) if ent else 0.0)
        g[t, a] += slope
    return g, lps, Hs, stats, scale


def pl(scores, order, cu_order, old, A, ref=None, weight=None, segments=None, low=0.2, high=0.2, kl_coef=0.0):
    """scores: float64 flat; segments: (offset, length) per image.  Returns
    dscores (flat), logp, stats, scale.  Sums from scratch at every step."""
    B = len(segments)
    g, lps, stats, scale = np.zeros_like(scores), np.zeros(B), np.zeros(6), np.zeros(6)
    for b, (off, n) in enumerate(segments):
        w = 1.0 if weight is None else float(weight[b])
        if w == 0.0:
            continue
        s = scores[off + 1:off + n]
        draws = np.asarray(order[cu_order[b]:cu_order[b + 1]], dtype=np.int64) - 1
        left = np.ones(n - 1, bool)
        d = np.zeros(n - 1)
        lp = 0.0
        for i in draws:
            m = s[left].max()
            e = np.where(left, np.exp(np.minimum(s - m, 0.0)), 0.0)
            S = e.sum()
            lp += s[i] - m - np.log(S)
            d -= e / S
            d[i] += 1.0
            left[i] = False
        lps[b] = lp
        terms, slope = decision(lp, 0.0, float(old[b]), None if ref is None else float(ref[b]), float(A[b]), w, low,
                                high, kl_coef, 0.0)
        stats += terms
        scale += np.abs(terms)
        scale[0] += abs(terms[1]) + abs(kl_coef * terms[2])
        g[off + 1:off + n] = slope * d
    return g, lps, stats, scale


def clip(grads, max_norm, eps=1e-6):
    norm = np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads))
    c = 1.0 if norm == 0 else min(1.0, max_norm / (norm + eps))
    return [g.astype(np.float64) * c for g in grads], norm


def off_border(logp, log_ratio, low, high, gap=1e-3):
    """Old log-probabilities (fp32) whose ratio to logp is `log_ratio`, moved
    off the clip's borders by more than any rounding here."""
    for border in (np.log1p(-low) if low < 1 else -np.inf, np.log1p(high)):
        near = np.abs(log_ratio - border) < gap
        log_ratio = np.where(near, border + np.where(log_ratio < border, -2 * gap, 2 * gap), log_ratio)
    return (logp - log_ratio).astype(np.float32)
