"""The transformer block's operators in plain 64-bit torch on the CPU, with a bound
for what each kernel's roundings can add up to, element by element.

Roundings: U = 2^-24 of an fp32 operation; HALF[dtype] of a result's type (bf16
2^-8, fp32 2^-24), the most that rounding to nearest changes a value by."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float64: 2.0 ** -53}
TINY = 1e-37  # below it fp32 has no more bits to lose


def rounding(x, dtype):
    return HALF[dtype] * x.abs() + TINY


# ---------------------------------------------------------------- rotary positions

def rope(x, positions, freq, interleaved, inverse, scale):
    """(turned, bound) of x [rows, heads, D]."""
    half = freq.numel()
    pos = positions.view(x.shape[0], -1).double()
    t = pos.repeat_interleave(half // pos.shape[1], 1) * freq * (-1.0 if inverse else 1.0)
    c, s = torch.cos(t)[:, None] * scale, torch.sin(t)[:, None] * scale
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out, bound = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    u, v = x.double()[..., a], x.double()[..., b]
    out[..., a], out[..., b] = u * c - v * s, u * s + v * c
    # The fraction of a turn to fp32: pi 2^-25 radians.  The sine and cosine two units, times scale one rounding;
    # then a product and a multiply-add.
    # Turns are formed from t by a product with 1 / 2 pi in 64 bits: two roundings of t's size.
    far = 2.0 ** -51 * t.abs()[:, None]
    turn = (math.pi * 2.0 ** -25 + far + 2 * 2.0 ** -24 + U + 2 * U) * abs(scale) * (u.abs() + v.abs())
    bound[..., a] = bound[..., b] = turn
    touched = torch.zeros(x.shape[-1], dtype=torch.bool)
    touched[a] = touched[b] = True
    return out, torch.where(touched, bound + rounding(out, x.dtype), torch.zeros_like(bound))


# ---------------------------------------------------------------- attention

def attention(q, k, v, cu_q, cu_k, causal, scale=None, dout=None, out=None, lse=None):
    """Forward: dict(out, lse) and their bounds.  With dout, and out and lse as
    given to the backward call: dq, dk, dv and their bounds."""
    H, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    G, dtype = H // Hk, q.dtype
    c = float(torch.tensor(1 / math.sqrt(D) if not scale else scale, dtype=torch.float32))
    # P and dS stand in the inputs' type in their products.
    held = 0.0 if dtype == torch.float32 else HALF[dtype]
    Q, K, V = q.double(), k.double(), v.double()
    names = ("out", "lse") if dout is None else ("dq", "dk", "dv")
    like = {"out": Q, "lse": Q[..., 0], "dq": Q, "dk": K, "dv": V}
    r = {n: torch.zeros_like(like[n]) for n in names}
    e = {n: torch.zeros_like(like[n]) for n in names}
    for b in range(len(cu_q) - 1):
        rq, rk = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        seen = torch.ones((nq, nk), dtype=torch.bool)
        if causal:
            seen = seen.tril(nk - nq)
        for h in range(H):
            qh, kh, vh = Q[rq, h], K[rk, h // G], V[rk, h // G]
            S = c * qh @ kh.T
            # D products and sums (c and log2 e on top), then the exponential's argument: two roundings of its size.
            dS = (D + 4) * U * c * (qh.abs() @ kh.abs().T)
            if dout is None:
                S, dS = S.masked_fill(~seen, -math.inf), dS.masked_fill(~seen, 0.0)
                L = torch.logsumexp(S, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
                empty = L == -math.inf
                L0 = torch.where(empty, torch.zeros_like(L), L)
                P = torch.exp(S - L0[:, None])
                top = S.abs().masked_fill(~seen, 0.0).amax(1, keepdim=True) if nk else torch.zeros(nq, 1)
                one = dS + 4 * U * (1 + top)              # of a term, relative
                far = one.amax(1, keepdim=True) if nk else torch.zeros(nq, 1)
                terms = (nk + 24) * U                     # sums over the keys, rescaled as the maximum rises
                r["out"][rq, h] = P @ vh
                spread = (P * (one + far + 2 * terms + held)) @ vh.abs()
                e["out"][rq, h] = spread + rounding(r["out"][rq, h], dtype) * (1 + 8 * U)
                r["lse"][rq, h] = L
                e["lse"][rq, h] = far[:, 0] + terms + 4 * U * (1 + L0.abs() + top[:, 0])
                continue
            g, o, L = dout.double()[rq, h], out.double()[rq, h], lse.double()[rq, h]
            L = torch.where(L == -math.inf, torch.full_like(L, math.inf), L)
            P = torch.exp(S - L[:, None]).masked_fill(~seen, 0.0)
            Lf = torch.where(torch.isinf(L), torch.zeros_like(L), L)
            one = dS + 4 * U * (1 + S.abs() + Lf.abs()[:, None])
            dP, delta = g @ vh.T, (g * o).sum(1, keepdim=True)
            T = P * (dP - delta)
            eT = T.abs() * (one + 2 * U) + P * (D + 4) * U * (g.abs() @ vh.abs().T + (g * o).abs().sum(1, keepdim=True))
            if dtype == torch.bfloat16:
                # Rows of few keys have delta as the sum of P dP, of which g . out differs by out's rounding, half a step of
                # each element; P's own errors and those of the products (as above, P adds up to 1) come on top.
                eT = eT + P * ((g * o).abs().sum(1, keepdim=True) * HALF[dtype] + (P * one * dP.abs()).sum(1, keepdim=True) +
                               (P * (D + 4 + nk) * U * (g.abs() @ vh.abs().T)).sum(1, keepdim=True))
            eT = eT * (1 + held) + T.abs() * held
            r["dq"][rq, h] = c * T @ kh
            e["dq"][rq, h] = c * (eT + T.abs() * (nk + 24) * U) @ kh.abs()
            r["dk"][rk, h // G] += c * T.T @ qh
            e["dk"][rk, h // G] += c * (eT + T.abs() * (nq * G + 24) * U).T @ qh.abs()
            r["dv"][rk, h // G] += P.T @ g
            e["dv"][rk, h // G] += (P * (one * (1 + held) + held + (nq * G + 24) * U)).T @ g.abs()
    if dout is not None:
        for n in names:
            e[n] += rounding(r[n], dtype) + 2 * U * r[n].abs()
    return r, e


# ---------------------------------------------------------------- norms

# Roundings of one sum over a row: up to 16 terms in a lane, 6 exchanges in a wave, 8 waves, and the mean's product.
ROW = 32 * U


def _hat(z, ez, kind, eps):
    """The normed row, its bound, and 1 / deviation; ez the bound of z."""
    size = z.abs().mean(1, keepdim=True)
    mean = z.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(size)
    emean = (ROW * size + ez.mean(1, keepdim=True)) if kind == "layer" else torch.zeros_like(size)
    d = z - mean
    ed = ez + emean + U * (z.abs() + mean.abs())
    var = (d * d).mean(1, keepdim=True)
    evar = (2 * d.abs() * ed).mean(1, keepdim=True) + (ed * ed).mean(1, keepdim=True) + ROW * var
    r = 1 / torch.sqrt(var + eps)
    er = r * (0.5 * evar / (var + eps) + 6 * U)
    hat = d * r
    return hat, d.abs() * er + ed * (r + er) + U * hat.abs(), r, er


def _hat_grad(g, eg, hat, ehat, r, er, kind):
    m = g.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(r)
    em = eg.mean(1, keepdim=True) + ROW * g.abs().mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(r)
    c = (g * hat).mean(1, keepdim=True)
    ec = (g.abs() * ehat + eg * (hat.abs() + ehat)).mean(1, keepdim=True) + ROW * (g * hat).abs().mean(1, keepdim=True)
    x = g - m - hat * c
    ex = eg + em + hat.abs() * ec + ehat * (c.abs() + ec) + 3 * U * (g.abs() + m.abs() + (hat * c).abs())
    return r * x, (r + er) * ex + er * x.abs() + U * (r * x).abs()


def _params(p, T, C):
    one, zero = torch.ones(1, C, dtype=torch.float64), torch.zeros(1, C, dtype=torch.float64)

    def get(n, default):
        return default if p.get(n) is None else p[n].double().view(1, C)
    gate = torch.ones(T, 1, dtype=torch.float64) if p.get("gate") is None else p["gate"].double().view(T, 1)
    return (get("gamma", one), get("beta", zero), get("scale", one), gate, get("post_gamma", one), get("post_beta", zero))


def _branch(a, p, kind, eps):
    """u, its bound, and the norm's parts."""
    T, C = a.shape
    _, _, _, _, pg, pb = _params(p, T, C)
    A, zero = a.double(), torch.zeros(a.shape, dtype=torch.float64)
    if p.get("post_gamma") is None:
        return A, zero, None
    hat, ehat, r, er = _hat(A, zero, kind, eps)
    u = hat * pg + pb
    return u, ehat * pg.abs() + U * u.abs(), (hat, ehat, r, er)


def residual_norm(x, a, p, kind="layer", eps=1e-6):
    """dict(h, y) and their bounds."""
    T, C = x.shape
    gamma, beta, scale, gate, _, _ = _params(p, T, C)
    h, eh = x.double(), torch.zeros(x.shape, dtype=torch.float64)
    if a is not None:
        u, eu, _ = _branch(a, p, kind, eps)
        add = torch.where(gate == 0, torch.zeros_like(u), gate * scale * u)
        eadd = torch.where(gate == 0, torch.zeros_like(u), (gate * scale).abs() * eu + U * add.abs())
        h = h + add
        eh = eadd + U * h.abs()
    hat, ehat, _, _ = _hat(h, eh, kind, eps)
    y = hat * gamma + beta
    return ({"h": h, "y": y},
            {"h": eh + rounding(h, x.dtype), "y": ehat * gamma.abs() + U * y.abs() + rounding(y, x.dtype)})


def residual_norm_backward(dy, dh, h, a, p, kind="layer", eps=1e-6):
    """Every gradient and its bound, by the formulas."""
    T, C = h.shape
    gamma, beta, scale, gate, pg, pb = _params(p, T, C)
    zero = torch.zeros(h.shape, dtype=torch.float64)
    r, e = {}, {}
    rows = (T + 24) * U  # sums over the rows

    def column(n, x, ex):
        r[n], e[n] = x.sum(0), (ex + (rows + U) * x.abs()).sum(0) + HALF[torch.float32] * x.sum(0).abs() + TINY
    g, eg = zero, zero
    if dy is not None:
        hat, ehat, rr, er = _hat(h.double(), zero, kind, eps)
        column("dgamma", dy.double() * hat, dy.double().abs() * ehat)
        column("dbeta", dy.double().expand(T, C), zero)
        w = dy.double() * gamma
        g, eg = _hat_grad(w, U * w.abs(), hat, ehat, rr, er, kind)
    else:
        column("dgamma", zero, zero)
        column("dbeta", zero, zero)
    if dh is not None:
        g = g + dh.double()
        eg = eg + U * g.abs()
    r["dx"], e["dx"] = g, eg + rounding(g, h.dtype)
    if a is None:
        return r, e
    u, eu, post = _branch(a, p, kind, eps)
    su = u * scale
    r["dgate"] = (g * su).sum(1)
    e["dgate"] = (eg * su.abs() + (g.abs() + eg) * scale.abs() * eu + 3 * U * (g * su).abs()).sum(1) + \
        ROW * (g * su).abs().sum(1) + TINY
    on = gate != 0
    gated = torch.where(on, g * gate, zero)
    egated = torch.where(on, eg * gate.abs() + U * gated.abs(), zero)
    column("dscale", torch.where(on, gated * u, zero), torch.where(on, egated * u.abs() + (gated.abs() + egated) * eu, zero))
    d = gated * scale
    ed = egated * scale.abs() + U * d.abs()
    if post is not None:
        hat, ehat, rr, er = post
        column("dpost_gamma", torch.where(on, d * hat, zero),
               torch.where(on, ed * hat.abs() + (d.abs() + ed) * ehat, zero))
        column("dpost_beta", d, ed)
        w = d * pg
        d, ed = _hat_grad(w, ed * pg.abs() + U * w.abs(), hat, ehat, rr, er, kind)
        d, ed = torch.where(on, d, zero), torch.where(on, ed, zero)
    r["da"], e["da"] = d, ed + rounding(d, h.dtype)
    return r, e


def check(got, want, bound, what=""):
    """Every element within its bound."""
    got, want = got.detach().double().cpu(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    bad = ~(off <= bound)
    if bad.any():
        i = int(torch.where(bad, off / (bound + 1e-300), torch.zeros_like(off)).nan_to_num(1e9).argmax())
        at = tuple(int(x) for x in torch.unravel_index(torch.tensor(i), want.shape))
        raise AssertionError(f"{what}: {int(bad.sum())} of {want.numel()} past their bound, at {at} got "
                             f"{float(got[at])} for {float(want[at])}, bound {float(bound[at]):.3g}")
