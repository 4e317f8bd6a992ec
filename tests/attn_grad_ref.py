"""Gradients of grouped attention in plain 64-bit torch, with a bound for the
kernels' roundings that follows the form of delta, row by row.

delta is the sum of P dP over the sum of P (`few`: rows of bf16 whose tile's keys
are staged at once), or dout . out with out as it was given.  A row that sees one
key has P 1 and dS 0 whatever its score."""
import math

import torch

from block_ref import HALF, U, rounding

LEAST = 2.0 ** -126  # fp32's least normal number: the kernels' exponentials, and products, below it are 0


def gradients(q, k, v, dout, out, lse, cu_q, cu_k, causal, few, scale=None):
    """dict(dq, dk, dv) and their bounds, from out and lse as the backward call has them."""
    H, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    G, dtype = H // Hk, q.dtype
    c = float(torch.tensor(1 / math.sqrt(D) if not scale else scale, dtype=torch.float32))
    held = 0.0 if dtype == torch.float32 else HALF[dtype]     # P and dS in their products
    Q, K, V = q.double(), k.double(), v.double()
    r = {"dq": torch.zeros_like(Q), "dk": torch.zeros_like(K), "dv": torch.zeros_like(V)}
    e = {n: torch.zeros_like(x) for n, x in r.items()}
    for b in range(len(cu_q) - 1):
        rq, rk = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        if nq == 0 or nk == 0:
            continue
        seen = torch.ones((nq, nk), dtype=torch.bool)
        if causal:
            seen = seen.tril(nk - nq)
        one_key = (seen.sum(1) == 1)[:, None]
        for h in range(H):
            qh, kh, vh = Q[rq, h], K[rk, h // G], V[rk, h // G]
            g, o, L = dout.double()[rq, h], out.double()[rq, h], lse.double()[rq, h]
            S = c * qh @ kh.T
            L = torch.where(L == -math.inf, torch.full_like(L, math.inf), L)
            P = torch.exp(S - L[:, None]).masked_fill(~seen, 0.0)
            Lf = torch.where(torch.isinf(L), torch.zeros_like(L), L)
            # P, relative: D products and sums (c and log2 e on top), two roundings of the score's and of lse's size
            one = (D + 4) * U * c * (qh.abs() @ kh.abs().T) + 4 * U * (1 + S.abs() + Lf.abs()[:, None])
            one = torch.where(seen, one, torch.zeros_like(one))
            dP, edP = g @ vh.T, (D + 4) * U * (g.abs() @ vh.abs().T)
            if few:
                # The kernel's P are P (1 + x), |x| <= one: their mean of dP is off by the sum of P x (dP - delta) over that of
                # P (1 + x); sums of nk terms in lanes and exchanges and a division on top.
                total = P.sum(1, keepdim=True)
                total = torch.where(total == 0, torch.ones_like(total), total)
                delta = (P * dP).sum(1, keepdim=True) / total
                top = one.amax(1, keepdim=True)
                assert bool((top < 0.2).all())
                edelta = (P * (one * (dP - delta).abs() + edP * (1 + one) + 2 * (nk + 16) * U * dP.abs())).sum(1, keepdim=True)
                edelta = edelta / (total * (1 - top)) + 4 * U * delta.abs()
            else:
                delta = (g * o).sum(1, keepdim=True)
                edelta = (D + 4) * U * (g * o).abs().sum(1, keepdim=True)
            T = (P * (dP - delta)).masked_fill(one_key, 0.0)
            eT = T.abs() * (one + 4 * U) + P * (1 + one) * (edP + edelta)
            # A P below LEAST is 0 there, off by up to LEAST times what it multiplies; dS below it too.  Under scores hundreds
            # apart that is all of a key's gradient: 2^-126 of dP and q, past the 1e-37 of a result's own end.
            eT = eT + torch.where(seen, LEAST * (1 + dP.abs() + delta.abs()), torch.zeros_like(dP))
            eT = (eT * (1 + held) + T.abs() * held).masked_fill(one_key, 0.0)
            r["dq"][rq, h] = c * T @ kh
            e["dq"][rq, h] = c * (eT + T.abs() * (nk + 24) * U) @ kh.abs()
            r["dk"][rk, h // G] += c * T.T @ qh
            e["dk"][rk, h // G] += c * (eT + T.abs() * (nq * G + 24) * U).T @ qh.abs()
            r["dv"][rk, h // G] += P.T @ g
            e["dv"][rk, h // G] += (P * (one * (1 + held) + held + (nq * G + 24) * U) + LEAST * seen).T @ g.abs()
    for n in r:
        none = (r[n] == 0) & (e[n] == 0)
        e[n] += torch.where(none, torch.zeros_like(r[n]), rounding(r[n], dtype) + 2 * U * r[n].abs())
    return r, e
