"""The gradients' reference with either form of delta, against automatic
differentiation in 64 bits on the CPU."""
import itertools

import pytest
import torch

import attn_grad_ref as tight


@pytest.mark.parametrize("causal,few", itertools.product((False, True), (False, True)))
def test_gradients(causal, few):
    g = torch.Generator().manual_seed(1)
    cu_q, cu_k, H, Hk, D = [0, 1, 6, 9], [0, 1, 6, 13], 4, 2, 32
    q, k, v, dout = (torch.randn((n, h, D), generator=g, dtype=torch.float64).requires_grad_(i < 3)
                     for i, (n, h) in enumerate(((9, H), (13, Hk), (13, Hk), (9, H))))
    outs, lses = [], []
    for b in range(3):
        qb, kb, vb = (t[c[b]:c[b + 1]].transpose(0, 1) for t, c in ((q, cu_q), (k, cu_k), (v, cu_k)))
        kb, vb = kb.repeat_interleave(H // Hk, 0), vb.repeat_interleave(H // Hk, 0)
        s = qb @ kb.transpose(1, 2) * float(torch.tensor(D ** -0.5))
        if causal:
            n, m = s.shape[1:]
            s = s.masked_fill(torch.arange(m)[None] > torch.arange(n)[:, None] + m - n, -float("inf"))
        outs.append((torch.softmax(s, -1) @ vb).transpose(0, 1))
        lses.append(torch.logsumexp(s, -1).transpose(0, 1))
    out, lse = torch.cat(outs), torch.cat(lses)
    want = torch.autograd.grad(out, (q, k, v), dout)
    got, bound = tight.gradients(q.detach(), k.detach(), v.detach(), dout, out.detach(), lse.detach(), cu_q, cu_k, causal, few)
    for x, n in zip(want, ("dq", "dk", "dv")):
        assert torch.allclose(got[n], x, atol=1e-12), n
        assert bool((bound[n] >= 0).all())
    one = [0, 1] if causal else [0]          # the first sequence's row, and the second's first
    assert bool((got["dq"][one] == 0).all()) and bool((bound["dq"][one] == 0).all())
    assert bool((got["dk"][0] == 0).all()) and bool((bound["dk"][0] == 0).all())
