"""The gate's Bernoulli choice through the operators on logits: one logit x an
image is the row (0, x), action 1 keeps the gate on; d loss / d x is the second
column.  Against automatic differentiation of the sigmoid's form in 64 bits.

Two terms' sum and the exponents' roundings put log p off by at most 70 u
(u = 2^-24), the slope by as much of itself; the entropy's two terms likewise."""
import numpy as np
import pytest
import torch

from policy_ref import U32

pytestmark = pytest.mark.gpu

LOW, HIGH, KL, ENT = 0.2, 0.28, 0.05, 0.01


@pytest.mark.parametrize("B", [1, 48, 1000])
def test_gate(gpu, B):
    g = torch.Generator("cuda").manual_seed(B)
    x = 3 * torch.randn(B, generator=g, device="cuda")
    x[:1] = -40.0                                       # a gate that is all but shut
    on = (torch.rand(B, generator=g, device="cuda") < torch.sigmoid(x)).int()
    on[:1] = 0
    f = lambda v: float(np.float32(v))
    z = x.double().requires_grad_()
    lp = torch.nn.functional.logsigmoid(torch.where(on == 1, z, -z))
    p = torch.sigmoid(z)
    H = -(p * torch.nn.functional.logsigmoid(z) + (1 - p) * torch.nn.functional.logsigmoid(-z))
    shift = 0.1 * torch.randn(B, generator=g, device="cuda", dtype=torch.float64)
    shift = torch.where((shift - np.log1p(HIGH)).abs() < 2e-3, 0.0, shift)
    shift = torch.where((shift - np.log1p(-LOW)).abs() < 2e-3, 0.0, shift)
    old, ref = (lp.detach() - shift).float(), (lp.detach() + 0.1).float()
    adv = torch.randn(B, generator=g, device="cuda")
    w = torch.full((B,), 1.0 / B, device="cuda")
    r = torch.exp(lp - old.double())
    gain = torch.minimum(r * adv.double(), r.clamp(1 - f(LOW), 1 + f(HIGH)) * adv.double())
    d = ref.double() - lp
    loss = (w.double() * (f(KL) * (torch.exp(d) - d - 1) - gain - f(ENT) * H)).sum()
    want, = torch.autograd.grad(loss, z)

    rows = torch.zeros((B, 2), device="cuda")
    rows[:, 1] = x
    got_lp, got_H, st = gpu.dora_action_logprob(rows, on)
    assert int(st.item()) == 0
    assert bool(((got_lp - lp).abs() <= 70 * U32 + U32 * lp.abs()).all())
    assert bool(((got_H - H).abs() <= 70 * U32 * (2 + H)).all())
    dl, _, stats, st = gpu.dora_policy_loss(rows, on, old, adv, ref_logprob=ref, weight=w, clip_low=LOW, clip_high=HIGH,
                                            kl_coef=KL, entropy_coef=ENT)
    assert int(st.item()) == 0
    pull = w * (r.detach().abs() * adv.abs() + KL * (1 + torch.exp(d.detach())) + ENT * (3 + x.abs()))
    tol = 200 * U32 * pull
    assert bool(((dl[:, 1] - want).abs() <= tol).all()) and bool(((dl[:, 0] + want).abs() <= tol).all())
    assert abs(float(stats[0]) - loss.item()) <= float(tol.sum()) + U32 * abs(loss.item())
