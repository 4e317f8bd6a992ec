"""GPU parity of dora_policy_loss on batches whose rows keep a workgroup of
their own (more than 128 rows), through every width of it, with the formulas
in 64-bit torch operations; tolerances as derived in test_gpu_policy.py."""
import numpy as np
import pytest
import torch

from policy_ref import HALF, U32

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LOW, HIGH, KL = 0.2, 0.28, 0.05


def f32(v):
    return float(np.float32(v))


def case(T, V, dtype, seed, pad=0, legal=False, masked=False):
    g = torch.Generator("cuda").manual_seed(seed)
    full = (3 * torch.randn((T, V + pad), generator=g, device="cuda")).to(DT[dtype])
    c = dict(logits=full[:, :V], legal=None, weight=None)
    if legal:
        c["legal"] = torch.randint(1, V + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
        c["legal"][:3] = torch.tensor([1, V, max(V - 1, 1)], dtype=torch.int32)
        c["logits"][torch.arange(V, device="cuda")[None, :] >= c["legal"][:, None]] = float("nan")
    n = c["legal"] if legal else torch.full((T,), V, device="cuda")
    c["actions"] = (torch.rand(T, generator=g, device="cuda") * n).int().minimum(n.int() - 1)
    if masked:
        w = torch.rand(T, generator=g, device="cuda") + 0.1
        w[torch.rand(T, generator=g, device="cuda") < 0.3] = 0.0
        c["weight"] = w
    lp = softmax(c)[0]
    lr = 0.3 * torch.randn(T, generator=g, device="cuda", dtype=torch.float64)
    for border in (np.log1p(-LOW), np.log1p(HIGH)):
        d = lr - border
        lr = torch.where(d.abs() < 1e-3, border + torch.where(d < 0, -2e-3, 2e-3), lr)
    c["old"] = (lp - lr).float()
    c["A"] = torch.randn(T, generator=g, device="cuda")
    c["ref"] = (lp + 0.3 * torch.randn(T, generator=g, device="cuda")).float()
    return c


def softmax(c):
    x = c["logits"].double()
    if c["legal"] is not None:
        x = x.masked_fill(torch.arange(x.shape[1], device="cuda")[None, :] >= c["legal"][:, None], -np.inf)
    lsm = torch.log_softmax(x, 1)
    return lsm.gather(1, c["actions"].long()[:, None])[:, 0], lsm, x


def run(dora, c, ent, **kw):
    return dora.dora_policy_loss(c["logits"], c["actions"], c["old"], c["A"], ref_logprob=c["ref"], weight=c["weight"],
                                 legal=c["legal"], clip_low=LOW, clip_high=HIGH, kl_coef=KL, entropy_coef=ent, **kw)


def check(dora, c, dtype, ent, **kw):
    T, V = c["logits"].shape
    u, err_lp = U32, (V / 16 + 68) * U32
    lp, lsm, x = softmax(c)
    on = torch.ones(T, dtype=torch.bool, device="cuda") if c["weight"] is None else c["weight"] != 0
    w = on.double() if c["weight"] is None else c["weight"].double()
    p = lsm.exp()
    H = -torch.where(p > 0, p * lsm, 0.0).sum(1)
    A, r = c["A"].double(), torch.exp(lp - c["old"].double())
    held = r.clamp(1 - f32(LOW), 1 + f32(HIGH)) * A
    clipped = held < r * A
    d = c["ref"].double() - lp
    G = w * (torch.where(clipped, 0.0, -r * A) - f32(KL) * torch.expm1(d))
    lpc = torch.where(p > 0, lsm, 0.0)
    g = -G[:, None] * p + (f32(ent) * w)[:, None] * p * (lpc + H[:, None])
    g.scatter_add_(1, c["actions"].long()[:, None], G[:, None])
    g[~on] = 0.0
    want_lp = torch.where(on, lp, 0.0)
    ref_terms = torch.stack([w * (f32(KL) * (torch.expm1(d) - d) - torch.minimum(r * A, held) - f32(ent) * H),
                             w * torch.minimum(r * A, held), w * (torch.expm1(d) - d), w * H, w * clipped, w])
    dl, glp, st, flag = run(dora, c, ent, **kw)
    torch.cuda.synchronize()
    assert int(flag.item()) == 0
    assert bool(((glp - want_lp).abs() <= err_lp + u * want_lp.abs()).all())
    pull = (r * A).abs() + KL * (1 + 2 * torch.exp(d))
    dist = torch.where(p > 0, (x - x.amax(1, keepdim=True)).abs(), 0.0)
    share = err_lp + u * (4 + dist)
    tol = w[:, None] * p * (pull[:, None] * (share + err_lp) + ent * (lpc.abs() + H[:, None]) * (share + 4 * u) +
                            ent * (err_lp * (3 + H[:, None]) + 2 * u * (dist + H[:, None])))
    tol.scatter_add_(1, c["actions"].long()[:, None], (w * pull * (err_lp + 4 * u))[:, None])
    tol += HALF[dtype] * g.abs() + 1e-38
    e = (dl.double() - g).abs()
    assert bool((e <= tol).all()), float((e - tol).max())
    err_H = err_lp * (2 + np.log(V + 1)) + u * np.log(V + 1)
    dkl = torch.exp(d) + 1
    lim = torch.stack([w * (err_lp * (pull + KL * dkl) + ent * err_H), w * err_lp * pull, w * err_lp * dkl, w * err_H,
                       0 * w, 0 * w]).sum(1) + u * ref_terms.sum(1).abs() * (1 + 1e-9) + 1e-30
    e = (st.double() - ref_terms.sum(1)).abs()
    assert bool((e <= lim).all()), (e, lim)
    return dl


# Threads a row and pieces a thread, through their borders: 16, 64, 256, 512 and 1024 threads, then shared memory, then re-read.
SIZES = [1024, 2048, 2049, 4096, 4097, 8191, 12288, 16385, 20001, 24577, 30001, 32768, 32769, 40961, 45001, 50257, 57345,
         65536, 65537, 81920, 90001, 114689, 131072, 131073, 163841, 196608, 200001, 300001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_widths(gpu, V, dtype):
    check(gpu, case(130, V, dtype, seed=V), dtype, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [513, 3001, 9001, 20003, 50257, 70001, 131075, 200003])
def test_legal_masks_strides_entropy(gpu, V, dtype):
    """Prefixes from one choice to all, NaN behind them, padding rows, rows any
    distance apart, the gradient at another alignment than the logits."""
    c = case(133, V, dtype, seed=V + 1, pad=5, legal=True, masked=True)
    room = torch.full((133, V + 9), 7.0, dtype=DT[dtype], device="cuda")
    check(gpu, c, dtype, 0.02, dlogits=room[:, 3:V + 3])
    assert bool((room[:, :3] == 7).all()) and bool((room[:, V + 3:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [97, 600, 5001, 33001, 70001, 140001, 300001])
def test_in_place_and_gaps(gpu, V, dtype):
    """In the gaps between the logits' rows (whose bits stay; the gradient's
    sums are grouped by its own 16-byte boundaries, so its last bits go by where
    it lies), and over the logits, to the last bit what it is in a place like
    theirs."""
    c = case(140, V, dtype, seed=V + 2, masked=True)
    both = torch.empty((140, 2 * V), dtype=DT[dtype], device="cuda")
    both[:, :V] = c["logits"]
    check(gpu, {**c, "logits": both[:, :V]}, dtype, 0.01, dlogits=both[:, V:])
    assert torch.equal(both[:, :V], c["logits"])
    want = run(gpu, c, 0.01)
    got = run(gpu, c, 0.01, dlogits=c["logits"])
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("V", [1, 2, 3])
def test_few_choices_far_apart(gpu, V):
    check(gpu, case(200, V, "bf16", seed=3, pad=6, legal=True), "bf16", 0.01)


def test_most_rows(gpu):
    """As many rows as a call takes."""
    T = gpu.DORA_MAX_DECISIONS
    g = torch.Generator("cuda").manual_seed(5)
    logits = torch.randn((T, 2), generator=g, device="cuda")
    actions = torch.randint(0, 2, (T,), generator=g, device="cuda", dtype=torch.int32)
    d = torch.where(actions == 0, logits[:, 1].double() - logits[:, 0].double(), logits[:, 0].double() - logits[:, 1].double())
    lp = -torch.log1p(torch.exp(d))
    A = torch.randn(T, generator=g, device="cuda")
    dl, got, st, flag = gpu.dora_policy_loss(logits, actions, lp.float(), A)
    assert int(flag.item()) == 0
    assert bool(((got - lp).abs() <= 70 * U32 + U32 * lp.abs()).all())
    slope = -A.double() * (1 - torch.exp(lp))               # at the action; the other has minus it
    at = dl.gather(1, actions.long()[:, None])[:, 0]
    assert bool(((at - slope).abs() <= 200 * U32 * A.abs()).all())
    assert bool(((dl.sum(1)).abs() <= 200 * U32 * A.abs()).all())
    assert float(st[5]) == T and abs(float(st[1]) - float(A.double().sum())) <= 100 * U32 * float(A.double().abs().sum())


@pytest.mark.parametrize("T,V", [(300, 70001), (257, 33000), (256, 40001), (5000, 9001)])
def test_logprob(gpu, T, V):
    c = case(T, V, "bf16", seed=V + 4, pad=1, legal=True, masked=True)
    lp, lsm, _ = softmax(c)
    H = -torch.where(lsm.exp() > 0, lsm.exp() * lsm, 0.0).sum(1)
    on = c["weight"] != 0
    got, gH, flag = gpu.dora_action_logprob(c["logits"], c["actions"], weight=c["weight"], legal=c["legal"])
    err = (V / 16 + 68) * U32
    assert int(flag.item()) == 0
    assert bool(((got - torch.where(on, lp, 0.0)).abs() <= err + U32 * lp.abs()).all())
    assert bool(((gH - torch.where(on, H, 0.0)).abs() <= err * (2 + H) + U32 * H).all())
