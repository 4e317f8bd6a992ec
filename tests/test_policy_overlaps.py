"""Outputs of the policy operators against the call's other tensors: refused
where they share memory, but that a row's (image's) log-probability may take the
place of one of its own inputs."""
import ctypes

import pytest
import torch

import paper_2609_34325_amd as dora

A = 0x10000000          # never dereferenced: every call on the host below is refused


class Room:
    """Addresses far apart, one for each name asked for."""

    def __init__(self, names):
        self.at = {n: A + (i << 24) for i, n in enumerate(names)}


T, V, LD = 6, 96, 100
VECTORS = ("act", "legal", "old", "ref", "A", "w")


def logprob(**kw):
    a = Room(("x", "act", "legal", "w", "lp", "H", "ws", "st")).at
    a.update(kw)
    return dora.load_library().dora_action_logprob(
        a["x"], LD, a["act"], a["legal"], a["w"], T, V, dora.DORA_F32, a["lp"], a["H"], a["ws"],
        dora.dora_policy_workspace_size(T, V), a["st"], None)


def loss(**kw):
    a = Room(("x",) + VECTORS + ("g", "lp", "stats", "ws", "st")).at
    a.update(kw)
    return dora.load_library().dora_policy_loss(
        a["x"], LD, a["act"], a["legal"], a["old"], a["ref"], a["A"], a["w"], T, V, dora.DORA_F32, 0.2, 0.2, 0.1, 0.0,
        a["g"], LD, a["lp"], a["stats"], a["ws"], dora.dora_policy_workspace_size(T, V), a["st"], None)


def test_logprob_outputs_apart():
    a = Room(("x", "act", "legal", "w", "lp", "H", "ws", "st")).at
    row = 4 * LD
    for out in ("lp", "H", "ws", "st"):
        for other in ("x", "act", "legal", "lp", "H", "ws", "st"):
            if out != other:
                assert logprob(**{out: a[other]}) == dora.DORA_ERR_OVERLAP, (out, other)
    for out in ("lp", "H"):
        assert logprob(**{out: a["w"] + 4}) == dora.DORA_ERR_OVERLAP                # shifted by a row
        assert logprob(**{out: a["w"] - 4}) == dora.DORA_ERR_OVERLAP
        assert logprob(**{out: a["x"] + 4 * V - 4}) == dora.DORA_ERR_OVERLAP        # a row's last element
        assert logprob(**{out: a["x"] + 5 * row + 4 * V - 4}) == dora.DORA_ERR_OVERLAP   # the last row's
        assert logprob(**{out: a["x"] - 20}) == dora.DORA_ERR_OVERLAP               # the first element
    assert logprob(st=a["x"] + 3 * row) == dora.DORA_ERR_OVERLAP
    assert logprob(lp=a["H"] + 20) == dora.DORA_ERR_OVERLAP                         # H's last entry


def test_loss_outputs_apart():
    a = Room(("x",) + VECTORS + ("g", "lp", "stats", "ws", "st")).at
    row = 4 * LD
    for out in ("lp", "stats", "ws", "st"):
        for other in ("x", "act", "legal", "g", "lp", "stats", "ws", "st"):
            if out != other:
                assert loss(**{out: a[other]}) == dora.DORA_ERR_OVERLAP, (out, other)
    for other in ("old", "ref", "A", "w"):
        assert loss(stats=a[other]) == dora.DORA_ERR_OVERLAP
        assert loss(ws=a[other]) == dora.DORA_ERR_OVERLAP
        assert loss(lp=a[other] + 4) == dora.DORA_ERR_OVERLAP                       # shifted by a row
        assert loss(lp=a[other] - 20) == dora.DORA_ERR_OVERLAP
    for vector in VECTORS:
        assert loss(g=a[vector]) == dora.DORA_ERR_OVERLAP
        assert loss(g=a[vector] + 20 - 2 * row) == dora.DORA_ERR_OVERLAP            # the third row over its last entry
    assert loss(lp=a["g"] + 4 * V - 4) == dora.DORA_ERR_OVERLAP                     # the first row's last element
    assert loss(lp=a["g"] + 4 * V - 4 + row) == dora.DORA_ERR_OVERLAP
    assert loss(stats=a["x"] - 20) == dora.DORA_ERR_OVERLAP


def draws(packed=True, cap=50, entry="dora_pl_policy_loss_cap", **kw):
    a = Room(("s", "order", "cuo", "cu", "old", "ref", "A", "w", "g", "lp", "stats", "ws", "st")).at
    a.update(kw)
    B, N = 7, 40
    return getattr(dora.load_library(), entry)(
        a["s"], a["order"], a["cuo"], *([cap] if entry.endswith("cap") else []), a["cu"] if packed else None,
        200 if packed else 0, a["old"], a["ref"], a["A"], a["w"], B, N, 0.2, 0.2, 0.1, a["g"], a["lp"], a["stats"], a["ws"],
        dora.dora_pl_policy_workspace_size(B), a["st"], None)


def test_draws_outputs_apart():
    a = Room(("s", "order", "cuo", "cu", "old", "ref", "A", "w", "g", "lp", "stats", "ws", "st")).at
    for out in ("g", "lp", "stats", "ws", "st"):
        for other in ("order", "cuo", "cu", "g", "lp", "stats", "ws", "st"):
            if out != other:
                assert draws(**{out: a[other]}) == dora.DORA_ERR_OVERLAP, (out, other)
        for other in ("old", "ref", "A", "w"):
            if out != "lp":
                assert draws(**{out: a[other]}) == dora.DORA_ERR_OVERLAP
        if out != "g":
            assert draws(**{out: a["s"]}) == dora.DORA_ERR_OVERLAP
            # the last score, packed (200 of them) and dense (7 of 40)
            assert out == "ws" or draws(**{out: a["s"] + 199 * 4}) == dora.DORA_ERR_OVERLAP
            assert out == "ws" or draws(packed=False, **{out: a["s"] + 279 * 4}) == dora.DORA_ERR_OVERLAP
        assert draws(entry="dora_pl_policy_loss", **{out: a["order"]}) == dora.DORA_ERR_OVERLAP
    for other in ("old", "ref", "A", "w"):
        assert draws(lp=a[other] + 4) == dora.DORA_ERR_OVERLAP
        assert draws(lp=a[other] - 24) == dora.DORA_ERR_OVERLAP
    assert draws(lp=a["cuo"] + 7 * 4) == dora.DORA_ERR_OVERLAP       # the last offset
    assert draws(lp=a["order"] + 49 * 4) == dora.DORA_ERR_OVERLAP    # the last draw


def clip(grads, out=None, max_norm=1.0, norm=A, ws=A + (1 << 24)):
    spans = lambda items: (dora.Span * len(items))(*(dora.Span(*i) for i in items))
    g, o = spans(grads), None if out is None else spans(out)
    return dora.load_library().dora_grad_clip(ctypes.addressof(g), None if o is None else ctypes.addressof(o), len(grads),
                                              max_norm, 1e-6, norm, ws, dora.dora_grad_clip_workspace_size(len(grads)), None)


@pytest.mark.parametrize("max_norm", [1.0, float("inf")])
def test_clip_outputs_apart(max_norm):
    """The norm and the workspace apart from every tensor, read or written."""
    a, b = (A + (2 << 24), 100, 0, 0), (A + (3 << 24), 33, 1, 0)
    for tensors in ([a, b], [b, a]):
        for at in (a[0], a[0] + 396, b[0], b[0] + 64):
            assert clip(tensors, max_norm=max_norm, norm=at) == dora.DORA_ERR_OVERLAP
        for at in (a[0], b[0], a[0] - 256):
            assert clip(tensors, max_norm=max_norm, ws=at) == dora.DORA_ERR_OVERLAP
    assert clip([a], max_norm=max_norm, norm=A + (1 << 24) + 8) == dora.DORA_ERR_OVERLAP     # inside the workspace
    if max_norm == 1.0:
        assert clip([a], out=[(A + (4 << 24), 100, 0, 0)], norm=A + (4 << 24) + 8) == dora.DORA_ERR_OVERLAP
        assert clip([a], out=[(A + (4 << 24), 100, 0, 0)], ws=A + (4 << 24)) == dora.DORA_ERR_OVERLAP


def scored(dora, rows, V, dtype):
    """A batch, the actions' log-probabilities in 64 bits, and old ones off the clip's border."""
    g = torch.Generator("cuda").manual_seed(rows + V)
    x = (3 * torch.randn((rows, V), generator=g, device="cuda")).to(dtype)
    act = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    lp = torch.log_softmax(x.double(), 1).gather(1, act.long()[:, None])[:, 0]
    old = (lp - 0.05).float()
    adv = torch.randn(rows, generator=g, device="cuda")
    return x, act, lp, old, adv


SPLIT = [(2, 131072), (8, 131072), (64, 40000), (3, 9001)]       # few long rows: several workgroups each
WHOLE = [(300, 96), (3, 97), (40, 3000), (200, 20000)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["old_logprob", "ref_logprob", "advantage", "weight"])
@pytest.mark.parametrize("rows,V", SPLIT + WHOLE)
def test_logprob_in_an_inputs_place(gpu, rows, V, name):
    """logprob_out in the place of a row's constant: the gradient is that of the
    constants as they were.  Rows that would be split keep one workgroup then, so
    that their fp32 sums are grouped otherwise: within both sums' roundings, at
    most V / 256 + 72 of 2^-24 each, which the slopes (at most 1.2 |A| + 0.2, and
    twice for its own error) and the probabilities (at most 1) carry over."""
    x, act, lp, old, adv = scored(gpu, rows, V, torch.float32)
    c = dict(old_logprob=old, ref_logprob=(lp + 0.1).float(), advantage=adv, weight=torch.full((rows,), 0.5, device="cuda"))
    kw = dict(kl_coef=0.1, entropy_coef=0.01)
    want = gpu.dora_policy_loss(x, act, **{k: v.clone() for k, v in c.items()}, **kw)
    for _ in range(5):
        own = {k: v.clone() for k, v in c.items()}
        got = gpu.dora_policy_loss(x, act, **own, **kw, logprob_out=own[name])
        torch.cuda.synchronize()
        assert got[1].data_ptr() == own[name].data_ptr() and int(got[3].item()) == 0
        u, n = 2.0 ** -24, 2 * (V / 256 + 72)
        assert bool(((got[1] - want[1]).abs() <= (n + 2 * 20) * u).all())           # |log p| below 20
        pull = 0.5 * (1.2 * adv.abs() + 0.2 + 0.01 * (20 + 20))                     # slope, entropy's share
        near = 2 * (n + 24) * u * pull[:, None] * 2 + 2 * u * want[0].abs() + 1e-38
        assert bool(((got[0] - want[0]).abs() <= near).all())
        if (rows, V) in WHOLE:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V", SPLIT + WHOLE)
def test_scores_in_the_weights_place(gpu, rows, V):
    x, act, lp, old, adv = scored(gpu, rows, V, torch.bfloat16)
    w = torch.ones(rows, device="cuda")
    w[0] = 0.0
    want = gpu.dora_action_logprob(x, act, weight=w)
    for k in ("logprob_out", "entropy_out"):
        own = w.clone()
        got = gpu.dora_action_logprob(x, act, weight=own, **{k: own})
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and int(got[2].item()) == 0


@pytest.mark.gpu
def test_outputs_in_the_gaps(gpu):
    """A vector may stand in a gap between rows."""
    x, act, lp, old, adv = scored(gpu, 4, 50, torch.float32)
    wide = torch.zeros((4, 60), device="cuda")
    wide[:, :50] = x
    want = gpu.dora_policy_loss(x, act, old, adv)
    got = gpu.dora_policy_loss(wide[:, :50], act, old, adv, logprob_out=wide[1, 50:54], stats_out=wide[2, 52:58])
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_policy_loss(wide[:, :50], act, old, adv, logprob_out=wide[1, 49:53])
    assert e.value.code == gpu.DORA_ERR_OVERLAP
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_policy_loss(x, act, old, adv, dev_status=act[:1])
    assert e.value.code == gpu.DORA_ERR_OVERLAP


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["old_logprob", "ref_logprob", "advantage", "weight"])
@pytest.mark.parametrize("B,N", [(1, 30), (48, 197), (1100, 577)])
def test_draws_in_an_inputs_place(gpu, B, N, name):
    g = torch.Generator("cuda").manual_seed(B)
    s = torch.randn((B, N), generator=g, device="cuda")
    gumbel = -torch.log(-torch.log(torch.rand((B, N), generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    k = torch.randint(0, N, (B,), generator=g, device="cuda", dtype=torch.int32)
    order, cu, old, _ = gpu.dora_pl_sample(s, gumbel, k)
    if B > 2:
        order[int(cu[1])] = -1                                # a bad image, and one that is padding
    w = torch.full((B,), 0.5, device="cuda")
    w[B // 2] = 0.0 if B > 1 else 0.5
    c = dict(old_logprob=old - 0.1, ref_logprob=old + 0.1, advantage=torch.randn(B, generator=g, device="cuda"), weight=w)
    want = gpu.dora_pl_policy_loss(s, order, cu, **{k: v.clone() for k, v in c.items()}, kl_coef=0.1)
    for _ in range(3):
        own = {k: v.clone() for k, v in c.items()}
        got = gpu.dora_pl_policy_loss(s, order, cu, **own, kl_coef=0.1, logprob_out=own[name])
        for a, b in zip(got, want):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


@pytest.mark.gpu
def test_clip_beside_the_norm(gpu):
    """Gradients, the norm and empty tensors as views of one buffer."""
    flat = torch.randn(400, device="cuda")
    ws = gpu.new_grad_clip_workspace(3)
    want, norm = gpu.dora_grad_clip([flat[:100].clone(), flat[101:].clone()], 0.5)
    empty = ws[64:64].view(torch.float32)
    gpu.dora_grad_clip([flat[:100], flat[100:100], flat[101:], empty], 0.5, norm_out=flat[100:101],
                       workspace=torch.cat([ws, ws]))
    assert torch.equal(flat[:100], want[0]) and torch.equal(flat[101:], want[1]) and torch.equal(flat[100:101], norm)
    out, norm2 = gpu.dora_grad_clip([want[0], empty], 1e9, out=[torch.empty_like(want[0]), empty], workspace=ws)
    assert torch.equal(out[0], want[0])
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_grad_clip([flat[:101]], 0.5, norm_out=flat[100:101])
    assert e.value.code == gpu.DORA_ERR_OVERLAP
