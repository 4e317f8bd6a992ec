"""Every open element of a row is counted once, at every width of a row's
workgroups: rows whose sums are whole numbers, rows with two places that count,
and random rows under the bound of the lanes that really hold them.

  test_equal_logits   n equal open logits of 0: each term is 2^0 = 1, the sum n is
                      exact in fp32, log p = -log n and H = log n are rounded once.
                      An element left out or taken twice moves log p by 1 / n.
  test_two_places     all logits at -60 but the action's and one other, at 0: log p
                      is -log 2, or 0 where the other is not seen (a million e^-60
                      are 1e-20).  The other stands at each border of what a lane,
                      a workgroup's share or a boundary of 16 bytes holds.
  test_random_rows    a lane adds V / lanes terms and those at the edges, the lanes
                      meet in 10 additions; each term has its exponent's rounding
                      and log2(e)'s (|x - m| u, up to 13 u each by the terms'
                      weight) and exp2's (2 u): V / lanes + E + 68 of u in all.
"""
import math

import numpy as np
import pytest
import torch

from policy_ref import HALF, U32

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
PER = {"f32": 4, "bf16": 8}                    # elements of 16 bytes

WIDTHS = [5, 250, 513, 1025, 2049, 4097, 9001, 12289, 16385, 20001, 28673, 32769, 40961, 50257, 65537, 81921, 98305, 114689,
          131073, 163841, 200001, 300001, 1048576]


def lanes(V, dtype, split=1):
    """Threads that hold a row of the loss."""
    pieces = -(-V // PER[dtype])
    if pieces <= 512:
        return 16 if pieces <= 64 else 64
    if split > 1:
        return 256 * split
    return 256 if pieces <= 4096 else (512 if pieces <= 8192 else 1024)


def split_of(T, V, dtype):
    """Workgroups a row of the loss."""
    pieces = -(-V // PER[dtype])
    if pieces <= 512 or T > 128 or pieces // 64 < T:
        return 1
    return max(1, min(512 // T, pieces // 512, 64))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_bounds_see_what_is_left_out(dtype):
    """On the host: a row's sum without one element (a piece of 16 bytes, past
    2^19 elements), in a plain form, is outside the bounds below."""
    for V in WIDTHS[1:]:
        gone = 1 if V < 1 << 19 else PER[dtype]
        for n in (V, V // 2 + 1):
            assert abs(math.log(n) - math.log(n - gone)) > 2 * (U32 * math.log(n) + 1e-12)
        two = np.full(V, -60.0)
        two[[3, V - 1]] = 0.0
        assert abs(math.log(np.exp(two).sum()) - math.log(np.exp(two[:-1]).sum())) > 0.69


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [130, 6, 1])
@pytest.mark.parametrize("V", WIDTHS)
def test_equal_logits(gpu, T, V, dtype):
    u, g = U32, torch.Generator("cuda").manual_seed(V + T)
    legal = torch.randint(1, V + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    legal[:3] = torch.tensor([V, max(V - 1, 1), 1], dtype=torch.int32)[:T]
    n = legal.double()
    x = torch.zeros((T, V), dtype=DT[dtype], device="cuda")
    x[torch.arange(V, device="cuda")[None, :] >= legal[:, None]] = float("nan")
    act = (torch.rand(T, generator=g, device="cuda", dtype=torch.float64) * n).int().minimum(legal - 1)
    adv = torch.randn(T, generator=g, device="cuda")
    old = (-torch.log(n) - 0.05).float()
    lp = -torch.log(n)
    for single in (False, True):
        got, H, st = gpu.dora_action_logprob(x, act, legal=legal, single=single)
        assert int(st.item()) == 0
        assert bool(((got - lp).abs() <= u * lp.abs() + 1e-12).all()) and bool(((H + lp).abs() <= u * lp.abs() + 1e-12).all())
    slope = -torch.exp(lp - old.double()) * adv.double()
    want = (-slope / n)[:, None].expand(T, V).clone()
    want.scatter_add_(1, act.long()[:, None], slope[:, None])
    want[torch.isnan(x)] = 0.0
    # the row's factor is rounded to fp32, so is the slope, and their sum at the action; then the type's own rounding
    tol = (HALF[dtype] * (1 + 2 * u) + 1.01 * u) * want.abs()
    tol.scatter_add_(1, act.long()[:, None], (1.01 * u * slope.abs() * (1 + 1 / n))[:, None])
    for ent in (0.0, 0.5):                     # the entropy is largest here: no gradient of its own
        dl, got, st, flag = gpu.dora_policy_loss(x, act, old, adv, legal=legal, entropy_coef=ent)
        assert int(flag.item()) == 0 and bool(((got - lp).abs() <= u * lp.abs() + 1e-12).all())
        # its two sides, 0.5 log n each by the sum, cancel to a few 2^-53 of themselves
        assert bool(((dl.double() - want).abs() <= tol + ent * 1e-13 + 1e-38).all())
        assert abs(float(st[3]) + float(lp.sum())) <= u * float(lp.abs().sum()) + 1e-9


def places(V, dtype, pieces_each, seed):
    """Borders of runs of `pieces_each` pieces, the row's ends, and some others."""
    E = PER[dtype]
    at = set(range(min(V, 18))) | set(range(max(V - 18, 0), V))
    for border in range(pieces_each * E, V + 18, pieces_each * E):
        at |= {border + d for d in (-9, -8, -5, -4, -1, 0, 1, 3, 7)}
    at |= set(np.random.default_rng(seed).integers(0, V, 40).tolist())
    return sorted(i for i in at if 0 <= i < V)


def two_places(dora, V, dtype, at, lead):
    """Rows with two places that count, the gradient `lead` elements past a 16-byte boundary."""
    T = len(at)
    x = torch.full((T, V), -60.0, dtype=DT[dtype], device="cuda")
    at = torch.tensor(at, device="cuda")
    act = torch.where(at == V // 3, V // 3 + 1, V // 3) if V > 1 else at
    rows = torch.arange(T, device="cuda")
    x[rows, at] = 0.0
    x[rows, act] = 0.0
    old = torch.full((T,), -0.75, device="cuda")
    adv = torch.where(rows % 2 == 0, -1.5, 1.0)
    room = torch.full((T * V + 64,), 7.0, dtype=DT[dtype], device="cuda")
    out = room[lead:lead + T * V].view(T, V)
    dl, lp, st, flag = dora.dora_policy_loss(x, act.int(), old, adv, dlogits=out)
    half = -math.log(2.0)
    assert int(flag.item()) == 0 and bool(((lp - half).abs() <= U32).all()), at[(lp - half).abs() > U32]
    slope = -math.exp(half + 0.75) * adv.double()
    pair = torch.stack([dl[rows, act], dl[rows, at]]).double()
    want = torch.stack([slope / 2, -slope / 2])
    assert bool(((pair - want).abs() <= (HALF[dtype] + 4 * U32) * want.abs() + 2 * U32 * slope.abs()).all())
    dl[rows, act] = 0.0
    dl[rows, at] = 0.0
    assert float(dl.abs().max()) <= 1e-20      # e^-60 = 9e-27 of the slope
    assert bool((room[:lead] == 7).all()) and bool((room[lead + T * V:] == 7).all())
    one, H, flag = dora.dora_action_logprob(x, act.int())
    assert bool(((one - half).abs() <= U32).all()) and bool(((H + half).abs() <= U32).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", WIDTHS[1:])
def test_two_places(gpu, V, dtype):
    at = places(V, dtype, lanes(V, dtype), V)
    at += at[:max(0, 130 - len(at))]           # past 128 rows: none is split
    two_places(gpu, V, dtype, at, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(1, 9001), (3, 16385), (8, 50257), (8, 131072), (2, 300001), (1, 1048576), (32, 65537)])
def test_two_places_of_split_rows(gpu, T, V, dtype):
    split = split_of(T, V, dtype)
    assert split > 1
    at = places(V, dtype, -(-(-(-V // PER[dtype])) // split), V + 1)
    for i in range(0, len(at), T):
        part = at[i:i + T]
        two_places(gpu, V, dtype, part + part[:1] * (T - len(part)), 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9001, 20001, 50257, 90001, 131073, 200001, 300001])
@pytest.mark.parametrize("T", [130, 4])
def test_random_rows(gpu, T, V, dtype):
    g = torch.Generator("cuda").manual_seed(V + 7)
    x = (3 * torch.randn((T, V), generator=g, device="cuda")).to(DT[dtype])
    act = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    lsm = torch.log_softmax(x.double(), 1)
    lp = lsm.gather(1, act.long()[:, None])[:, 0]
    H = -(lsm.exp() * lsm).sum(1)
    _, got, st, _ = gpu.dora_policy_loss(x, act, lp.float(), torch.ones(T, device="cuda"))
    err = (V / lanes(V, dtype, split_of(T, V, dtype)) + PER[dtype] + 68) * U32
    assert bool(((got - lp).abs() <= err + U32 * lp.abs()).all()), float((got - lp).abs().max())
    err = (V / 256 + PER[dtype] + 68) * U32    # log-probabilities alone: 256 threads or more
    for single in (False, True):
        got, gH, _ = gpu.dora_action_logprob(x, act, single=single)
        assert bool(((got - lp).abs() <= err + U32 * lp.abs()).all())
        assert bool(((gH - H).abs() <= err * (2 + H) + U32 * H).all())
