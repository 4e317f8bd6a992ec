"""GPU parity of dora_action_logprob and dora_policy_loss with the formulas in
64 bits (policy_ref), at the sizes, strides and masks where they can go wrong.

Tolerances, in half steps u = 2^-24 of fp32, from what the kernel does.  A row's sum of
n terms is at most n / 16 additions a lane and a merge of the lanes (under 64
roundings more); each term has its exponent's rounding (|x - m| u, weighted by
the term itself, so at most u / e) and exp2's (2 u).  So the sum is within
(n / 16 + 68) u, and so are log p and, with terms up to |x - m| long, H:
  |logp| error <= (n / 16 + 68) u + u |logp|   (the last for storing it)
  |H| error    <= (n / 16 + 68) u (2 + H) + u H
The slope w G has the relative error of the ratio and of exp(ref - logp): the error of
logp above.  p_j carries the sum's and |x_j - m| u and 4 u more.  dlogits is
rounded once to its type.
"""
import numpy as np
import pytest
import torch

import policy_ref as P
from gpu_util import to_dev, widen

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(T, V, dtype, seed=0, pad=0, legal=False, masked=0.0, ref=True, scale=3.0, low=0.2, high=0.28):
    """A case: device tensors by argument name, and the same values in numpy."""
    rng = np.random.default_rng([seed, T, V])
    full = torch.from_numpy((scale * rng.standard_normal((T, V + pad))).astype(np.float32)).to(DT[dtype]).cuda()
    logits = full[:, :V]
    x = logits.double().cpu().numpy()
    n = rng.integers((V + 1) // 2, V + 1, T).astype(np.int32) if legal else None
    top = np.full(T, V) if n is None else n
    actions = (rng.random(T) * top).astype(np.int32)
    lp = np.array([P.softmax_row(x[t, :top[t]], actions[t])[0] for t in range(T)])
    h = dict(x=x, actions=actions, legal=n, low=low, high=high,
             old=P.off_border(lp, 0.3 * rng.standard_normal(T), low, high),
             A=rng.standard_normal(T).astype(np.float32),
             ref=(lp + 0.3 * rng.standard_normal(T)).astype(np.float32) if ref else None,
             weight=None)
    if masked:
        h["weight"] = np.where(rng.random(T) < masked, 0.0, rng.random(T) + 0.1).astype(np.float32)
    return logits, h


def dev(a):
    return None if a is None else to_dev(a)


def run(dora, logits, h, kl=0.0, ent=0.0, **kw):
    kl = kl if h["ref"] is not None else 0.0
    out = dora.dora_policy_loss(logits, dev(h["actions"]), dev(h["old"]), dev(h["A"]), ref_logprob=dev(h["ref"]),
                                weight=dev(h["weight"]), legal=dev(h["legal"]), clip_low=h["low"], clip_high=h["high"],
                                kl_coef=kl, entropy_coef=ent, **kw)
    torch.cuda.synchronize()
    return out


def plain(h, kl, ent):
    f32 = lambda v: float(np.float32(v))   # the coefficients reach the kernel in fp32
    return P.policy(h["x"], h["actions"], h["old"].astype(np.float64), h["A"].astype(np.float64),
                    None if h["ref"] is None else h["ref"].astype(np.float64), h["weight"], h["legal"], f32(h["low"]),
                    f32(h["high"]), f32(kl) if h["ref"] is not None else 0.0, f32(ent))


def check(dora, logits, h, dtype, kl=0.05, ent=0.0, **kw):
    u = P.U32
    g, lp, H, stats, scale = plain(h, kl, ent)
    dl, glp, gst, st = run(dora, logits, h, kl, ent, **kw)
    assert int(st.item()) == 0
    T, V = h["x"].shape
    err_lp = (V / 16 + 68) * u
    got_lp = glp.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got_lp - lp) <= err_lp + u * np.abs(lp)), np.abs(got_lp - lp).max()
    # the slopes' parts, for their errors
    r = np.exp(lp - h["old"])
    w = np.ones(T) if h["weight"] is None else h["weight"].astype(np.float64)
    pull = np.abs(r * h["A"])
    if h["ref"] is not None:
        pull = pull + kl * (1 + 2 * np.exp(h["ref"] - lp))
    got = widen(dl)
    worst = 0.0
    for t in range(T):
        n = V if h["legal"] is None else int(h["legal"][t])
        if w[t] == 0:
            assert not got[t].any()
            continue
        row = h["x"][t, :n]
        lpr = P.softmax_row(row, h["actions"][t])[2]
        p, d = np.exp(lpr), np.abs(row - row.max())
        # p log p is 0 at p = 0, where |log p| and d are infinite: no share in the error either
        lpr, d = np.where(p > 0, lpr, 0.0), np.where(p > 0, d, 0.0)
        share = err_lp + u * (4 + d)
        tol = w[t] * p * (pull[t] * (share + err_lp) + ent * (np.abs(lpr) + H[t]) * (share + 4 * u) +
                          ent * (err_lp * (3 + H[t]) + 2 * u * (d + H[t])))
        tol[h["actions"][t]] += w[t] * pull[t] * (err_lp + 4 * u)
        tol += P.HALF[dtype] * np.abs(g[t, :n]) + 1e-38   # the type's own rounding; subnormal results
        e = np.abs(got[t, :n] - g[t, :n])
        assert np.all(e <= tol), (t, int(np.argmax(e - tol)), e.max())
        worst = max(worst, float((e / tol).max()))
        assert not got[t, n:].any()
    got_st = gst.cpu().numpy().astype(np.float64)
    err_H = err_lp * (2 + np.log(V)) + u * np.log(V + 1)
    dkl = kl * (np.exp(h["ref"] - lp) + 1) if h["ref"] is not None else 0
    each = np.abs(w) * err_lp
    tol = np.array([(each * (pull + dkl)).sum() + ent * (np.abs(w) * err_H).sum(), (each * pull).sum(),
                    (each * (0 if h["ref"] is None else np.expm1(np.abs(h["ref"] - lp)) + 1)).sum(),
                    (np.abs(w) * err_H).sum(), 0, 0]) + u * np.abs(stats) + 1e-30
    assert np.all(np.abs(got_st - stats) <= tol), (got_st, stats, tol)
    print(f"[policy] {dtype} T={T} V={V} gradient error at most {worst:.2f} of the bound", flush=True)
    return dl, glp, gst


SIZES = [(1, 1), (5, 1), (3, 2), (4, 3), (2, 7), (3, 8), (3, 9), (300, 15), (7, 16), (33, 17), (1024, 96), (50, 126),
         (17, 127), (5, 511), (6, 512), (9, 513), (3, 1000), (5, 2047), (4, 2049), (3, 4097), (2, 10000), (260, 8191),
         (2, 32000), (3, 50257), (1, 65537), (2, 131072), (1, 140001), (20, 70001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", SIZES)
def test_sizes(gpu, T, V, dtype):
    logits, h = make(T, V, dtype, seed=1)
    check(gpu, logits, h, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad", [(96, 0), (97, 3), (500, 13), (5001, 1), (40000, 7)])
def test_strides_legal_masks_entropy(gpu, V, pad, dtype):
    logits, h = make(29, V, dtype, seed=2, pad=pad, legal=True, masked=0.3)
    T = 29
    room = torch.full((T, V + 5), 7.0, dtype=DT[dtype], device="cuda")
    check(gpu, logits, h, dtype, ent=0.02, dlogits=room[:, 2:V + 2])
    assert bool((room[:, :2] == 7).all()) and bool((room[:, V + 2:] == 7).all())   # between the rows


def test_no_reference_no_kl(gpu):
    logits, h = make(40, 333, "f32", seed=3, ref=False)
    check(gpu, logits, h, "f32", kl=0.0)


def test_coefficient_zero_ignores_infinite_kl(gpu):
    """The reference gives the action no chance and the other way round: kl is
    infinite or huge, and counts for nothing at coefficient 0."""
    logits, h = make(4, 50, "f32", seed=4)
    h["ref"][:2] = -np.inf
    h["ref"][2] = 1e30
    dl, lp, st, _ = run(gpu, logits, h, kl=0.0)
    h["ref"] = np.zeros(4, np.float32)
    dl2, lp2, st2, _ = run(gpu, logits, h, kl=0.0)
    assert torch.equal(dl, dl2) and torch.equal(lp, lp2) and torch.equal(st[:2], st2[:2])
    assert bool(torch.isfinite(dl).all()) and not bool(torch.isfinite(st[2]).all())


def test_clip_sides(gpu):
    """The four corners of the clip, with the slope that each leaves."""
    logits, h = make(4, 64, "f32", seed=5, ref=False)
    lp = np.array([P.softmax_row(h["x"][t], h["actions"][t])[0] for t in range(4)])
    h["old"] = (lp - np.array([0.5, 0.5, -0.5, -0.5])).astype(np.float32)
    h["A"] = np.array([1, -1, 1, -1], np.float32)
    dl, _, st = check(gpu, logits, h, "f32", kl=0.0)
    assert not bool(dl[0].any()) and not bool(dl[3].any()) and bool(dl[1].any()) and bool(dl[2].any())
    assert float(st[4]) == 2.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 700, 9000, 70000])
def test_masked_places(gpu, V, dtype):
    """Minus infinity and the type's lowest value as masks, in the open part;
    NaN and infinities where nothing may look."""
    logits, h = make(12, V, dtype, seed=6, legal=True, pad=3)
    full = torch.full((12, V + 3), float("nan"), dtype=DT[dtype], device="cuda")
    full[:, :V] = logits
    low = torch.finfo(DT[dtype]).min
    keep = torch.rand((12, V), generator=torch.Generator("cuda").manual_seed(7), device="cuda") < 0.5
    keep[torch.arange(12), torch.from_numpy(h["actions"]).long().cuda()] = True
    full[:4, :V] = torch.where(keep[:4], full[:4, :V], torch.full_like(full[:4, :V], -float("inf")))
    full[4:8, :V] = torch.where(keep[4:8], full[4:8, :V], torch.full_like(full[4:8, :V], low))
    full[8] = low                       # all alike: uniform
    full[9] = -float("inf")             # all but the action closed
    full[9, int(h["actions"][9])] = 1.5
    full[10, :V] = torch.where(keep[10], full[10, :V] + 1e30, full[10, :V])   # large, and equal only in part
    for t in range(12):
        full[t, int(h["legal"][t]):] = float("nan")
    logits = full[:, :V]
    h["x"] = logits.double().cpu().numpy()
    lp = np.array([P.softmax_row(h["x"][t, :h["legal"][t]], h["actions"][t])[0] for t in range(12)])
    h["old"] = P.off_border(lp, np.full(12, 0.05), h["low"], h["high"])
    h["ref"] = (lp + 0.1).astype(np.float32)
    check(gpu, logits, h, dtype, ent=0.01)


@pytest.mark.parametrize("base", [2e6, 5.3e8, 9e8, 1.2e9, -5.3e8, -1.2e9, 3.3e38, -3.3e38])
@pytest.mark.parametrize("V", [300, 70000])
def test_vast_logits(gpu, V, base):
    """A few logits of one value, all others the next float below: as far apart
    as the type allows there, so the few share the probability (at 2e6 they
    differ by an eighth)."""
    logits, h = make(2, V, "f32", seed=17)
    top = np.float32(base)
    logits[:] = float(np.nextafter(top, np.float32(-np.inf)))
    logits[:, 5:8] = float(top)
    h["actions"][:] = [6, V - 1]
    h["x"] = logits.double().cpu().numpy()
    lp = np.array([P.softmax_row(h["x"][t], h["actions"][t])[0] for t in range(2)])
    h["old"] = P.off_border(lp, np.full(2, 0.05), h["low"], h["high"])
    h["ref"] = (lp + 0.1).astype(np.float32)
    if abs(base) > 1e8:      # the second row's action has no chance
        h["actions"][1] = 7
        h["old"][1], h["ref"][1] = h["old"][0], h["ref"][0]
    check(gpu, logits, h, "f32", ent=0.01)


@pytest.mark.parametrize("V", [40, 700, 9000, 70000])
def test_rows_left_out(gpu, V):
    """Padding rows are not looked at; bad rows are reported, get NaN and a
    zero gradient, and have no share in the sums."""
    logits, h = make(10, V, "f32", seed=8, legal=True)
    h["weight"] = np.full(10, 0.1, np.float32)
    h["weight"][[1, 4]] = 0.0
    good = [0, 2, 3, 6]
    dl0, lp0, st0, _ = run(gpu, logits[good].contiguous(), {**h, **{k: h[k][good] for k in
                           ("actions", "legal", "old", "A", "ref", "weight")}}, kl=0.05, ent=0.01)
    logits[[1, 4]] = float("nan")                 # padding: anything
    h["actions"][[1, 4]] = [-5, 1 << 30]
    h["legal"][1] = -7
    for k in ("old", "A", "ref"):
        h[k][[1, 4]] = np.nan
    h["actions"][5] = h["legal"][5]               # just past the open ones
    h["actions"][7] = -1
    h["legal"][8] = 0
    logits[9] = -float("inf")                     # nothing open
    dl, lp, st, flag = run(gpu, logits, h, kl=0.05, ent=0.01)
    assert int(flag.item()) == gpu.DORA_DEV_ACTION
    bad = [5, 7, 8, 9]
    assert bool(torch.isnan(lp[bad]).all()) and not bool(lp[[1, 4]].any())
    assert not bool(dl[bad + [1, 4]].any())
    assert torch.equal(dl[good], dl0) and torch.equal(lp[good], lp0)
    assert torch.allclose(st, st0, rtol=2e-6, atol=0)   # the same terms; sums of another order
    h["legal"][2] = V + 1                         # past the row's end
    _, lp, _, flag = run(gpu, logits, h, kl=0.05)
    assert int(flag.item()) == gpu.DORA_DEV_ACTION and bool(torch.isnan(lp[2]))
    lp, H, flag = gpu.dora_action_logprob(logits, dev(h["actions"]), weight=dev(h["weight"]), legal=dev(h["legal"]))
    assert int(flag.item()) == gpu.DORA_DEV_ACTION
    assert bool(torch.isnan(lp[bad]).all()) and bool(torch.isnan(H[bad]).all()) and not bool(H[[1, 4]].any())


@pytest.mark.parametrize("V", [40, 9000, 70000])
def test_nan_and_infinity_are_seen(gpu, V):
    logits, h = make(3, V, "f32", seed=9)
    logits[0, V - 1] = float("nan")
    logits[1, V // 2] = float("inf")
    dl, lp, st, flag = run(gpu, logits, h, kl=0.05)
    assert bool(torch.isnan(lp[:2]).all()) and bool(torch.isfinite(lp[2])) and int(flag.item()) == 0
    assert bool(torch.isnan(dl[0]).any()) and bool(torch.isnan(dl[1]).any()) and bool(torch.isfinite(dl[2]).all())
    assert bool(torch.isnan(st[0]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(50, 96), (3, 97), (20, 513), (4, 4096), (3, 9001), (2, 131072), (2, 150001), (30, 70001)])
def test_in_place(gpu, T, V, dtype):
    """The gradient over the logits, to the last bit what it is beside them."""
    logits, h = make(T, V, dtype, seed=10, masked=0.2)
    want, lp, st, _ = run(gpu, logits, h, kl=0.05, ent=0.01)
    got, lp2, st2, _ = run(gpu, logits, h, kl=0.05, ent=0.01, dlogits=logits)
    assert got.data_ptr() == logits.data_ptr()
    assert torch.equal(got, want) and torch.equal(lp, lp2) and torch.equal(st, st2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(1, 1), (1, 131072), (3, 50257), (1, 1048576), (5, 200003), (64, 97), (700, 5000), (1, 33)])
def test_logprob(gpu, T, V, dtype):
    logits, h = make(T, V, dtype, seed=11, pad=1)
    want = [P.softmax_row(h["x"][t], h["actions"][t])[:2] for t in range(T)]
    u, n = P.U32, V / 16 + 68
    for single in (False, True):
        lp, H, st = gpu.dora_action_logprob(logits, dev(h["actions"]), single=single)
        assert int(st.item()) == 0
        for got, w, each in ((lp, 0, 1), (H, 1, 2 + np.log(V))):
            w = np.array([row[w] for row in want])
            assert np.all(np.abs(got.cpu().numpy() - w) <= n * u * each + u * np.abs(w))
    # without the entropy, by the C entry
    only = torch.empty(T, device="cuda")
    lib, flag = gpu.load_library(), gpu.new_status()
    rc = lib.dora_action_logprob(logits.data_ptr(), logits.stride(0) if T > 1 else V, dev(h["actions"]).data_ptr(), None,
                                 None, T, V, gpu.DORA_BF16 if dtype == "bf16" else gpu.DORA_F32, only.data_ptr(), None,
                                 None, 0, flag.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and torch.equal(only, lp)


def test_loss_and_logprob_agree(gpu):
    """The ratio of a row scored by the two entry points is 1 up to the rounding
    of the stored log-probability, whatever the size class of the rows."""
    for V in (96, 4096, 50257, 131072):
        logits, h = make(5, V, "bf16", seed=12, ref=False)
        lp, _, _ = gpu.dora_action_logprob(logits, dev(h["actions"]))
        h["A"] = np.ones(5, np.float32)
        _, lp2, st, _ = run(gpu, logits, {**h, "old": lp.cpu().numpy()})
        u = P.U32
        assert torch.all((lp - lp2).abs() <= 2 * (V / 16 + 68) * u + 2 * u * lp.abs())
        assert abs(float(st[1]) - 5.0) <= 5 * (2 * (V / 16 + 68) + 2 * 20) * u


def test_offsets_past_32_bits(gpu):
    """Logits of more than 2^32 elements' reach: rows far apart, few of them."""
    V, ld = 1000, (1 << 30) + 8
    buf = torch.empty(4 * ld + V, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((5, V), (ld, 1))
    small, h = make(5, V, "bf16", seed=13)
    rows.copy_(small)
    want = run(gpu, small, h, kl=0.05)
    got = run(gpu, rows, h, kl=0.05, dlogits=rows)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)


def test_many_rows(gpu):
    """More rows than workgroups, so that each takes several."""
    T = 300000
    g = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn((T, 5), generator=g, device="cuda")
    actions = torch.randint(0, 5, (T,), generator=g, device="cuda", dtype=torch.int32)
    lp = torch.log_softmax(logits.double(), 1).gather(1, actions.long()[:, None])[:, 0]
    A = torch.randn(T, generator=g, device="cuda")
    dl, got, st, flag = gpu.dora_policy_loss(logits, actions, lp.float(), A, weight=torch.full((T,), 1.0, device="cuda"))
    assert int(flag.item()) == 0 and bool(((got - lp).abs() <= 70 * P.U32 + P.U32 * lp.abs()).all())
    p = torch.softmax(logits.double(), 1)
    want = A.double()[:, None] * p
    want.scatter_add_(1, actions.long()[:, None], -A.double()[:, None])
    assert bool(((dl - want).abs() <= 200 * P.U32 * A.abs()[:, None]).all())
    assert abs(float(st[1]) - float(A.double().sum())) <= 100 * P.U32 * float(A.double().abs().sum())
    assert float(st[5]) == T


@pytest.mark.parametrize("T,V", [(64, 96), (40, 3000), (3, 131072), (600, 20000)])
def test_repeats_to_the_last_bit(gpu, T, V):
    logits, h = make(T, V, "bf16", seed=14, masked=0.2)
    first = run(gpu, logits, h, kl=0.05, ent=0.01)
    ws = torch.randint(0, 255, (gpu.dora_policy_workspace_size(T, V),), dtype=torch.uint8, device="cuda")   # no required contents
    again = run(gpu, logits, h, kl=0.05, ent=0.01, workspace=ws)
    for a, b in zip(first[:3], again[:3]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("by_handle", [False, True])
def test_on_a_stream(gpu, by_handle):
    """Enqueued on the given stream, after what that stream waits for, with all
    that the call makes for itself; the current stream need not wait."""
    logits, h = make(300, 5000, "bf16", seed=15)
    want = run(gpu, logits, h, kl=0.05)
    side = torch.cuda.Stream()
    late = torch.zeros_like(logits)
    args = {k: dev(h[k]) for k in ("actions", "old", "A", "ref")}
    torch.cuda.synchronize()
    busy = torch.ones(1 << 28, device="cuda")
    for _ in range(20):
        busy.mul_(1.0)                                 # the current stream has work of its own
    with torch.cuda.stream(side):
        for _ in range(20):
            late.copy_(logits)
        late.neg_().neg_()
    stream = side.cuda_stream if by_handle else side
    got = gpu.dora_policy_loss(late, args["actions"], args["old"], args["A"], ref_logprob=args["ref"], clip_low=0.2,
                               clip_high=0.28, kl_coef=0.05, stream=stream)
    lp, H, st = gpu.dora_action_logprob(late, args["actions"], stream=stream)
    out, norm = gpu.dora_grad_clip([got[0]], 1e9, out=[torch.empty_like(late)], stream=stream)
    side.synchronize()
    assert int(got[3].item()) == 0 and int(st.item()) == 0
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)
    assert torch.equal(out[0], want[0])
    assert torch.all((lp - want[1]).abs() <= 2 * (5000 / 16 + 68) * P.U32 + 2 * P.U32 * want[1].abs())


def test_refusals(gpu):
    logits, h = make(4, 20, "f32", seed=16)
    a, f = dev(h["actions"]), dev(h["old"])
    with pytest.raises(ValueError, match="adjacent"):
        gpu.dora_action_logprob(logits.t(), a[:4].repeat(5))
    with pytest.raises(TypeError, match="dtype"):
        gpu.dora_action_logprob(logits.half(), a)
    with pytest.raises(TypeError, match="actions must be"):
        gpu.dora_action_logprob(logits, a.long())
    with pytest.raises(ValueError, match=r"actions must be \[4\]"):
        gpu.dora_policy_loss(logits, a[:3], f, f)
    with pytest.raises(ValueError, match="tensors on"):
        gpu.dora_policy_loss(logits, a, f, f.cpu())
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_policy_loss(logits, a, f, f, kl_coef=0.1)
    assert e.value.code == gpu.DORA_ERR_NULL
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_policy_loss(logits[:, :10], a, f, f, dlogits=logits[:, 5:15])
    assert e.value.code == gpu.DORA_ERR_OVERLAP
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_policy_loss(logits, a, f, f, workspace=gpu.new_workspace(1, 1, 1)[:64])
    assert e.value.code == gpu.DORA_ERR_WORKSPACE
    with pytest.raises(gpu.DoraError) as e:
        gpu.dora_policy_loss(logits[:0], a[:0], f[:0], f[:0], workspace=gpu.new_policy_workspace(1, 20))
    assert e.value.code in (gpu.DORA_ERR_SHAPE, gpu.DORA_ERR_NULL)     # an empty tensor may have no address
    gpu.dora_policy_loss(logits[:, :10], a.clamp(max=9), f, f, dlogits=logits[:, 10:])   # rows in the gaps of the others
    torch.cuda.synchronize()
