"""Grouped attention, forward and backward, against the 64-bit reference, element
by element, and by sums that are exact."""
import itertools

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def cu_of(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def dev_cu(cu):
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def make(nq, nk, H, Hk, D, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    cu_q, cu_k = cu_of(nq), cu_of(nk)

    def heads(n, h):
        return (size * torch.randn((n, h, D), generator=g)).to(dtype)
    t = dict(q=heads(cu_q[-1], H), k=heads(cu_k[-1], Hk), v=heads(cu_k[-1], Hk), dout=heads(cu_q[-1], H))
    return t, cu_q, cu_k


def cuda(t):
    return {n: x.cuda() for n, x in t.items()}


def run_both(gpu, t, cu_q, cu_k, causal, scale=0.0, what=""):
    d = cuda(t)
    cq, ck = dev_cu(cu_q), dev_cu(cu_k)
    max_q = max(b - a for a, b in zip(cu_q, cu_q[1:]))
    kw = dict(cu_k=ck, causal=causal, softmax_scale=scale)
    out, lse, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], cq, max_q, **kw)
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal, scale or None)
    assert int(st) == 0
    ref.check(out, want["out"], bound["out"], what + " out")
    ref.check(lse, want["lse"], bound["lse"], what + " lse")
    dq, dk, dv, st = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, cq, max_q, **kw)
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal, scale or None, dout=t["dout"], out=out.cpu(),
                                lse=lse.cpu())
    assert int(st) == 0
    for n, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        ref.check(x, want[n], bound[n], f"{what} {n}")
    return out, lse, dq, dk, dv


SELF = [[1], [2, 1, 0, 3], [31, 32, 33], [63, 64, 65, 0], [127, 128, 129], [197, 60, 1], [300]]


@pytest.mark.parametrize("dtype,causal,D", itertools.product(DTYPES, (False, True), (32, 64, 128)))
@pytest.mark.parametrize("H,Hk", [(3, 3), (4, 1), (14, 2)])
def test_self_attention(gpu, dtype, causal, D, H, Hk):
    for i, lens in enumerate(SELF):
        t, cu, _ = make(lens, lens, H, Hk, D, dtype, 10 * i + H)
        run_both(gpu, t, cu, cu, causal, what=str(lens))


@pytest.mark.parametrize("dtype,causal", itertools.product(DTYPES, (False, True)))
@pytest.mark.parametrize("H,Hk,D", [(8, 2, 128), (12, 12, 64), (6, 3, 32)])
def test_own_boundaries(gpu, dtype, causal, H, Hk, D):
    """Queries without keys, keys without queries, more queries than keys (rows that see nothing), a few new tokens."""
    for nq, nk in (([1, 1, 1, 1], [5, 64, 0, 257]), ([3, 0, 9], [100, 7, 65]), ([70, 5, 130], [20, 5, 0]),
                   ([2, 33], [129, 1])):
        t, cu_q, cu_k = make(nq, nk, H, Hk, D, dtype, sum(nq) + D)
        out, lse, *_ = run_both(gpu, t, cu_q, cu_k, causal, 0.3 if D == 64 else 0.0, f"{nq} {nk}")
        if causal:
            for b, (n, m) in enumerate(zip(nq, nk)):
                shut = slice(cu_q[b], cu_q[b] + max(0, n - m))
                assert bool((out[shut] == 0).all()) and bool((lse[shut] == -float("inf")).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,H,Hk,D", [(1, 8, 2, 128), (1, 4, 4, 64), (1, 7, 1, 32), (3, 8, 4, 64), (64, 2, 2, 32), (5, 24, 2, 128)])
def test_split_keys(gpu, dtype, nq, H, Hk, D):
    """Few queries against many keys: split over workgroups and joined, parts of every size."""
    for causal in (False, True):
        for nk in ([3000, 10, 0, 1025], [4097], [257, 2048, 511, 2500, 1]):
            nq_list = [nq] * len(nk)
            t, cu_q, cu_k = make(nq_list, nk, H, Hk, D, dtype, nk[0])
            d = cuda(t)
            out, lse, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu_q), nq, cu_k=dev_cu(cu_k), causal=causal)
            want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal)
            assert int(st) == 0
            ref.check(out, want["out"], bound["out"], f"{nk} out")
            ref.check(lse, want["lse"], bound["lse"], f"{nk} lse")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,H,Hk,D", [(1, 8, 1, 128), (1, 3, 3, 64), (4, 8, 2, 128), (2, 5, 1, 64), (1, 16, 1, 64)])
def test_few_rows(gpu, dtype, nq, H, Hk, D):
    """Few rows a key head: whole and split, lengths on both sides of a part's, the longest known and not, queries that see
    none of a part, values that the last query alone sees."""
    for causal in (False, True):
        for nk in ([1, 2, 31, 32, 33, 255, 256, 257, 0, 511, 513, 3], [9000, 300, 0, 2500, 1, 4097], [8000, 1, 193],
                   [100, 256, 200, 0]):
            t, cu_q, cu_k = make([nq] * len(nk), nk, H, Hk, D, dtype, nk[0] + nq)
            d = cuda(t)
            args = (d["q"], d["k"], d["v"], dev_cu(cu_q), nq)
            out, lse, st = gpu.dora_grouped_attn(*args, cu_k=dev_cu(cu_k), causal=causal)
            want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal)
            assert int(st) == 0
            ref.check(out, want["out"], bound["out"], f"{nk} out")
            ref.check(lse, want["lse"], bound["lse"], f"{nk} lse")
            whole, lse2, st = gpu.dora_grouped_attn(*args, cu_k=dev_cu(cu_k), causal=causal, max_k=max(nk))
            assert int(st) == 0
            ref.check(whole, want["out"], bound["out"], f"{nk} out, longest known")
            ref.check(lse2, want["lse"], bound["lse"], f"{nk} lse, longest known")
            if causal and nq > 1:
                ends = torch.tensor([b - 1 for a, b in zip(cu_k, cu_k[1:]) if b - a > 1])
                d["v"][ends, :, 2] = float("inf")
                d["v"][ends, :, 5] = float("nan")
                out, _, _ = gpu.dora_grouped_attn(*args, cu_k=dev_cu(cu_k), causal=True)
                for b in range(len(nk)):
                    rows = slice(cu_q[b], cu_q[b + 1] - 1)
                    ref.check(out[rows], want["out"][rows], bound["out"][rows], f"{nk} {b} odd")
                    if nk[b] > 1:
                        assert bool((out[cu_q[b + 1] - 1, :, 2] == float("inf")).all())
                        assert bool(torch.isnan(out[cu_q[b + 1] - 1, :, 5]).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_split_tiles(gpu, dtype):
    """Several tiles of queries, still few: keys split, causal and not; dk and dv split over many rows."""
    for causal, nq, nk, H, Hk, D in ((True, [150], [5000], 4, 2, 64), (False, [90, 40], [4000, 3500], 4, 1, 128),
                                     (True, [3000], [3000], 4, 1, 32), (False, [2500], [100], 8, 1, 64)):
        t, cu_q, cu_k = make(nq, nk, H, Hk, D, dtype, nq[0])
        run_both(gpu, t, cu_q, cu_k, causal, what=f"{nq} {nk}")


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
@pytest.mark.parametrize("nq,nk,G,causal", [(1, 70, 1, True), (70, 70, 1, True), (70, 70, 3, False), (40, 200, 2, True),
                                            (1, 3000, 4, True), (130, 2500, 1, True)])
def test_each_key_counts_once(gpu, dtype, D, nq, nk, G, causal):
    """Equal scores weigh every key that a row sees the same: 1 / their number, and no other key at all."""
    q = torch.zeros((nq, G, D), dtype=dtype, device="cuda")
    k = torch.randn((nk, 1, D), device="cuda").to(dtype)
    cq, ck = dev_cu([0, nq]), dev_cu([0, nk])
    sees = torch.arange(nq) + 1 + nk - nq if causal else torch.full((nq,), nk)
    places = sorted({0, 1, 15, 16, 31, 32, 63, 64, 69, nk // 2, nk - 2, nk - 1, nk - nq, max(0, nk - nq - 1), 255, 256, 1023, 1024}
                    & set(range(nk)))
    # one key's value at a time, each in an element of its own
    for lo in range(0, len(places), D):
        v = torch.zeros((nk, 1, D), dtype=dtype, device="cuda")
        for e, j in enumerate(places[lo:lo + D]):
            v[j, 0, e] = 1.0
        out, lse, _ = gpu.dora_grouped_attn(q, k, v, cq, nq, cu_k=ck, causal=causal)
        got = out.double().cpu()
        for e, j in enumerate(places[lo:lo + D]):
            want = torch.where(j < sees, 1.0 / sees.double(), torch.zeros(nq, dtype=torch.float64))
            # every term is exactly 1, sums of up to 4096 ones too; a reciprocal, a product, the result's rounding
            tol = want * (ref.HALF[dtype] + 8 * ref.U)
            assert bool(((got[:, :, e] - want[:, None]).abs() <= tol[:, None]).all()), j
        assert bool((lse.cpu().double() - torch.log(sees.double())[:, None]).abs().max() < 3e-6)


@pytest.mark.parametrize("dtype", DTYPES)
def test_each_row_counts_once(gpu, dtype):
    """dv of equal scores and an output gradient of one row: 1 / (keys it sees), to each key it sees."""
    nq, nk, G, D = 200, 330, 2, 64
    q = torch.zeros((nq, G, D), dtype=dtype, device="cuda")
    k = torch.zeros((nk, 1, D), dtype=dtype, device="cuda")
    v = torch.zeros_like(k)
    cq, ck = dev_cu([0, nq]), dev_cu([0, nk])
    out, lse, _ = gpu.dora_grouped_attn(q, k, v, cq, nq, cu_k=ck, causal=True)
    rows = [0, 15, 16, 31, 32, 63, 64, 65, 127, 128, 198, 199]
    dout = torch.zeros_like(q)
    for e, i in enumerate(rows):
        dout[i, e % G, e] = 1.0
    _, _, dv, _ = gpu.dora_grouped_attn_backward(dout, q, k, v, out, lse, cq, nq, cu_k=ck, causal=True)
    got = dv.double().cpu()[:, 0]
    for e, i in enumerate(rows):
        sees = i + 1 + nk - nq
        want = torch.where(torch.arange(nk) < sees, 1.0 / sees, 0.0).double()
        # P from a stored log: 2^(−lse log2 e), lse near 6, within 16 roundings of it; held in the inputs' type
        tol = want * (2 * ref.HALF[dtype] + 4 * ref.U * (8 + 16))
        assert bool(((got[:, e] - want).abs() <= tol).all()), i


@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(gpu, dtype):
    """Slices of one product, heads before rows, gradients as slices of one tensor; what lies between stays."""
    H, Hk, D, lens = 6, 2, 64, [65, 1, 130]
    t, cu, _ = make(lens, lens, H, Hk, D, dtype, 3)
    n = cu[-1]
    d = cuda(t)
    c = dev_cu(cu)
    out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], c, 130, causal=True)
    dq, dk, dv, _ = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, c, 130, causal=True)
    qkv = torch.full((n, H + 2 * Hk + 1, D), 7.0, dtype=dtype, device="cuda")
    qs, ks, vs = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:H + 2 * Hk]
    qs.copy_(d["q"]), ks.copy_(d["k"]), vs.copy_(d["v"])
    o2 = torch.empty((H, n, D), dtype=dtype, device="cuda").transpose(0, 1)
    _, lse2, _ = gpu.dora_grouped_attn(qs, ks, vs, c, 130, causal=True, out=o2)
    assert torch.equal(o2, out) and torch.equal(lse, lse2)
    g = torch.full_like(qkv, 9.0)
    gpu.dora_grouped_attn_backward(d["dout"].transpose(0, 1).contiguous().transpose(0, 1), qs, ks, vs, o2, lse, c, 130,
                                   causal=True, dq=g[:, :H], dk=g[:, H:H + Hk], dv=g[:, H + Hk:H + 2 * Hk])
    assert torch.equal(g[:, :H], dq) and torch.equal(g[:, H:H + Hk], dk) and torch.equal(g[:, H + Hk:-1], dv)
    assert bool((g[:, -1] == 9.0).all())
    # one key head read by all: an expanded view, and its gradient the sum over the views
    wide = d["k"][:, :1].expand(n, H, D)
    got, _, _ = gpu.dora_grouped_attn(d["q"], wide, wide, c, 130)
    want, _, _ = gpu.dora_grouped_attn(d["q"], d["k"][:, :1], d["k"][:, :1], c, 130)
    bound = ref.attention(t["q"], t["k"][:, :1], t["k"][:, :1], cu, cu, False)[1]["out"]
    ref.check(got, want.cpu().double(), 2 * bound, "expanded")


@pytest.mark.parametrize("dtype,split", itertools.product(DTYPES, (False, True)))
def test_rows_outside_are_left(gpu, dtype, split):
    """Rows before the first and behind the last sequence: not read (NaN there) and not written."""
    nq, nk, H, Hk, D = [1, 1, 1] if split else [40, 3, 70], [900, 600, 1000] if split else [80, 3, 70], 4, 2, 64
    t, cu_q, cu_k = make(nq, nk, H, Hk, D, dtype, 5)
    pad = 37

    def padded(x, fill):
        y = torch.full((x.shape[0] + 2 * pad, *x.shape[1:]), fill, dtype=dtype)
        y[pad:-pad] = x
        return y.cuda()
    d = {n: padded(x, float("nan")) for n, x in t.items()}
    cq, ck = dev_cu([c + pad for c in cu_q]), dev_cu([c + pad for c in cu_k])
    out = torch.full_like(d["q"], 5.0)
    lse = torch.full(out.shape[:2], 5.0, device="cuda")
    gpu.dora_grouped_attn(d["q"], d["k"], d["v"], cq, max(nq), cu_k=ck, causal=True, out=out, lse_out=lse)
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, True)
    ref.check(out[pad:-pad], want["out"], bound["out"], "out")
    grads = [torch.full_like(d[n], 5.0) for n in "qkv"]
    gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, cq, max(nq), cu_k=ck, causal=True,
                                   dq=grads[0], dk=grads[1], dv=grads[2])
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, True, dout=t["dout"], out=out[pad:-pad].cpu(),
                                lse=lse[pad:-pad].cpu())
    for n, x in zip(("dq", "dk", "dv"), grads):
        ref.check(x[pad:-pad], want[n], bound[n], n)
    for x in [out, lse, *grads]:
        assert bool((x[:pad] == 5.0).all()) and bool((x[-pad:] == 5.0).all())


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
def test_values_that_a_row_does_not_see(gpu, dtype, D):
    """A later token's NaN or infinity does not reach the rows before it, nor another sequence."""
    lens, H, Hk = [100, 90], 4, 2
    t, cu, _ = make(lens, lens, H, Hk, D, dtype, 6)
    clean, _ = ref.attention(t["q"], t["k"], t["v"], cu, cu, True)[0], None
    bound = ref.attention(t["q"], t["k"], t["v"], cu, cu, True)[1]
    at = 70
    t["k"][at, :, 3] = float("nan")
    t["v"][at, :, 1] = float("inf")
    t["v"][at + 5, 0] = float("nan")
    d = cuda(t)
    out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 100, causal=True)
    keep = torch.ones(cu[-1], dtype=torch.bool)
    keep[at:100] = False
    ref.check(out.cpu()[keep], clean["out"][keep], bound["out"][keep], "out")
    ref.check(lse.cpu()[keep], clean["lse"][keep], bound["lse"][keep], "lse")
    assert bool(torch.isnan(out[at:100]).any(dim=2).all())
    # values alone: the row that sees an infinite one has it, in that element only
    t, cu, _ = make(lens, lens, H, Hk, D, dtype, 6)
    t["v"][at, :, 1] = float("inf")
    d = cuda(t)
    out, _, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 100, causal=True)
    assert bool((out[at:100, :, 1] == float("inf")).all())
    rest = torch.arange(D) != 1
    ref.check(out.cpu()[:, :, rest], clean["out"][:, :, rest], bound["out"][:, :, rest], "other elements")
    # the backward pass keeps it in its sequence
    dout = d["dout"]
    out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 100, causal=True)
    grads = gpu.dora_grouped_attn_backward(dout, d["q"], d["k"], d["v"], out, lse, dev_cu(cu), 100, causal=True)[:3]
    for x in grads:
        assert bool(torch.isfinite(x[100:]).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_extreme_scores(gpu, dtype):
    """Scores hundreds apart and large, all equal to -inf, keys that are infinite."""
    H, Hk, D, lens = 2, 1, 64, [70, 33]
    t, cu, _ = make(lens, lens, H, Hk, D, dtype, 8, size=6.0)
    run_both(gpu, t, cu, cu, True, what="large")
    q = torch.ones((4, 1, D), dtype=dtype, device="cuda")
    k = torch.full((4, 1, D), -float("inf"), dtype=dtype, device="cuda")
    v = torch.ones((4, 1, D), dtype=dtype, device="cuda")
    k[3] = 1.0
    out, lse, _ = gpu.dora_grouped_attn(q, k, v, dev_cu([0, 4]), 4, causal=True)
    assert bool((out[:3] == 0).all()) and bool((lse[:3] == -float("inf")).all())
    assert bool((out[3] == 1).all()) and abs(float(lse[3]) - D ** 0.5) < 1e-5
    low = torch.finfo(dtype).min
    k = torch.zeros((4, 1, D), dtype=dtype, device="cuda")
    k[1:3, :, 0] = low                                        # a mask of the type's lowest value, added through the key
    v[:, 0, 0] = torch.tensor([1.0, 2.0, 4.0, 8.0], device="cuda").to(dtype)
    out, _, _ = gpu.dora_grouped_attn(q, k, v, dev_cu([0, 4]), 4, causal=True)
    want = torch.tensor([1.0, 1.0, 1.0, 4.5], device="cuda").to(dtype)
    assert bool((out[:, 0, 0] == want).all())


def test_bad_boundaries(gpu):
    """Reported; nothing is written outside, and the good sequences have their results."""
    H, Hk, D = 4, 2, 64
    t, cu, _ = make([40, 30, 20], [40, 30, 20], H, Hk, D, torch.float32, 9)
    d = cuda(t)
    good, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 40)
    for bad in ([0, 40, 70, 91], [0, 40, 30, 90], [-1, 40, 70, 90], [0, 40, 2 ** 31 - 1, 90], [50, 40, 70, 90]):
        out, _, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(bad), 90)
        assert int(st) == gpu.DORA_DEV_CU_SEQLENS, bad
        *_, st = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], good, lse, dev_cu(bad), 90)
        assert int(st) == gpu.DORA_DEV_CU_SEQLENS, bad
    out = torch.full_like(good, 5.0)
    _, _, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 35, out=out)     # the first is too long
    assert int(st) == gpu.DORA_DEV_CU_SEQLENS
    assert torch.equal(out[40:], good[40:]) and bool((out[:40] == 5.0).all())
    out = torch.full_like(good, 5.0)
    _, _, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 40, max_k=35, out=out)
    assert int(st) == gpu.DORA_DEV_CU_SEQLENS
    assert torch.equal(out[40:], good[40:]) and bool((out[:40] == 5.0).all())
    _, _, st = gpu.dora_grouped_attn(d["q"][:3], d["k"], d["v"], dev_cu([0, 1, 2, 3]), 1, cu_k=dev_cu([0, 95, 70, 90]))
    assert int(st) == gpu.DORA_DEV_CU_SEQLENS


def test_many_sequences(gpu):
    """More sequences than a wave's ballots take at once, most of them empty or tiny."""
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 4, (9000,), generator=g).tolist()
    lens[5000] = 200
    t, cu, _ = make(lens, lens, 2, 1, 32, torch.float32, 11)
    run_both(gpu, t, cu, cu, True, what="many")


@pytest.mark.parametrize("split", [False, True])
def test_far_rows(gpu, split):
    """Rows past 2^31 elements of a cache."""
    D, rows = 128, (1 << 24) + 200
    k = torch.zeros((rows, 1, D), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(2)
    n, nq = (3000, 1) if split else (150, 150)
    t = dict(q=torch.randn((nq, 1, D), generator=g).bfloat16(), k=torch.randn((n, 1, D), generator=g).bfloat16())
    k[rows - n:] = t["k"].cuda()
    cu_k = [rows - n, rows]
    out, lse, st = gpu.dora_grouped_attn(t["q"].cuda(), k, k, dev_cu([0, nq]), nq, cu_k=dev_cu(cu_k), causal=True)
    want, bound = ref.attention(t["q"], t["k"], t["k"], [0, nq], [0, n], True)
    assert int(st) == 0
    ref.check(out, want["out"], bound["out"], "out")


def test_repeats_streams_and_versions(gpu):
    """Bit for bit the same on every call, on another stream and in a reused workspace."""
    t, cu, _ = make([700, 30, 1200], [700, 30, 1200], 4, 1, 64, torch.bfloat16, 12)
    d, c = cuda(t), dev_cu(cu)
    ws = gpu.new_grouped_attn_workspace(3, 4, 1, 64, 1200, cu[-1], cu[-1], backward=True)
    first = None
    for i in range(3):
        stream = torch.cuda.Stream() if i == 1 else None
        torch.cuda.synchronize()
        out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], c, 1200, causal=True, workspace=ws, stream=stream)
        grads = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, c, 1200, causal=True,
                                               workspace=ws, stream=stream)
        torch.cuda.synchronize()
        now = [out, lse, *grads[:3]]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))
    before = out._version
    gpu.dora_grouped_attn(d["q"], d["k"], d["v"], c, 1200, causal=True, out=out)
    assert out._version > before


def test_no_rows(gpu):
    e = torch.empty((0, 4, 64), device="cuda")
    out, lse, st = gpu.dora_grouped_attn(e, e[:, :2], e[:, :2], dev_cu([0, 0]), 0)
    assert out.shape == (0, 4, 64) and int(st) == 0
    k = torch.randn((5, 2, 64), device="cuda")
    dk = torch.full_like(k, 5.0)
    dv = torch.full_like(k, 5.0)
    gpu.dora_grouped_attn_backward(e, e, k, k, out, lse, dev_cu([0, 0]), 0, cu_k=dev_cu([0, 5]), dk=dk, dv=dv)
    assert bool((dk == 0).all()) and bool((dv == 0).all())
    q = torch.randn((3, 4, 64), device="cuda")
    out, lse, _ = gpu.dora_grouped_attn(q, e[:, :2], e[:, :2], dev_cu([0, 3]), 3, cu_k=dev_cu([0, 0]))
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("causal,D", itertools.product((False, True), (64, 128)))
@pytest.mark.parametrize("H,Hk", [(3, 1), (10, 2), (7, 1), (12, 1), (48, 1), (64, 1), (20, 1), (33, 1)])
def test_group_sizes(gpu, causal, D, H, Hk):
    """Heads of a group that do not divide a tile of rows; more queries than keys and fewer, and parts of them."""
    for lens, keys in (([200, 0, 190, 260], [200, 5, 190, 260]), ([21, 22], [300, 200]), ([150, 1], [190, 182])):
        t, cu_q, cu_k = make(lens, keys, H, Hk, D, torch.bfloat16, 13 * H + D)
        run_both(gpu, t, cu_q, cu_k, causal, what=f"{lens} {keys}")
    if H in (3, 12):
        t, cu_q, cu_k = make([1500], [190], H, Hk, D, torch.bfloat16, 14 * H + D)
        run_both(gpu, t, cu_q, cu_k, causal, what="parts")


def test_group_rows_beyond(gpu):
    """One sequence's infinities stay out of another's gradients where a tile of rows ends before a wave's last."""
    lens, H, Hk, D = [180, 200], 5, 1, 64
    t, cu, _ = make(lens, lens, H, Hk, D, torch.bfloat16, 15)
    t["q"][179, :, 5] = float("inf")
    t["dout"][180 - 12, :, 1] = float("nan")
    d = cuda(t)
    out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), 200, causal=True)
    grads = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, dev_cu(cu), 200, causal=True)[:3]
    want, bound = ref.attention(t["q"][180:], t["k"][180:], t["v"][180:], [0, 200], [0, 200], True, None,
                                dout=t["dout"][180:], out=out[180:].cpu(), lse=lse[180:].cpu())
    for n, x in zip(("dq", "dk", "dv"), grads):
        ref.check(x[180:], want[n], bound[n], n)


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
@pytest.mark.parametrize("long", [False, True])
def test_one_key_has_no_gradient(gpu, dtype, D, long):
    """A row that sees one key has P 1 whatever its score: dq is 0 but for the roundings of fp32 sums, though the output
    that goes in is rounded to its type."""
    lens, H, Hk = [1, 1, 40, 1] + [300] * long, 4, 2
    t, cu, _ = make(lens, lens, H, Hk, D, dtype, 16)
    d = cuda(t)
    out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], dev_cu(cu), max(lens), causal=True)
    dq = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, dev_cu(cu), max(lens), causal=True)[0]
    u, c = 2.0 ** -24, D ** -0.5
    for i in cu[:-1]:                                           # first rows
        q, g = t["q"][i].double().abs(), t["dout"][i].double().abs()
        k, v = (t[n][i].double().abs().repeat_interleave(H // Hk, 0) for n in ("k", "v"))
        # P is 2 to a difference of two numbers of the score's size: roundings of the products' sum and of the two
        one = (D + 4) * u * c * (q * k).sum(1) + 8 * u * (1 + c * (q * k).sum(1))
        # dS = P (dP - delta), both sums of D products; its rounding, the product's and the result's come on top
        ds = (one + 2 * (D + 4) * u) * (g * v).sum(1)
        assert bool((dq[i].double().cpu().abs() <= 1.02 * c * ds[:, None] * k).all()), i
