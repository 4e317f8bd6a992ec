"""Gradients of grouped attention where dS should vanish or almost does: rows of one
key, few keys under large scores, and rows of many keys without allowance for out's
rounding, which their delta takes as it is given."""
import itertools

import pytest
import torch

import attn_grad_ref as tight
import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def cu_of(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def both_passes(gpu, nq, nk, H, Hk, D, dtype, causal, score, seed):
    """Inputs whose scores have a deviation of `score`, and what the two calls give."""
    g = torch.Generator().manual_seed(seed)
    cu_q, cu_k = cu_of(nq), cu_of(nk)

    def heads(n, h, size=1.0):
        return (size * torch.randn((n, h, D), generator=g)).to(dtype)
    t = dict(q=heads(cu_q[-1], H, score ** 0.5), k=heads(cu_k[-1], Hk, score ** 0.5), v=heads(cu_k[-1], Hk),
             dout=heads(cu_q[-1], H))
    d = {n: x.cuda() for n, x in t.items()}
    cq, ck = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in (cu_q, cu_k))
    kw = dict(cu_k=ck, causal=causal)
    out, lse, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], cq, max(nq), **kw)
    *grads, st2 = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, cq, max(nq), **kw)
    assert int(st) == 0 and int(st2) == 0
    return t, cu_q, cu_k, out.cpu(), lse.cpu(), dict(zip(("dq", "dk", "dv"), grads))


def compare(r, causal, few, what):
    t, cu_q, cu_k, out, lse, grads = r
    want, bound = tight.gradients(t["q"], t["k"], t["v"], t["dout"], out, lse, cu_q, cu_k, causal, few)
    for n in ("dq", "dk", "dv"):
        ref.check(grads[n], want[n], bound[n], f"{what} {n}")


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
@pytest.mark.parametrize("score", [1.0, 100.0, 1000.0])
@pytest.mark.parametrize("H,Hk", [(3, 3), (8, 1), (64, 1)])
def test_rows_of_one_key(gpu, dtype, D, score, H, Hk):
    """dq and the key's share of dk are 0, exactly: lone tokens, first rows of causal sequences, many queries of one key;
    between long sequences (the kernels of 128 rows and keys) and with the queries of a key in parts."""
    G = H // Hk
    for causal, nq, nk in ((False, [1] * 5, [1] * 5), (True, [1, 40, 1], [1, 40, 1]), (True, [1, 300, 1, 200], [1, 300, 1, 200]),
                           (False, [70, 5], [1, 1]), (True, [70, 5, 1], [1, 1, 1]), (False, [1, 1, 20], [1, 700, 1]),
                           (True, [50, 20], [30, 1]), (False, [6000 // G], [1])):
        t, cu_q, cu_k, out, lse, grads = both_passes(gpu, nq, nk, H, Hk, D, dtype, causal, score, H + D)
        what = f"{nq} {nk} causal {causal}"
        for b, (n, m) in enumerate(zip(nq, nk)):
            first = n - m if causal else 0              # the row that sees key 0 alone, or all of one key's rows
            rows = range(n) if m == 1 else [first] if causal and first >= 0 else []
            for i in rows:
                assert bool((grads["dq"][cu_q[b] + i] == 0).all()), (what, b, i)
            if m == 1:
                assert bool((grads["dk"][cu_k[b]] == 0).all()), (what, b)
                dout = t["dout"][cu_q[b] + (n - 1 if causal else 0):cu_q[b + 1]].double()
                want = dout.view(-1, Hk, G, D).sum((0, 2))
                # P within 2^-24 (D + 12) of c |q||k| and of lse of 1, held in the inputs' type; sums, the result's rounding
                size = (t["q"][cu_q[b]:cu_q[b + 1]].double().abs().view(n, Hk, G, D) *
                        t["k"][cu_k[b]].double().abs().view(1, Hk, 1, D)).sum(3).max() * D ** -0.5
                held = ref.HALF[dtype] if dtype == torch.bfloat16 else 0.0
                one = (D + 12) * ref.U * (1 + float(size)) + held + (n * G + 24) * ref.U
                bound = one * dout.abs().view(-1, Hk, G, D).sum((0, 2)) + ref.HALF[dtype] * want.abs()
                ref.check(grads["dv"][cu_k[b]], want, bound * 1.01, f"{what} {b} dv")


@pytest.mark.parametrize("dtype,D,causal", itertools.product(DTYPES, (32, 64, 128), (False, True)))
@pytest.mark.parametrize("score", [1.0, 30.0, 200.0])
def test_few_keys_under_large_scores(gpu, dtype, D, causal, score):
    few = dtype == torch.bfloat16
    for nq, nk, H, Hk in (([2, 2, 1], [2, 2, 2], 4, 2), ([16, 3], [16, 16], 4, 1), ([64, 33], [64, 64], 3, 3),
                          ([60, 64, 64], [1, 64, 50], 6, 2)):
        compare(both_passes(gpu, nq, nk, H, Hk, D, dtype, causal, score, 5 * H), causal, few, f"{nq} {nk} score {score}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("score", [1.0, 100.0])
def test_few_keys_in_the_wide_kernels(gpu, D, score):
    """Up to 128 keys of a tile are staged at once."""
    for nq, nk in (([300, 200], [100, 128]), ([290], [2])):
        compare(both_passes(gpu, nq, nk, 2, 1, D, torch.bfloat16, False, score, 7), False, True, f"{nq} {nk}")


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
@pytest.mark.parametrize("score", [1.0, 100.0])
def test_many_keys(gpu, dtype, D, score):
    """delta from out as it is given: nothing is allowed for out's rounding."""
    for nq, nk, H, Hk in (([40, 70], [129, 200], 4, 2), ([300, 150], [300, 150], 2, 1), ([3], [1500], 2, 1)):
        compare(both_passes(gpu, nq, nk, H, Hk, D, dtype, False, score, 9), False, False, f"{nq} {nk}")
