"""Infinite values under weights of 0: a row that sees one has p times it, NaN where p
has underflowed to 0 and infinity above that, whichever tile the key stands in and
whichever kernel takes the row."""
import itertools
import math

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
@pytest.mark.parametrize("nq,nk", [(300, 300), (150, 150), (40, 40), (1, 700), (3, 2500), (130, 2100), (20, 90)])
def test_infinite_values(gpu, dtype, D, nq, nk):
    H, Hk = 4, 2
    g = torch.Generator().manual_seed(D + nq)
    q, k, v = (torch.randn((n, h, D), generator=g).to(dtype) for n, h in ((nq, H), (nk, Hk), (nk, Hk)))
    q[..., 0], k[..., 0] = 16.0, 0.0
    first = nk - nq                                     # keys that every row sees
    for bits, j in itertools.product((300.0, 90.0), (5, 63, 64, 100, 140, nk - 3, nk - 1)):
        if not 0 < j < nk:
            continue
        # key j's score lies about this many bits below the others, whose scores are a few bits: p 2^-300 is 0, 2^-90 is not
        kj = k.clone()
        kj[j, :, 0] = -bits * math.log(2) * math.sqrt(D) / 16.0
        want, bound = ref.attention(q, kj, v, [0, nq], [0, nk], True)
        vj = v.clone()
        vj[j, :, 1], vj[j, :, 2], vj[j, :, 9] = math.inf, -math.inf, math.nan
        cu = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (nq, nk)]
        out, lse, st = gpu.dora_grouped_attn(q.cuda(), kj.cuda(), vj.cuda(), cu[0], nq, cu_k=cu[1], causal=True)
        assert int(st) == 0
        out, what = out.cpu(), (bits, j)
        seen = max(0, j - first)                        # the first row that sees key j
        odd = torch.zeros(D, dtype=torch.bool)
        odd[[1, 2, 9]] = True
        ref.check(out[:seen], want["out"][:seen], bound["out"][:seen], f"{what} rows before")
        ref.check(out[..., ~odd], want["out"][..., ~odd], bound["out"][..., ~odd], f"{what} other elements")
        ref.check(lse, want["lse"], bound["lse"], f"{what} lse")
        assert bool(torch.isnan(out[seen:, :, 9]).all()), what
        for e, x in ((1, math.inf), (2, -math.inf)):
            got = out[seen:, :, e]
            assert bool((torch.isnan(got) if bits == 300.0 else got == x).all()), (what, e)
