"""Grouped attention over batches of more sequences than a wave holds boundaries of,
and of none: the order of tiles, the parts of keys and of rows, and what joins them."""
import itertools

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_queries_against_a_cache(gpu, dtype):
    """Nothing to do, and nothing refused: with the workspace that the call makes and with a given one."""
    cu = [torch.tensor(c, dtype=torch.int32, device="cuda") for c in ([0, 0], [0, 5])]
    q = torch.empty((0, 4, 64), dtype=dtype, device="cuda")
    k = torch.randn((5, 2, 64), device="cuda").to(dtype)
    ws = gpu.new_grouped_attn_workspace(1, 4, 2, 64, 0, 0, 5, backward=True)
    for workspace in (None, ws):
        out, lse, st = gpu.dora_grouped_attn(q, k, k, cu[0], 0, cu_k=cu[1], workspace=workspace)
        assert out.shape == (0, 4, 64) and lse.shape == (0, 4) and int(st) == 0
        dq, dk, dv, st = gpu.dora_grouped_attn_backward(q, q, k, k, out, lse, cu[0], 0, cu_k=cu[1], workspace=workspace)
        assert int(st) == 0 and dq.shape == (0, 4, 64) and bool((dk == 0).all()) and bool((dv == 0).all())
    # every sequence longer than it was said to be: reported and skipped
    q = torch.randn((6, 4, 64), device="cuda").to(dtype)
    out = torch.full_like(q, 5.0)
    cq, ck = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in ([0, 2, 4, 6], [0, 3, 4, 5]))
    _, _, st = gpu.dora_grouped_attn(q, k, k, cq, 0, cu_k=ck, out=out)
    assert int(st) == gpu.DORA_DEV_CU_SEQLENS and bool((out == 5.0).all())


def cu_of(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def make(nq, nk, H, Hk, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    cu_q, cu_k = cu_of(nq), cu_of(nk)
    t = {n: torch.randn((c[-1], h, D), generator=g).to(dtype) for n, c, h in (("q", cu_q, H), ("k", cu_k, Hk), ("v", cu_k, Hk),
                                                                               ("dout", cu_q, H))}
    return t, cu_q, cu_k


def forward(gpu, t, cu_q, cu_k, max_q, causal, what, **kw):
    d = {n: x.cuda() for n, x in t.items()}
    cq, ck = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in (cu_q, cu_k))
    out, lse, st = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], cq, max_q, cu_k=ck, causal=causal, **kw)
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal)
    assert int(st) == 0
    ref.check(out, want["out"], bound["out"], what + " out")
    ref.check(lse, want["lse"], bound["lse"], what + " lse")
    return d, cq, ck, out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [0, 300, 500])
def test_one_long_list_among_short_ones(gpu, dtype, at):
    """501 new tokens, one with 60000 keys, the others with one or none; the longest known and not."""
    nk = [1 if i % 7 else 0 for i in range(501)]
    nk[at] = 60000
    t, cu_q, cu_k = make([1] * 501, nk, 4, 2, 64, dtype, at)
    for max_k in (0, 60000):
        forward(gpu, t, cu_q, cu_k, 1, True, f"longest {max_k}", max_k=max_k)


def both(gpu, nq, nk, H, Hk, D, dtype, causal, seed, what):
    t, cu_q, cu_k = make(nq, nk, H, Hk, D, dtype, seed)
    d, cq, ck, out, lse = forward(gpu, t, cu_q, cu_k, max(nq), causal, what)
    *grads, st = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, cq, max(nq), cu_k=ck, causal=causal)
    assert int(st) == 0
    want, bound = ref.attention(t["q"], t["k"], t["v"], cu_q, cu_k, causal, dout=t["dout"], out=out.cpu(), lse=lse.cpu())
    for n, x in zip(("dq", "dk", "dv"), grads):
        ref.check(x, want[n], bound[n], f"{what} {n}")


def lengths(B, lo, hi, seed, empty=9):
    """B lengths, tiles' own among them (one with a number of tiles that holds none beside it), every `empty`th 0."""
    g = torch.Generator().manual_seed(seed)
    n = torch.randint(lo, hi + 1, (B,), generator=g)
    n[::5] = 64 if lo <= 64 <= hi else hi
    n[1::7] = min(128, hi)
    n[empty - 1::empty] = 0
    return n.tolist()


# sequences on both sides of a wave's 64 boundaries, of about one tile to four (whose numbers are turned), of the kernels of 64
# and of 128 rows and keys
@pytest.mark.parametrize("B", [63, 64, 65, 130])
@pytest.mark.parametrize("dtype,D,lo,hi,causal", [(torch.bfloat16, 64, 20, 64, True), (torch.bfloat16, 64, 40, 140, False),
                                                  (torch.bfloat16, 64, 150, 260, True), (torch.bfloat16, 128, 30, 128, True),
                                                  (torch.bfloat16, 128, 90, 200, False), (torch.bfloat16, 32, 40, 140, True),
                                                  (torch.float32, 32, 40, 140, False), (torch.float32, 64, 30, 100, True)])
def test_many_sequences(gpu, B, dtype, D, lo, hi, causal):
    lens = lengths(B, lo, hi, B + hi)
    both(gpu, lens, lens, 2, 1 if hi < 150 else 2, D, dtype, causal, B, f"{B}")


@pytest.mark.parametrize("B", [64, 66])
@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (64, 128)))
def test_own_boundaries_of_many(gpu, B, dtype, D):
    """Queries without keys, keys without queries, more of either, rows that see nothing."""
    both(gpu, lengths(B, 1, 150, 1, 8), lengths(B, 1, 190, 2, 11), 3, 1, D, dtype, True, B, "causal")
    both(gpu, lengths(B, 1, 70, 3, 8), lengths(B, 100, 250, 4, 11), 2, 2, D, dtype, False, B, "full")


@pytest.mark.parametrize("B", [63, 64, 65, 130])
@pytest.mark.parametrize("dtype,D,nq", [(torch.bfloat16, 128, 1), (torch.bfloat16, 64, 3), (torch.float32, 32, 1)])
def test_new_tokens_of_many(gpu, B, dtype, D, nq):
    """Their lists of keys in parts and joined: longer and shorter than a part, a part exactly, none; the longest known too."""
    nk = lengths(B, 1, 900, B, 10)
    nk[::13], nk[2::17] = [2000] * len(nk[::13]), [192] * len(nk[2::17])
    t, cu_q, cu_k = make([nq] * B, nk, 4, 2, D, dtype, B)
    for max_k in (0, 2000):
        forward(gpu, t, cu_q, cu_k, nq, True, f"longest {max_k}", max_k=max_k)


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (32, 64, 128)))
def test_parts_of_rows_of_many(gpu, dtype, D):
    """More than 64 sequences of few keys and many rows: dk and dv in parts of rows, joined."""
    B = 66
    nk = lengths(B, 1, 12, 5, 9)
    both(gpu, [130] * B, nk, 8, 1, D, dtype, False, 6, "parts of rows")


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (64, 128)))
def test_parts_of_keys_of_many(gpu, dtype, D):
    """More than 64 sequences of several tiles of rows and long lists of keys: the tiles' keys in parts, joined."""
    B = 66
    nq = lengths(B, 1, 70, 7, 9)
    nk = [n + 1100 for n in lengths(B, 1, 100, 8, 9)]
    nk[3], nk[11] = 0, 70
    t, cu_q, cu_k = make(nq, nk, 1, 1, D, dtype, 9)
    forward(gpu, t, cu_q, cu_k, max(nq), True, "parts of keys")


@pytest.mark.parametrize("dtype,D", itertools.product(DTYPES, (64, 128)))
def test_heads_before_rows(gpu, dtype, D):
    """q, k, v and their gradients as slices of [H, T, 3 D] tensors of thousands of rows: bit for bit the packed ones' results."""
    H, lens = 3, [1500, 0, 700, 33]
    t, cu, _ = make(lens, lens, H, H, D, dtype, 10)
    d = {n: x.cuda() for n, x in t.items()}
    c = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out, lse, _ = gpu.dora_grouped_attn(d["q"], d["k"], d["v"], c, 1500, causal=True)
    grads = gpu.dora_grouped_attn_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, c, 1500, causal=True)[:3]

    def slices(x):
        return [x[:, :, i * D:(i + 1) * D].transpose(0, 1) for i in range(3)]
    qkv = slices(torch.full((H, cu[-1], 3 * D), 7.0, dtype=dtype, device="cuda"))
    for x, n in zip(qkv, "qkv"):
        x.copy_(d[n])
    out2, lse2, _ = gpu.dora_grouped_attn(*qkv, c, 1500, causal=True)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    into = slices(torch.full((H, cu[-1], 3 * D), 9.0, dtype=dtype, device="cuda"))
    gpu.dora_grouped_attn_backward(d["dout"], *qkv, out, lse, c, 1500, causal=True, dq=into[0], dk=into[1], dv=into[2])
    for x, want in zip(into, grads):
        assert torch.equal(x, want)
