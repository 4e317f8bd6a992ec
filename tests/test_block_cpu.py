"""The block operators' refusals, and which descriptions share memory, on the host:
no call below reaches the GPU."""
import ctypes
import os
import random
import re
import subprocess

import pytest
import torch

import paper_2609_34325_amd as dora
from paper_2609_34325_amd import build

A = 0x10000000          # never dereferenced: every call below is refused
OK_SIZES = dict(T=6, H=4, Hk=2, D=64)


def rows(at, n=6, heads=4, dim=64, row=None, head=None, dtype=dora.DORA_BF16):
    head = dim if head is None else head
    return dora.Rows(at, n, heads, dim, heads * dim if row is None else row, head, dtype, 0)


class Names(dict):
    """Descriptions and addresses far apart; refused calls name what differs."""

    def ref(self, n):
        t = self[n]
        return None if t is None else ctypes.byref(t) if isinstance(t, dora.Rows) else t


def rope(axes=1, R=64, inter=0, inv=0, scale=1.0, **kw):
    a = Names(q=rows(A), k=rows(A + (1 << 24), heads=2), pos=A + (2 << 24), freq=A + (3 << 24), qo=rows(A + (4 << 24)),
              ko=rows(A + (5 << 24), heads=2))
    a.update(kw)
    return dora.load_library().dora_rope(a.ref("q"), a.ref("k"), a["pos"], axes, a["freq"], R, inter, inv, scale, a.ref("qo"),
                                         a.ref("ko"), None)


def test_rope_refusals():
    for n in ("q", "qo", "ko", "pos", "freq"):
        assert rope(**{n: None}) == dora.DORA_ERR_NULL, n
    for kw in (dict(R=0), dict(R=7), dict(R=66), dict(R=-2), dict(axes=0), dict(axes=5), dict(axes=3, R=64), dict(axes=2, R=62),
               dict(q=rows(A, dim=2048), qo=rows(A + (4 << 24), dim=2048), k=None, ko=None), dict(q=rows(A, n=7)),
               dict(qo=rows(A + (4 << 24), heads=3)), dict(k=rows(A + (1 << 24), heads=2, dim=32)), dict(q=rows(A, row=-1)),
               dict(q=rows(A, heads=0)), dict(qo=rows(A + (4 << 24), dtype=dora.DORA_F32))):
        assert rope(**kw) == dora.DORA_ERR_SHAPE, kw
    assert rope(q=rows(A, dtype=5)) == dora.DORA_ERR_DTYPE
    assert rope(q=rows(A + 1)) == dora.DORA_ERR_ALIGN
    assert rope(pos=A + (2 << 24) + 2) == dora.DORA_ERR_ALIGN
    assert rope(freq=A + (3 << 24) + 4) == dora.DORA_ERR_ALIGN
    assert rope(q=rows(None)) == dora.DORA_ERR_NULL
    over = dict(qo=rows(A + 2), q=rows(A))
    assert rope(**over) == dora.DORA_ERR_OVERLAP                                     # shifted by an element
    assert rope(qo=rows(A, row=300)) == dora.DORA_ERR_OVERLAP                        # other strides
    assert rope(qo=rows(A + (1 << 24))) == dora.DORA_ERR_OVERLAP                     # over k
    assert rope(ko=rows(A, heads=2, row=256)) == dora.DORA_ERR_OVERLAP               # over q
    assert rope(qo=rows(A + (5 << 24))) == dora.DORA_ERR_OVERLAP                     # over k's output
    assert rope(qo=rows(A + (2 << 24) + 20)) == dora.DORA_ERR_OVERLAP                # the last position
    assert rope(qo=rows(A + (3 << 24) - 2 * 6 * 256 + 2)) == dora.DORA_ERR_OVERLAP   # the first angle
    assert rope(qo=rows(A + (4 << 24), head=0)) == dora.DORA_ERR_OVERLAP             # an output over itself
    assert rope(qo=rows(A + (4 << 24), row=100)) == dora.DORA_ERR_OVERLAP


def attn_names(dtype=dora.DORA_BF16, n=6, m=9, H=4, Hk=2, D=64):
    big = 1 << 28
    r = lambda i, n, h: rows(A + i * big, n=n, heads=h, dim=D, dtype=dtype)  # noqa: E731
    return Names(q=r(0, n, H), k=r(1, m, Hk), v=r(2, m, Hk), cq=A + 3 * big, ck=A + 4 * big, out=r(5, n, H), lse=A + 6 * big,
                 ws=A + 7 * big, st=A + 8 * big, dout=r(9, n, H), dq=r(10, n, H), dk=r(11, m, Hk), dv=r(12, m, Hk))


def attn(a, B=2, max_q=5, causal=1, scale=0.0, ws_bytes=1 << 27, max_k=0):
    return dora.load_library().dora_grouped_attn(a.ref("q"), a.ref("k"), a.ref("v"), a["cq"], a["ck"], B, max_q, max_k, causal,
                                                 scale, a.ref("out"), a["lse"], a["ws"], ws_bytes, a["st"], None)


def attn_grad(a, B=2, max_q=5, causal=1, scale=0.0, ws_bytes=1 << 27):
    return dora.load_library().dora_grouped_attn_backward(
        a.ref("dout"), a.ref("q"), a.ref("k"), a.ref("v"), a.ref("out"), a["lse"], a["cq"], a["ck"], B, max_q, causal, scale,
        a.ref("dq"), a.ref("dk"), a.ref("dv"), a["ws"], ws_bytes, a["st"], None)


@pytest.mark.parametrize("call", [attn, attn_grad])
def test_attention_refusals(call):
    def bad(code, *args, **kw):
        a = attn_names()
        names = {n: v for n, v in kw.items() if n in a}
        a.update(names)
        assert call(a, **{n: v for n, v in kw.items() if n not in a}) == code, kw

    for n in ("q", "k", "v", "cq", "ck", "out", "st") + (() if call is attn else ("dout", "lse", "dq", "dk", "dv")):
        bad(dora.DORA_ERR_NULL, **{n: None})
    bad(dora.DORA_ERR_WORKSPACE, ws=None)
    bad(dora.DORA_ERR_WORKSPACE, ws=A + 7 * (1 << 28) + 16)
    bad(dora.DORA_ERR_WORKSPACE, ws_bytes=0)
    big = 1 << 28
    for kw in (dict(B=0), dict(B=dora.DORA_MAX_SEQUENCES + 1), dict(max_q=-1), dict(scale=float("inf")), dict(scale=float("nan")),
               dict(k=rows(A + big, n=9, heads=3), v=rows(A + 2 * big, n=9, heads=3)), dict(v=rows(A + 2 * big, n=8, heads=2)),
               dict(q=rows(A, dim=32)), dict(out=rows(A + 5 * big, n=5)), dict(out=rows(A + 5 * big, heads=2))):
        bad(dora.DORA_ERR_SHAPE, **kw)
    if call is attn:
        bad(dora.DORA_ERR_SHAPE, max_k=-1)
    for D in (16, 96, 256):
        a = attn_names(D=D)
        assert call(a) == dora.DORA_ERR_SHAPE
    a = attn_names(H=512, Hk=2)
    assert call(a) == dora.DORA_ERR_SHAPE
    bad(dora.DORA_ERR_DTYPE, q=rows(A, dtype=7))
    bad(dora.DORA_ERR_DTYPE, q=rows(A, dtype=dora.DORA_F32))
    bad(dora.DORA_ERR_ALIGN, q=rows(A + 8))
    bad(dora.DORA_ERR_ALIGN, k=rows(A + big, n=9, heads=2, row=132))
    bad(dora.DORA_ERR_ALIGN, out=rows(A + 5 * big, head=68, row=288))
    outs = {"out": rows, "lse": None, "ws": None, "st": None} if call is attn else {"dq": rows, "dk": rows, "dv": rows, "ws": None,
                                                                                 "st": None}
    at = {n: i * big for i, n in enumerate(("q", "k", "v", "cq", "ck", "out", "lse", "ws", "st", "dout", "dq", "dk", "dv"))}
    reads = [n for n in ("q", "k", "v", "cq", "ck") + (() if call is attn else ("dout", "out", "lse"))]
    for o, make in outs.items():
        for other in list(outs) + reads:
            if other == o or (call is attn and other in ("dout",)):
                continue
            heads, n = (2, 9) if o in ("dk", "dv") else (4, 6)
            a = attn_names()
            a[o] = rows(A + at[other], n=n, heads=heads) if make else A + at[other]
            assert call(a) == dora.DORA_ERR_OVERLAP, (o, other)
    lib = dora.load_library()
    sizes = (2, 4, 2, 64, 5, 6, 9)
    need = (lib.dora_grouped_attn_workspace_size if call is attn else lib.dora_grouped_attn_backward_workspace_size)
    assert need(*sizes) > 0
    bad(dora.DORA_ERR_WORKSPACE, ws_bytes=need(*sizes) - 1)
    for i, v in ((0, 0), (1, 0), (1, 257), (2, 0), (2, 3), (3, 48), (4, -1), (5, -1), (6, -1), (5, 1 << 31)):
        assert need(*sizes[:i], v, *sizes[i + 1:]) == 0, (i, v)


def test_gradient_slices_are_apart():
    """dq, dk and dv as slices of one tensor are refused for nothing but the workspace that comes after."""
    a = attn_names()
    at = A + 10 * (1 << 28)
    for n, lo, heads in (("dq", 0, 4), ("dk", 4, 2), ("dv", 6, 2)):
        a[n] = rows(at + lo * 64 * 2, n=6, heads=heads, row=8 * 64)
    for n in ("k", "v"):
        a[n] = rows(a[n].data, n=6, heads=2)
    assert attn_grad(a, ws_bytes=0) == dora.DORA_ERR_WORKSPACE
    a["ws"] = at - 256                     # and what lies in front of them is too
    assert attn_grad(a) == dora.DORA_ERR_OVERLAP


def norm(kind=0, eps=1e-6, **kw):
    big = 1 << 24
    a = Names({n: rows(A + i * big, heads=1) for i, n in enumerate(("x", "a", "h", "y"))})
    a.update({n: A + (i + 8) * big for i, n in enumerate(("gamma", "beta", "scale", "gate", "pg", "pb"))})
    a.update(kw)
    return dora.load_library().dora_residual_norm(a.ref("x"), a.ref("a"), *(a[n] for n in ("gamma", "beta", "scale", "gate", "pg", "pb")),
                                                  kind, eps, a.ref("h"), a.ref("y"), None)


def norm_grad(kind=0, eps=1e-6, ws_bytes=1 << 23, **kw):
    big = 1 << 24
    a = Names({n: rows(A + i * big, heads=1) for i, n in enumerate(("dy", "dh", "h", "a", "dx", "da"))})
    a.update({n: A + (i + 8) * big for i, n in enumerate(("gamma", "scale", "gate", "pg", "pb"))})
    outs = ("dgamma", "dbeta", "dscale", "dgate", "dpg", "dpb")
    a.update({n: A + (i + 16) * big for i, n in enumerate(outs + ("ws",))})
    a.update(kw)
    return dora.load_library().dora_residual_norm_backward(
        *(a.ref(n) for n in ("dy", "dh", "h", "a")), *(a[n] for n in ("gamma", "scale", "gate", "pg", "pb")), kind, eps,
        a.ref("dx"), a.ref("da"), *(a[n] for n in outs), a["ws"], ws_bytes, None)


def test_norm_refusals():
    big = 1 << 24
    for n in ("x", "y", "gamma", "h"):
        assert norm(**{n: None}) == dora.DORA_ERR_NULL, n
    for n in ("h", "dx", "gamma"):
        assert norm_grad(**{n: None}) == dora.DORA_ERR_NULL, n
    assert norm_grad(dy=None, dh=None) == dora.DORA_ERR_NULL
    wide = dict(n=6, heads=1, dim=8200)
    for kw in (dict(kind=2), dict(eps=-1.0), dict(eps=float("nan")), dict(a=rows(A + big, heads=1, n=5)),
               dict(h=rows(A + 2 * big, heads=1, dim=56))):
        assert norm(**kw) == dora.DORA_ERR_SHAPE, kw
    assert norm(x=rows(A, **wide), a=rows(A + big, **wide), h=rows(A + 2 * big, **wide), y=rows(A + 3 * big, **wide)) == dora.DORA_ERR_SHAPE
    assert norm(x=rows(A, heads=2), a=None, scale=None, gate=None, pg=None, pb=None) == dora.DORA_ERR_SHAPE
    odd = dict(n=6, heads=1, dim=60, row=64)
    assert norm(x=rows(A, **odd), a=rows(A + big, **odd), h=rows(A + 2 * big, **odd), y=rows(A + 3 * big, **odd)) == dora.DORA_ERR_SHAPE
    assert norm(x=rows(A, heads=1, dtype=9)) == dora.DORA_ERR_DTYPE
    assert norm(a=rows(A + big, heads=1, dtype=dora.DORA_F32)) == dora.DORA_ERR_DTYPE
    assert norm(x=rows(A + 8, heads=1)) == dora.DORA_ERR_ALIGN
    assert norm(a=rows(A + big, heads=1, row=68)) == dora.DORA_ERR_ALIGN
    for n in ("scale", "gate", "pg", "pb"):
        rest = {m: None for m in ("scale", "gate", "pg", "pb") if m != n}
        assert norm(a=None, **rest) == dora.DORA_ERR_UNSUPPORTED, n
        assert norm_grad(a=None, da=None, **rest) == dora.DORA_ERR_UNSUPPORTED, n
    assert norm(pg=None) == dora.DORA_ERR_UNSUPPORTED
    for n, of in (("dscale", "scale"), ("dgate", "gate")):
        assert norm_grad(**{of: None}) == dora.DORA_ERR_UNSUPPORTED, n
    assert norm_grad(a=None, scale=None, gate=None, pg=None, pb=None) == dora.DORA_ERR_UNSUPPORTED   # da without a
    assert norm_grad(ws=None) == dora.DORA_ERR_WORKSPACE
    assert norm_grad(ws_bytes=dora.dora_residual_norm_workspace_size(6, 64) - 1) == dora.DORA_ERR_WORKSPACE
    assert dora.dora_residual_norm_workspace_size(-1, 64) == dora.dora_residual_norm_workspace_size(6, 0) == 0
    assert dora.dora_residual_norm_workspace_size(6, 8193) == 0 and dora.dora_residual_norm_workspace_size(0, 8192) > 0


def test_norm_overlaps():
    big = 1 << 24
    vectors = {n: A + (i + 8) * big for i, n in enumerate(("gamma", "beta", "scale", "gate", "pg", "pb"))}
    for o in ("h", "y"):
        for n in ("x", "a"):
            assert norm(**{o: rows(A + (0 if n == "x" else 1) * big + 128, heads=1)}) == dora.DORA_ERR_OVERLAP   # a row later
        for n, at in vectors.items():
            assert norm(**{o: rows(at, heads=1)}) == dora.DORA_ERR_OVERLAP, (o, n)
    assert norm(h=rows(A + 3 * big, heads=1)) == dora.DORA_ERR_OVERLAP
    assert norm(h=rows(A + 2 * big, heads=1, row=0)) == dora.DORA_ERR_OVERLAP
    outs = ("dgamma", "dbeta", "dscale", "dgate", "dpg", "dpb", "ws")
    for i, o in enumerate(outs):
        for at in list(range(6)) + list(range(8, 13)) + [16 + j for j in range(7) if j != i]:
            assert norm_grad(**{o: A + at * big}) == dora.DORA_ERR_OVERLAP, (o, at)
    assert norm_grad(dx=rows(A + 5 * big, heads=1)) == dora.DORA_ERR_OVERLAP
    assert norm_grad(dx=rows(A + 2 * big, heads=1, row=128)) == dora.DORA_ERR_OVERLAP


PROBE = """
#include "grouped_attn_split.h"
#include "rows.h"
extern "C" int pair(const dora_rows* s, const dora_rows* t) { return dora::rows_meet(s, t); }
extern "C" int vector(const dora_rows* s, void* p, size_t n) { return dora::rows_meet(s, dora::Extent(p, n)); }
extern "C" int itself(const dora_rows* s) { return dora::meets_itself(s); }
// Bytes that a forward call's parts take beyond those of the workspace that any call of its sizes has to bring.
extern "C" long beyond(int B, int H, int Hk, int D, int max_q, long total_q, long total_k, int max_k) {
  const dora::Sizes z{B, H, Hk, D, max_q, total_q, total_k};
  const dora::Split p = dora::forward_split(z, max_k);
  if (p.splits == 1 && !p.chunk) return 0;
  return p.blocks * Hk * p.part_rows * (D + 2) * 4L - static_cast<long>(dora::forward_bytes(z));
}
"""


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    """The overlap checks as host code of their own."""
    d = tmp_path_factory.mktemp("probe")
    (d / "probe.hip").write_text(PROBE)
    so = str(d / "probe.so")
    subprocess.run([build.hipcc(), "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", build.INCLUDE, "-I",
                    build.CSRC, str(d / "probe.hip"), "-o", so], check=True, capture_output=True, timeout=300)
    return ctypes.CDLL(so)


def places(t):
    return [(t.data - A) // 4 + r * t.row_stride + h * t.head_stride + d for r in range(t.rows) for h in range(t.heads)
            for d in range(t.dim)]


def some_rows(rng, at):
    dim, heads, n = rng.choice((1, 2, 4)), rng.randint(1, 3), rng.randint(1, 4)
    hs = dim + rng.choice((0, 0, 2, 2 * dim))
    row = (heads - 1) * hs + dim + rng.choice((0, 0, 2, 7, 12, 20))
    if rng.random() < 0.3:      # heads before rows
        row = dim + rng.choice((0, 0, 3))
        hs = (n - 1) * row + dim + rng.choice((0, 5, 15))
    return rows(A + 4 * at, n, heads, dim, row, hs, dora.DORA_F32)


def test_overlap_against_every_element(probe):
    """Descriptions at random places and strides.  What shares an element is found; what shares none is told apart
    where the rows are the same distance apart, or one lies wholly before the other."""
    rng = random.Random(7)
    shared = apart = unsure = 0
    for _ in range(20000):
        s, t = some_rows(rng, 0), some_rows(rng, rng.randint(-60, 60))
        if rng.random() < 0.7:
            t.row_stride, t.head_stride = s.row_stride, s.head_stride
            t.rows, t.heads, t.dim = s.rows, rng.randint(1, s.heads), s.dim
        a, b = places(s), places(t)
        if len(set(b)) < len(b) or len(set(a)) < len(a):
            continue
        got = bool(probe.pair(ctypes.byref(s), ctypes.byref(t)))
        assert got == bool(probe.pair(ctypes.byref(t), ctypes.byref(s)))
        if set(a) & set(b):
            assert got
            shared += 1
        elif max(a) < min(b) or max(b) < min(a):
            assert not got
            apart += 1
        else:
            alike = (s.rows, s.row_stride, s.head_stride, s.dim) == (t.rows, t.row_stride, t.head_stride, t.dim)
            order = (s.row_stride < s.head_stride) and s.heads > 1 and t.heads == 1 and s.rows > 1
            assert not got or not alike or order
            unsure += 1
    assert shared > 3000 and apart > 1000 and unsure > 1000


def test_vector_overlap_against_every_element(probe):
    rng = random.Random(8)
    shared = apart = 0
    for _ in range(20000):
        s, at, n = some_rows(rng, 0), rng.randint(-20, 80), rng.randint(1, 12)
        a = places(s)
        if len(set(a)) < len(a):
            continue
        want = bool(set(a) & set(range(at, at + n)))
        assert bool(probe.vector(ctypes.byref(s), ctypes.c_void_p(A + 4 * at), ctypes.c_size_t(4 * n))) == want
        shared, apart = shared + want, apart + (not want)
    assert shared > 3000 and apart > 3000


def test_outputs_over_themselves(probe):
    rng = random.Random(9)
    for _ in range(5000):
        s = some_rows(rng, 0)
        if rng.random() < 0.5:
            s.row_stride = rng.randint(0, 8)
        if rng.random() < 0.5:
            s.head_stride = rng.randint(0, 8)
        a = places(s)
        if len(set(a)) < len(a):
            assert probe.itself(ctypes.byref(s)), (s.rows, s.heads, s.dim, s.row_stride, s.head_stride)


def test_parts_fit_the_workspace(probe):
    """Whatever a call says of its longest sequence (right or not), its parts lie in the workspace of its sizes."""
    probe.beyond.argtypes = [ctypes.c_int] * 5 + [ctypes.c_long] * 2 + [ctypes.c_int]
    probe.beyond.restype = ctypes.c_long
    # sequences that stay whole and have keys enough for tiles' parts: about 500 of them and a little over 1024 keys
    # each, then a longest sequence said to be shorter than the average
    assert probe.beyond(250, 2, 2, 64, 1, 250, 250 * 1050, 1050) <= 0
    assert probe.beyond(4, 8, 8, 64, 1, 4, 4 * 100000, 128) <= 0
    rng = random.Random(10)
    log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())  # noqa: E731
    for _ in range(200000):
        Hk, D = log(1, 32), rng.choice((32, 64, 128))
        B, H, keys, max_q = log(1, 2000), Hk * rng.choice((1, 2, 4, 5, 8)), log(1, 20000), log(1, 300)
        total_q, total_k = B * min(max_q, log(1, 300)), min(B * keys + rng.randint(0, B), 0x7FFF0000)
        max_k = rng.choice((0, keys + 1, keys * 2, log(1, 5000)))
        assert probe.beyond(B, H, Hk, D, max_q, total_q, total_k, max_k) <= 0, (B, H, Hk, D, max_q, total_q, total_k, max_k)


def test_binding_refusals():
    q = torch.zeros((4, 2, 64))
    pos, freq = torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        dora.dora_rope(q, pos, freq)
    with pytest.raises(ValueError, match="rows, heads, dim"):
        dora.dora_rope(q[:, 0], pos, freq)
    with pytest.raises(TypeError, match="freq must be torch.float64"):
        dora.dora_rope(q, pos, freq.float())
    with pytest.raises(TypeError, match="positions must be a torch tensor"):
        dora.dora_rope(q, [0, 1, 2, 3], freq)
    with pytest.raises(ValueError, match="positions must be"):
        dora.dora_rope(q, pos[:3], freq)
    with pytest.raises(ValueError, match="goes with k"):
        dora.dora_rope(q, pos, freq, k_out=q)
    with pytest.raises(ValueError, match="on the GPU"):
        dora.dora_grouped_attn(q, q, q, cu, 4, workspace=torch.zeros(1 << 20, dtype=torch.uint8), dev_status=cu)
    with pytest.raises(ValueError, match="lse_out"):
        dora.dora_grouped_attn(q, q, q, cu, 4, lse_out=torch.zeros(3), dev_status=cu)
    with pytest.raises(ValueError, match="cu_q"):
        dora.dora_grouped_attn(q, q, q, cu[:1], 4)
    with pytest.raises(ValueError, match="lse"):
        dora.dora_grouped_attn_backward(q, q, q, q, q, None, cu, 4)
    with pytest.raises(ValueError, match="kind"):
        dora.dora_residual_norm(torch.zeros((2, 8)), None, torch.zeros(8), kind="batch")
    with pytest.raises(ValueError, match=r"\[T, C\]"):
        dora.dora_residual_norm(torch.zeros(8), None, torch.zeros(8))
    with pytest.raises(ValueError, match="on the GPU"):
        dora.dora_residual_norm_backward(torch.zeros((2, 8)), torch.zeros((2, 8)), None, torch.zeros(8),
                                         workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    for t in (torch.zeros((4, 2, 64), dtype=torch.float16), torch.zeros((4, 2, 64)).to_sparse()):
        with pytest.raises((TypeError, ValueError)):
            dora.dora_rope(t, pos, freq, q_out=t)


def test_constants():
    text = open(os.path.join(build.INCLUDE, "dora.h")).read()
    m = re.search(r"#define\s+DORA_MAX_SEQUENCES\s+(\d+)", text)
    assert int(m.group(1)) == dora.DORA_MAX_SEQUENCES
    for name in ("DORA_NORM_LAYER", "DORA_NORM_RMS"):
        assert int(re.search(name + r" = (\d)", text).group(1)) == getattr(dora, name)
    assert ctypes.sizeof(dora.Rows) == 48


@pytest.mark.parametrize("source", build.BLOCK_SOURCES)
def test_no_scratch(source):
    flags = [f for f in build.POLICY_FLAGS if f != "-shared"]
    cmd = [build.hipcc(), *flags, "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage",
           os.path.join(build.CSRC, source), "-o", os.devnull]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr
    names = re.findall(r"Function Name: (\S+)", res.stderr)
    scratch = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", res.stderr)]
    assert names and len(names) == len(scratch)
    assert not [(n, b) for n, b in zip(names, scratch) if b]
