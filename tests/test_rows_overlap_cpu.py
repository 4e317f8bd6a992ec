"""Which descriptions of rows share memory, however many rows there are: against every
element of small ones, and by construction for long ones."""
import ctypes
import random
import subprocess

import pytest

import paper_2609_34325_amd as dora
from paper_2609_34325_amd import build

A = 0x10000000          # never dereferenced
PROBE = """
#include "rows.h"
extern "C" int pair(const dora_rows* s, const dora_rows* t) { return dora::rows_meet(s, t); }
extern "C" int vector(const dora_rows* s, void* p, size_t n) { return dora::rows_meet(s, dora::Extent(p, n)); }
"""


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "probe.hip").write_text(PROBE)
    so = str(d / "probe.so")
    subprocess.run([build.hipcc(), "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", build.INCLUDE, "-I",
                    build.CSRC, str(d / "probe.hip"), "-o", so], check=True, capture_output=True, timeout=300)
    lib = ctypes.CDLL(so)
    lib.vector.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t]
    return lib


def rows(at, n, heads, dim, row, head, dtype=dora.DORA_F32):
    return dora.Rows(A + (4 if dtype == dora.DORA_F32 else 2) * at, n, heads, dim, row, head, dtype, 0)


def meet(probe, s, t):
    got = bool(probe.pair(ctypes.byref(s), ctypes.byref(t)))
    assert got == bool(probe.pair(ctypes.byref(t), ctypes.byref(s)))
    return got


def places(t):
    return {(t.data - A) // 4 + r * t.row_stride + h * t.head_stride + d for r in range(t.rows) for h in range(t.heads)
            for d in range(t.dim)}


@pytest.mark.parametrize("T", [1, 100, 1100, 1366, 4096, 4097, 100000, 2000000])
@pytest.mark.parametrize("H,D", [(1, 64), (12, 64), (32, 128), (3, 32)])
def test_slices_of_heads_before_rows(probe, T, H, D):
    """q, k and v in the last dimension of one [H, T, 3 D] buffer."""
    q, k, v = (rows(i * D, T, H, D, 3 * D, 3 * D * T, dora.DORA_BF16) for i in range(3))
    assert not meet(probe, q, k) and not meet(probe, k, v) and not meet(probe, q, v)
    assert meet(probe, q, q)
    assert meet(probe, q, rows(8, T, H, D, 3 * D, 3 * D * T, dora.DORA_BF16))                 # eight elements on
    late = rows((T - 1) * 3 * D + D - 8, T, H, D, 3 * D, 3 * D * T, dora.DORA_BF16)            # from q's last row on, over its end
    assert meet(probe, q, late)
    if H > 1:
        assert not meet(probe, q, rows((T - 1) * 3 * D + D, T, H, D, 3 * D, 3 * D * T, dora.DORA_BF16))  # over k's places alone


def test_slices_are_taken():
    """dq, dk and dv in that layout are refused for nothing but the workspace that comes after."""
    T, H, D, big = 5000, 12, 64, 1 << 32
    r = [rows(i * D, T, H, D, 3 * D, 3 * D * T, dora.DORA_BF16) for i in range(3)]
    others = [rows(i * big, T, H, D, H * D, D, dora.DORA_BF16) for i in range(1, 6)]
    ref = ctypes.byref
    lib = dora.load_library()

    def call(ws, n):
        return lib.dora_grouped_attn_backward(*(ref(t) for t in others), A + 12 * big, A + 13 * big, A + 14 * big, 2, T, 1, 0.0,
                                              *(ref(t) for t in r), ws, n, A + 15 * big, None)
    assert call(A + 16 * big, 0) == dora.DORA_ERR_WORKSPACE
    need = lib.dora_grouped_attn_backward_workspace_size(2, H, H, D, T, T, T)
    assert call(A + 2 * 3 * D * T, need) == dora.DORA_ERR_OVERLAP         # in the second head's gradients
    r[1] = rows(D - 8, T, H, D, 3 * D, 3 * D * T, dora.DORA_BF16)
    assert call(A + 16 * big, need) == dora.DORA_ERR_OVERLAP


def test_alike_against_every_element(probe):
    """The same strides in both (or one of them a single row or head): told apart exactly."""
    rng = random.Random(17)
    shared = apart = 0
    for _ in range(30000):
        dim, heads, n = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 5)
        hs = dim + rng.choice((0, 0, 1, 2, 5, 2 * dim))
        row = (heads - 1) * hs + dim + rng.choice((0, 0, 1, 7, 12))
        if rng.random() < 0.5:      # heads before rows
            row, hs = dim + rng.choice((0, 1, 3, 2 * dim)), 0
            hs = (n - 1) * row + dim + rng.choice((0, 0, 5, 15))
        s = rows(0, n, heads, dim, row, hs)
        t = rows(rng.randint(-70, 70), n, heads, rng.randint(1, dim), row, hs)
        a, b = places(s), places(t)
        if len(a) < n * heads * s.dim:
            continue
        want = bool(a & b)
        if blocks(s) != blocks(t):
            assert meet(probe, s, t) or not want
            continue
        assert meet(probe, s, t) == want, [(x.data - A, x.rows, x.heads, x.dim, x.row_stride, x.head_stride) for x in (s, t)]
        shared, apart = shared + want, apart + (not want)
    assert shared > 3000 and apart > 3000


def blocks(t):
    """Distances that count: of a tensor whose heads (rows) are adjacent, the outer one alone."""
    outer = max((t.row_stride, t.rows), (t.head_stride, t.heads)) if t.rows > 1 and t.heads > 1 else None
    return (outer, t.row_stride == t.dim and t.rows > 1, t.head_stride == t.dim and t.heads > 1)


def test_one_level_against_two(probe):
    """A tensor of evenly spaced pieces between another's rows and heads."""
    rng = random.Random(19)
    shared = apart = 0
    for _ in range(20000):
        dim, heads, n = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 5)
        hs = dim + rng.choice((0, 1, 2, 5, 2 * dim))
        s = rows(0, n, heads, dim, (heads - 1) * hs + dim + rng.choice((0, 1, 7, 12)), hs)
        m, d = rng.randint(1, 9), rng.randint(1, 3)
        t = rows(rng.randint(-40, 80), m, 1, d, d + rng.choice((0, 1, 4, hs, 9)), 0)
        want = bool(places(s) & places(t))
        assert meet(probe, s, t) == want, [(x.data - A, x.rows, x.heads, x.dim, x.row_stride, x.head_stride) for x in (s, t)]
        shared, apart = shared + want, apart + (not want)
    assert shared > 3000 and apart > 3000


def test_many_pieces_and_vectors(probe):
    """More pieces than are looked at one by one, single places between them."""
    n, dim, row = 50000, 8, 24
    s = rows(0, n, 1, dim, row, dim)
    rng = random.Random(18)
    for _ in range(2000):
        at, length = rng.randint(0, n * row), rng.randint(1, 30)
        first = max(0, (at - dim) // row)
        want = any(r * row < at + length and at < r * row + dim for r in range(first, min(n, first + 4)))
        assert bool(probe.vector(ctypes.byref(s), A + 4 * at, 4 * length)) == want, (at, length)
        heads = rows(0, n, 3, dim, row, n * row)                      # heads before rows
        at = rng.randint(0, 3 * n * row)
        got = bool(probe.vector(ctypes.byref(heads), A + 4 * at, 4 * length))
        want = any(at + i < 3 * n * row and (at + i) % row < dim for i in range(length))
        assert got == want, (at, length)


def test_read_again_and_again(probe):
    """Inputs with strides of 0 are one row or head of memory."""
    out = rows(0, 6, 4, 8, 64, 16)
    assert not meet(probe, out, rows(8, 6, 4, 8, 0, 16))              # between the heads of the first row
    assert not meet(probe, out, rows(64 + 24, 6, 4, 8, 0, 0))
    assert meet(probe, out, rows(64 + 23, 6, 4, 8, 0, 0))
    assert meet(probe, out, rows(64 + 24, 6, 4, 9, 0, 0))
    assert not meet(probe, out, rows(6 * 64, 60000, 4, 8, 0, 0))
    assert bool(probe.vector(ctypes.byref(rows(0, 9, 1, 8, 0, 0)), A + 4 * 7, 4)) is True
    assert bool(probe.vector(ctypes.byref(rows(0, 9, 1, 8, 0, 0)), A + 4 * 8, 4)) is False
