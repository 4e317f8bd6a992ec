"""Policy operators (CPU): the plain forms the GPU tests compare with, against
differences and brute force; and the refusals of the entry points, which all
come before anything reaches the GPU."""
import ctypes
import itertools
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_34325_amd as dora
import policy_ref as P
from paper_2609_34325_amd import build

FAKE = 0x100000  # never dereferenced


# ------------------------------------------------------- the plain forms

@pytest.mark.parametrize("A,lr,ref", [(1.3, 0.05, None), (-0.7, 0.1, 0.2), (0.9, 0.5, -0.3), (-1.1, -0.6, 0.1),
                                      (1.0, -0.6, 0.4), (-1.0, 0.5, None)])
def test_plain_policy_gradient_against_differences(A, lr, ref):
    rng = np.random.default_rng(5)
    x, a, n = rng.normal(0, 2, (1, 9)), np.array([3]), np.array([7])
    lp = P.softmax_row(x[0, :7], 3)[0]
    old, rf = np.array([lp - lr]), None if ref is None else np.array([lp + ref])
    kw = dict(ref=rf, weight=np.array([0.6]), legal=n, low=0.2, high=0.3, kl_coef=0.4 if ref else 0.0, ent=0.05)
    g = P.policy(x, a, old, np.array([A]), **kw)[0]
    h = 1e-6
    for j in range(9):
        y = x.copy()
        y[0, j] += h
        z = x.copy()
        z[0, j] -= h
        num = (P.policy(y, a, old, np.array([A]), **kw)[3][0] - P.policy(z, a, old, np.array([A]), **kw)[3][0]) / (2 * h)
        # second-order differences: error h^2 times a third derivative of a few units, and rounding 1e-16 / h
        assert abs(num - g[0, j]) < 1e-8


def test_plain_pl_gradient_against_differences():
    rng = np.random.default_rng(6)
    s = rng.normal(0, 2, 8)
    order, cu = np.array([4, 1, 6]), [0, 3]
    lp = P.pl(s, order, cu, [0.0], [0.0], segments=[(0, 8)])[1][0]
    kw = dict(ref=[lp + 0.2], weight=[1.5], segments=[(0, 8)], kl_coef=0.3)
    g = P.pl(s, order, cu, [lp - 0.1], [0.8], **kw)[0]
    assert g[0] == 0
    h = 1e-6
    for j in range(1, 8):
        hi, lo = s.copy(), s.copy()
        hi[j] += h
        lo[j] -= h
        num = (P.pl(hi, order, cu, [lp - 0.1], [0.8], **kw)[2][0] - P.pl(lo, order, cu, [lp - 0.1], [0.8], **kw)[2][0]) / (2 * h)
        assert abs(num - g[j]) < 1e-8


def test_plain_pl_probabilities_sum_to_one():
    s = np.random.default_rng(7).normal(0, 1, 6)
    total = sum(np.exp(P.pl(s, np.array(o), [0, 2], [0.0], [0.0], segments=[(0, 6)])[1][0])
                for o in itertools.permutations(range(1, 6), 2))
    assert abs(total - 1) < 1e-12


# --------------------------------------------------------- C ABI refusals

def logprob(**kw):
    a = dict(x=FAKE, ld=100, act=FAKE, legal=None, w=None, T=4, V=96, dtype=1, lp=FAKE, H=None, ws=None, wsb=0, st=FAKE,
             stream=None)
    a.update(kw)
    return dora.load_library().dora_action_logprob(*a.values())


def policy(**kw):
    a = dict(x=FAKE, ld=100, act=FAKE, legal=None, old=FAKE, ref=None, A=FAKE, w=None, T=4, V=96, dtype=1, low=0.2,
             high=0.2, kl=0.0, ent=0.0, g=0x900000, ldg=96, lp=FAKE, stats=FAKE, ws=FAKE,
             wsb=dora.dora_policy_workspace_size(4, 96), st=FAKE, stream=None)
    a.update(kw)
    return dora.load_library().dora_policy_loss(*a.values())


def pl(**kw):
    a = dict(s=FAKE, order=FAKE, cuo=FAKE, cu=None, total=0, old=FAKE, ref=None, A=FAKE, w=None, B=4, N=197, low=0.2,
             high=0.2, kl=0.0, g=0x900000, lp=FAKE, stats=FAKE, ws=FAKE, wsb=dora.dora_pl_policy_workspace_size(4),
             st=FAKE, stream=None)
    a.update(kw)
    return dora.load_library().dora_pl_policy_loss(*a.values())


def spans(*items):
    return (dora.Span * len(items))(*(dora.Span(*i) for i in items))


def clip(grads, out=None, n=None, max_norm=1.0, eps=1e-6, norm=FAKE, ws=FAKE, wsb=None):
    n = len(grads) if n is None else n
    wsb = dora.dora_grad_clip_workspace_size(len(grads)) if wsb is None else wsb
    return dora.load_library().dora_grad_clip(ctypes.addressof(grads), None if out is None else ctypes.addressof(out),
                                              n, max_norm, eps, norm, ws, wsb, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("call", [logprob, policy])
def test_logits_refusals(call):
    assert call(x=None) == dora.DORA_ERR_NULL
    assert call(act=None) == dora.DORA_ERR_NULL
    assert call(lp=None) == dora.DORA_ERR_NULL
    assert call(st=None) == dora.DORA_ERR_NULL
    assert call(dtype=2) == dora.DORA_ERR_DTYPE
    assert call(T=0) == dora.DORA_ERR_SHAPE
    assert call(T=dora.DORA_MAX_DECISIONS + 1) == dora.DORA_ERR_SHAPE
    assert call(V=0) == dora.DORA_ERR_SHAPE
    assert call(V=dora.DORA_MAX_ACTIONS + 1, ld=1 << 21) == dora.DORA_ERR_SHAPE
    assert call(ld=95) == dora.DORA_ERR_SHAPE
    assert call(ld=(1 << 32) + 1) == dora.DORA_ERR_SHAPE
    assert call(x=FAKE + 1) == dora.DORA_ERR_ALIGN
    assert call(x=FAKE + 2, dtype=0) == dora.DORA_ERR_ALIGN
    need = dora.dora_policy_workspace_size(4, 96)
    assert call(ws=FAKE + 16, wsb=need) == dora.DORA_ERR_WORKSPACE
    assert call(ws=FAKE, wsb=need - 1) == dora.DORA_ERR_WORKSPACE


def test_policy_refusals():
    assert policy(old=None) == dora.DORA_ERR_NULL
    assert policy(A=None) == dora.DORA_ERR_NULL
    assert policy(g=None) == dora.DORA_ERR_NULL
    assert policy(stats=None) == dora.DORA_ERR_NULL
    assert policy(kl=0.1) == dora.DORA_ERR_NULL                      # a KL term needs the reference
    assert policy(ws=None) == dora.DORA_ERR_WORKSPACE
    assert policy(ldg=95) == dora.DORA_ERR_SHAPE
    for bad in (dict(low=-0.1), dict(low=1.1), dict(low=NAN), dict(high=-0.1), dict(high=NAN), dict(kl=NAN, ref=FAKE),
                dict(kl=INF, ref=FAKE), dict(ent=NAN), dict(ent=-INF)):
        assert policy(**bad) == dora.DORA_ERR_SHAPE, bad
    assert policy(g=0x900001) == dora.DORA_ERR_ALIGN
    # 4 bf16 rows of 96, 100 apart, at FAKE: 792 bytes
    assert policy(g=FAKE + 2, ldg=100) == dora.DORA_ERR_OVERLAP      # rows shifted by one element
    assert policy(g=FAKE, ldg=96) == dora.DORA_ERR_OVERLAP           # same start, other rows
    assert policy(g=FAKE + 790, ldg=100) == dora.DORA_ERR_OVERLAP    # the last element only
    assert policy(g=FAKE + 8, ldg=100) == dora.DORA_ERR_OVERLAP      # half in the gap
    assert policy(g=FAKE - 790, ldg=100) == dora.DORA_ERR_OVERLAP


def test_policy_sizes():
    assert dora.dora_policy_workspace_size(0, 5) == 0
    assert dora.dora_policy_workspace_size(5, 0) == 0
    assert dora.dora_policy_workspace_size(dora.DORA_MAX_DECISIONS + 1, 5) == 0
    assert dora.dora_policy_workspace_size(5, dora.DORA_MAX_ACTIONS + 1) == 0
    assert dora.dora_policy_workspace_size(dora.DORA_MAX_DECISIONS, dora.DORA_MAX_ACTIONS) > 0
    assert dora.dora_policy_workspace_size(5, 5) % 256 == 0
    assert dora.DORA_MAX_DECISIONS * 256 < 1 << 32        # threads of a launch, for rows of 256 threads
    assert dora.dora_pl_policy_workspace_size(0) == 0 and dora.dora_pl_policy_workspace_size(8193) == 0
    assert dora.dora_grad_clip_workspace_size(0) == 0 and dora.dora_grad_clip_workspace_size(65537) == 0
    header = open(os.path.join(build.INCLUDE, "dora.h")).read()
    for name in ("DORA_MAX_DECISIONS", "DORA_MAX_ACTIONS", "DORA_DEV_ACTION"):
        m = re.search(r"#define\s+%s\s+(0x[0-9a-fA-F]+|\d+)" % name, header)
        assert int(m.group(1), 0) == getattr(dora, name)
    assert dora.dora_status_string(dora.DORA_ERR_OVERLAP).startswith("DORA_ERR_OVERLAP")
    assert ctypes.sizeof(dora.Span) == 24


def test_pl_refusals():
    for name in ("s", "order", "cuo", "old", "A", "g", "lp", "stats", "st"):
        assert pl(**{name: None}) == dora.DORA_ERR_NULL, name
    assert pl(kl=0.1) == dora.DORA_ERR_NULL
    for bad in (dict(B=0), dict(B=8193), dict(N=0), dict(N=dora.DORA_MAX_ROW_TOKENS + 1), dict(cu=FAKE, total=-1),
                dict(low=NAN), dict(high=-1.0), dict(kl=INF, ref=FAKE)):
        assert pl(**bad) == dora.DORA_ERR_SHAPE, bad
    assert pl(g=FAKE + 4) == dora.DORA_ERR_OVERLAP
    assert pl(ws=None) == dora.DORA_ERR_WORKSPACE
    assert pl(ws=FAKE + 128) == dora.DORA_ERR_WORKSPACE
    assert pl(wsb=dora.dora_pl_policy_workspace_size(4) - 1) == dora.DORA_ERR_WORKSPACE


def test_clip_refusals():
    one = spans((FAKE, 100, 0, 0))
    lib = dora.load_library()
    assert lib.dora_grad_clip(None, None, 1, 1.0, 1e-6, FAKE, FAKE, 1 << 20, None) == dora.DORA_ERR_NULL
    assert clip(one, norm=None) == dora.DORA_ERR_NULL
    assert clip(one, n=0) == dora.DORA_ERR_SHAPE
    assert clip(one, n=65537) == dora.DORA_ERR_SHAPE
    for bad in (dict(max_norm=-1.0), dict(max_norm=NAN), dict(eps=-1.0), dict(eps=NAN)):
        assert clip(one, **bad) == dora.DORA_ERR_SHAPE, bad
    assert clip(one, ws=None) == dora.DORA_ERR_WORKSPACE
    assert clip(one, ws=FAKE + 8) == dora.DORA_ERR_WORKSPACE
    assert clip(one, wsb=dora.dora_grad_clip_workspace_size(1) - 1) == dora.DORA_ERR_WORKSPACE
    assert clip(spans((FAKE, 100, 2, 0))) == dora.DORA_ERR_DTYPE
    assert clip(spans((FAKE, -1, 0, 0))) == dora.DORA_ERR_SHAPE
    assert clip(spans((None, 1, 0, 0))) == dora.DORA_ERR_NULL
    assert clip(spans((FAKE + 2, 1, 0, 0))) == dora.DORA_ERR_ALIGN
    assert clip(one, spans((0x900000, 99, 0, 0))) == dora.DORA_ERR_SHAPE
    assert clip(one, spans((0x900000, 100, 1, 0))) == dora.DORA_ERR_SHAPE


def test_clip_overlaps():
    a, b = (FAKE, 100, 0, 0), (FAKE + 396, 100, 0, 0)             # b starts at a's last element
    far, far2 = (0x900000, 100, 0, 0), (0xA00000, 100, 0, 0)
    assert clip(spans(a, a)) == dora.DORA_ERR_OVERLAP              # the same gradient twice, in place
    assert clip(spans(a, b)) == dora.DORA_ERR_OVERLAP
    assert clip(spans(a), spans(b)) == dora.DORA_ERR_OVERLAP       # onto part of its own input
    assert clip(spans(a, far), spans(far2, b)) == dora.DORA_ERR_OVERLAP   # onto part of another input
    assert clip(spans(a, far), spans(far, a)) == dora.DORA_ERR_OVERLAP    # swapped
    assert clip(spans(a, far), spans(far2, far2)) == dora.DORA_ERR_OVERLAP


# -------------------------------------------------- refusals of the binding

def test_binding_refusals():
    x, a, f = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    st = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="logits must be on the GPU"):
        dora.dora_action_logprob(x, a)
    with pytest.raises(ValueError, match=r"logits must be \[T, V\]"):
        dora.dora_policy_loss(x[0], a, f, f)
    with pytest.raises(TypeError, match="logits must be a torch tensor"):
        dora.dora_policy_loss(None, a, f, f)
    s, order, cuo = torch.zeros(4, 9), torch.zeros(4, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    ws = torch.empty(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="scores must be on the GPU"):
        dora.dora_pl_policy_loss(s, order, cuo, f, f, workspace=ws, dev_status=st)
    with pytest.raises(ValueError, match=r"advantage must be \[4\]"):
        dora.dora_pl_policy_loss(s, order, cuo, f, f[:3], workspace=ws, dev_status=st)
    with pytest.raises(ValueError, match=r"dscores must be"):
        dora.dora_pl_policy_loss(s, order, cuo, f, f, dscores=torch.zeros(4, 8), workspace=ws, dev_status=st)
    with pytest.raises(ValueError, match="packed input needs N"):
        dora.dora_pl_policy_loss(s.view(-1), order, cuo, f, f, cu_in=cuo, workspace=ws, dev_status=st)
    with pytest.raises(ValueError, match=r"grads\[0\] must be on the GPU"):
        dora.dora_grad_clip([f], 1.0)
    with pytest.raises(ValueError, match="grads is empty"):
        dora.dora_grad_clip([], 1.0)
    with pytest.raises(TypeError, match=r"grads\[0\] must be a torch tensor"):
        dora.dora_grad_clip([3], 1.0)


def test_native_helpers_leave_the_rest_to_python():
    """What the native checks do not take goes to those in Python."""
    dora.load_library()
    t = torch.zeros(4, 8)
    room = (dora.Span * 2)()
    for got in (dora._native_rows(t), dora._native_rows(3), dora._native_vectors(-1, 4, t[0]),
                dora._native_vectors(0, 8, t[0]), dora._native_vectors(0, 8), dora._native_vectors("x", 8, t[0]),
                dora._native_vectors(0, "x", t[0]), dora._native_spans([t], ctypes.addressof(room)),
                dora._native_spans((t,), ctypes.addressof(room)), dora._native_spans([3], ctypes.addressof(room))):
        assert got is NotImplemented
    assert dora._native_vectors(0, 8, None, -1, None) is True
    with pytest.raises(ValueError):
        dora._native_spans([t], 0)
    with pytest.raises(TypeError, match="b must be a torch tensor"):
        dora._vectors(("a", "b"), -1, 8, None, 3, 5)
    with pytest.raises(ValueError, match=r"a must be \[3\]"):
        dora._vectors(("a",), -1, 3, t[0])
    with pytest.raises(ValueError, match="tensors on devices 0 and -1"):
        dora._vectors(("a",), 0, -1, t)


@pytest.mark.parametrize("source", build.POLICY_SOURCES)
def test_no_scratch(source):
    """No register of these kernels lives in scratch memory."""
    flags = [f for f in build.POLICY_FLAGS if f != "-shared"]
    cmd = [build.hipcc(), *flags, "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage",
           os.path.join(build.CSRC, source), "-o", os.devnull]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr
    names = re.findall(r"Function Name: (\S+)", res.stderr)
    scratch = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", res.stderr)]
    assert names and len(names) == len(scratch)
    assert not [(n, b) for n, b in zip(names, scratch) if b]
