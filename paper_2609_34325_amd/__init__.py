"""DORA deployment hot path on AMD Instinct MI355X (gfx950).

Thin binding over ``libdora.so`` (C ABI in ``include/dora.h``).  Every
step of the path runs in the library's HIP kernels; this module only checks
tensor arguments, allocates outputs with torch when the caller does not pass
them, and forwards raw device pointers and the current HIP stream (through
``csrc/host_call.cpp``; calls that it leaves out go through ctypes).

DORA (arXiv 2609.34325): hard deletion keeps CLS and the survivors' order
(Sec. 3.1, Eq. (1)); deployment removes the highest-scoring visual tokens
(Sec. 3.2 "Sampling and deployment"; App. A.3); survivors are packed with
explicit sequence boundaries and run through variable-length attention that
never attends across images (Sec. 3.5 "Inference"; App. E.5).

There is no fallback: if the library is missing, every call raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import warnings
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdora.so")

DORA_F32 = 0
DORA_BF16 = 1

DORA_OK = 0
DORA_ERR_NULL = -1
DORA_ERR_SHAPE = -2
DORA_ERR_DTYPE = -3
DORA_ERR_ALIGN = -4
DORA_ERR_UNSUPPORTED = -5
DORA_ERR_CAPACITY = -6
DORA_ERR_HIP = -7
DORA_ERR_WORKSPACE = -8
DORA_ERR_STATIC_LIMIT = -9
DORA_ERR_OVERLAP = -10

DORA_DEV_KEEP_RANGE = 0x1
DORA_DEV_CAPACITY = 0x2
DORA_DEV_CU_IN = 0x4
DORA_DEV_CU_SEQLENS = 0x8
DORA_DEV_PLAN = 0x10

DORA_DEV_ACTOR = 0x20
DORA_DEV_ACTION = 0x40
DORA_MAX_ROW_TOKENS = 2048
DORA_MAX_SEQLEN = 16384
DORA_HEAD_DIM = 64
DORA_MAX_DECISIONS = (1 << 24) - 1
DORA_MAX_ACTIONS = 1 << 20
DORA_NOALLOC_WORKSPACE_BYTES = 4 << 20
DORA_MAX_SEQUENCES = 65536
DORA_NORM_LAYER = 0
DORA_NORM_RMS = 1

EXPORTS = (
    "dora_select_pack",
    "dora_select_pack_plan",
    "dora_select_pack_residual",
    "dora_actor_gate",
    "dora_actor_decode",
    "dora_pl_sample",
    "dora_pl_logprob",
    "dora_pl_logprob_cap",
    "dora_lc1_readout_workspace_size",
    "dora_lc1_readout",
    "dora_trajectory_flops",
    "dora_varlen_attn_workspace_size",
    "dora_varlen_attn_plan",
    "dora_varlen_attn_execute",
    "dora_varlen_attn",
    "dora_varlen_attn_noalloc",
    "dora_policy_workspace_size",
    "dora_action_logprob",
    "dora_policy_loss",
    "dora_pl_policy_workspace_size",
    "dora_pl_policy_loss",
    "dora_pl_policy_loss_cap",
    "dora_grad_clip_workspace_size",
    "dora_grad_clip",
    "dora_rope",
    "dora_grouped_attn_workspace_size",
    "dora_grouped_attn_backward_workspace_size",
    "dora_grouped_attn",
    "dora_grouped_attn_backward",
    "dora_residual_norm",
    "dora_residual_norm_workspace_size",
    "dora_residual_norm_backward",
    "dora_status_string",
)

# Entry points that host_call.cpp marshals, in its order, with the name and
# required type of each tensor argument (None: an integer, float or address).
_F32, _I32, _I64, _ANY = torch.float32, torch.int32, torch.int64, None
_PACK = (("scores", _F32), ("keep", _I32), ("tokens", _ANY))
_PACK_OUT = (("idx_out", _I32), ("cu_out", _I32), ("packed_out", _ANY), None)
_STATUS = (("dev_status", _I32), None)
_ATTN = (("q", _ANY), ("k", _ANY), ("v", _ANY), ("cu_seqlens", _I32)) + (None,) * 7 + \
    (("out", _ANY), ("workspace", _ANY), None) + _STATUS
# The rows of logits go by address and leading dimension (strided views are allowed).
_LOGITS = (None, None, ("actions", _I32), ("legal", _I32))
_DECISIONS = (("old_logprob", _F32), ("ref_logprob", _F32), ("advantage", _F32), ("weight", _F32))
_LOSS_OUT = (("logprob_out", _F32), ("stats_out", _F32), ("workspace", _ANY), None) + _STATUS
_NORM = ("gamma", "beta", "scale", "gate", "post_gamma", "post_beta")
_NORM_GRADS = tuple("d" + n for n in ("gamma", "beta", "scale", "gate", "post_gamma", "post_beta"))
_ENTRIES = (
    ("dora_select_pack", _PACK + (("cu_in", _I32),) + (None,) * 5 + _PACK_OUT + _STATUS),
    ("dora_select_pack_plan", _PACK + (("cu_in", _I32),) + (None,) * 5 + _PACK_OUT + (None,) * 3 +
     (("workspace", _ANY), None) + _STATUS),
    ("dora_select_pack_residual", _PACK + (("a", _ANY), ("cu_in", _I32)) + (None,) * 5 + _PACK_OUT + _STATUS),
    ("dora_actor_gate", (("p_gate", _F32), ("cu_in", _I32), None, None, None, ("on_rank", _I32), ("on_list", _I32),
                         ("n_on", _I32)) + _STATUS),
    ("dora_actor_decode", (("budget_logits", _F32), None, None, ("removal_scores", _F32), ("cu_in", _I32), None, None,
                           None, ("on_rank", _I32), ("keep_out", _I32), ("scores_out", _F32)) + _STATUS),
    ("dora_pl_sample", (("scores", _F32), ("gumbel", _F32), ("k", _I32), ("cu_in", _I32), None, None, None,
                        ("order_out", _I32), ("cu_order_out", _I32), ("logprob_out", _F32), None) + _STATUS),
    ("dora_pl_logprob_cap", (("scores", _F32), ("order", _I32), ("cu_order", _I32), None, ("cu_in", _I32), None, None, None,
                         ("logprob_out", _F32)) + _STATUS),
    ("dora_lc1_readout", (("x", _ANY), ("cu_seqlens", _I32), None, None, None, None, ("gamma", _F32), ("beta", _F32),
                          None, ("out", _F32), ("workspace", _ANY), None) + _STATUS),
    ("dora_trajectory_flops", (("tokens", _I32), None, None, ("flops_out", _I64), ("total_out", _I64)) + _STATUS),
    ("dora_varlen_attn_plan", (("cu_seqlens", _I32), None, None, None, None, ("workspace", _ANY), None) + _STATUS),
    ("dora_varlen_attn_execute", _ATTN),
    ("dora_varlen_attn", _ATTN),
    ("dora_action_logprob", _LOGITS + (("weight", _F32), None, None, None, ("logprob_out", _F32),
                                       ("entropy_out", _F32), ("workspace", _ANY), None) + _STATUS),
    ("dora_policy_loss", _LOGITS + _DECISIONS + (None,) * 9 + _LOSS_OUT),
    ("dora_pl_policy_loss_cap", (("scores", _F32), ("order", _I32), ("cu_order", _I32), None, ("cu_in", _I32), None) +
     _DECISIONS + (None,) * 5 + (("dscores", _F32),) + _LOSS_OUT),
    ("dora_grad_clip", (None,) * 5 + (("norm_out", _F32), ("workspace", _ANY), None, None)),
    # Rows go by the address of their description (strided views are allowed).
    ("dora_rope", (None, None, ("positions", _I32), None, ("freq", _ANY)) + (None,) * 7),
    ("dora_grouped_attn", (None,) * 3 + (("cu_q", _I32), ("cu_k", _I32)) + (None,) * 6 +
     (("lse_out", _F32), ("workspace", _ANY), None) + _STATUS),
    ("dora_grouped_attn_backward", (None,) * 5 + (("lse", _F32), ("cu_q", _I32), ("cu_k", _I32)) + (None,) * 7 +
     (("workspace", _ANY), None) + _STATUS),
    ("dora_residual_norm", (None, None) + tuple((n, _F32) for n in _NORM) + (None,) * 5),
    ("dora_residual_norm_backward", (None,) * 4 + tuple((n, _F32) for n in _NORM if n != "beta") + (None,) * 4 +
     tuple((n, _F32) for n in _NORM_GRADS) + (("workspace", _ANY), None, None)),
)
_INDEX = {name: i for i, (name, _) in enumerate(_ENTRIES)}

_OPTIONAL = ("cu_in", "budget_logits", "removal_scores", "scores_out", "workspace", "legal", "weight", "ref_logprob",
             "entropy_out", "lse_out") + _NORM[1:] + _NORM_GRADS

_lib = None
_native_call = None
_native_spans = None
_native_rows = None
_native_vectors = None
_native_written = None
_native_describe = None


class FlopsConfig(ctypes.Structure):
    """dora_flops_config of include/dora.h."""
    _fields_ = [(name, ctypes.c_int32) for name in
                ("d", "L", "N0", "patch", "in_chans", "classes", "head_inputs", "mlp_ratio", "M", "actor")]


class Span(ctypes.Structure):
    """dora_span of include/dora.h."""
    _fields_ = [("data", ctypes.c_void_p), ("numel", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class Rows(ctypes.Structure):
    """dora_rows of include/dora.h."""
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class DoraError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} failed: {dora_status_string(code)} ({code})")
        self.code = code


def _leave_to_ctypes(*args):
    return NotImplemented


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libdora.so (built in-tree by ``paper_2609_34325_amd.build``)."""
    global _lib, _native_call, _native_spans, _native_rows, _native_vectors, _native_written, _native_describe
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"libdora.so not found at {p}; build it with "
                           "`python -m paper_2609_34325_amd.build` (no fallback path exists)")
    lib = ctypes.CDLL(p)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.dora_select_pack.restype = ctypes.c_int
    lib.dora_select_pack.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, ctypes.c_int,
                                     vp, vp, vp, i64, vp, vp]
    lib.dora_select_pack_plan.restype = ctypes.c_int
    lib.dora_select_pack_plan.argtypes = lib.dora_select_pack.argtypes[:13] + [i32, i32, i64, vp, sz,
                                                                               vp, vp]
    lib.dora_select_pack_residual.restype = ctypes.c_int
    lib.dora_select_pack_residual.argtypes = lib.dora_select_pack.argtypes[:3] + [vp] + \
        lib.dora_select_pack.argtypes[3:]
    lib.dora_actor_gate.restype = ctypes.c_int
    lib.dora_actor_gate.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.dora_actor_decode.restype = ctypes.c_int
    lib.dora_actor_decode.argtypes = [vp, i64, i32, vp, vp, i64, i32, i32, vp, vp, vp, vp, vp]
    lib.dora_pl_sample.restype = ctypes.c_int
    lib.dora_pl_sample.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, vp, i64, vp, vp]
    lib.dora_pl_logprob.restype = ctypes.c_int
    lib.dora_pl_logprob.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, vp]
    lib.dora_pl_logprob_cap.restype = ctypes.c_int
    lib.dora_pl_logprob_cap.argtypes = [vp, vp, vp, i64, vp, i64, i32, i32, vp, vp, vp]
    lib.dora_lc1_readout.restype = ctypes.c_int
    lib.dora_lc1_readout.argtypes = [vp, vp, i64, i32, i32, ctypes.c_int, vp, vp, ctypes.c_float, vp, vp, sz, vp,
                                     vp]
    lib.dora_lc1_readout_workspace_size.restype = sz
    lib.dora_lc1_readout_workspace_size.argtypes = [i32, i32]
    lib.dora_trajectory_flops.restype = ctypes.c_int
    lib.dora_trajectory_flops.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.dora_varlen_attn_workspace_size.restype = sz
    lib.dora_varlen_attn_workspace_size.argtypes = [i32, i32, i32]
    lib.dora_varlen_attn_plan.restype = ctypes.c_int
    lib.dora_varlen_attn_plan.argtypes = [vp, i32, i32, i32, i64, vp, sz, vp, vp]
    lib.dora_varlen_attn_execute.restype = ctypes.c_int
    lib.dora_varlen_attn_execute.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i64,
                                             ctypes.c_float, ctypes.c_int, vp, vp, sz, vp, vp]
    lib.dora_varlen_attn.restype = ctypes.c_int
    lib.dora_varlen_attn.argtypes = lib.dora_varlen_attn_execute.argtypes
    lib.dora_varlen_attn_noalloc.restype = ctypes.c_int
    lib.dora_varlen_attn_noalloc.argtypes = lib.dora_varlen_attn_execute.argtypes[:12] + [vp, vp]
    f32 = ctypes.c_float
    lib.dora_policy_workspace_size.restype = sz
    lib.dora_policy_workspace_size.argtypes = [i32, i32]
    lib.dora_action_logprob.restype = ctypes.c_int
    lib.dora_action_logprob.argtypes = [vp, i64, vp, vp, vp, i32, i32, ctypes.c_int, vp, vp, vp, sz, vp, vp]
    lib.dora_policy_loss.restype = ctypes.c_int
    lib.dora_policy_loss.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, i32, i32, ctypes.c_int, f32, f32, f32, f32, vp,
                                     i64, vp, vp, vp, sz, vp, vp]
    lib.dora_pl_policy_workspace_size.restype = sz
    lib.dora_pl_policy_workspace_size.argtypes = [i32]
    lib.dora_pl_policy_loss.restype = ctypes.c_int
    lib.dora_pl_policy_loss.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp, vp, i32, i32, f32, f32, f32, vp, vp, vp, vp,
                                        sz, vp, vp]
    lib.dora_pl_policy_loss_cap.restype = ctypes.c_int
    lib.dora_pl_policy_loss_cap.argtypes = lib.dora_pl_policy_loss.argtypes[:3] + [i64] + \
        lib.dora_pl_policy_loss.argtypes[3:]
    lib.dora_grad_clip_workspace_size.restype = sz
    lib.dora_grad_clip_workspace_size.argtypes = [i32]
    lib.dora_grad_clip.restype = ctypes.c_int
    lib.dora_grad_clip.argtypes = [vp, vp, i32, f32, f32, vp, vp, sz, vp]
    lib.dora_rope.restype = ctypes.c_int
    lib.dora_rope.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, f32, vp, vp, vp]
    for name in ("dora_grouped_attn_workspace_size", "dora_grouped_attn_backward_workspace_size"):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = [i32, i32, i32, i32, i32, i64, i64]
    lib.dora_grouped_attn.restype = ctypes.c_int
    lib.dora_grouped_attn.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, sz, vp, vp]
    lib.dora_grouped_attn_backward.restype = ctypes.c_int
    lib.dora_grouped_attn_backward.argtypes = [vp] * 8 + [i32, i32, i32, f32, vp, vp, vp, vp, sz, vp, vp]
    lib.dora_residual_norm.restype = ctypes.c_int
    lib.dora_residual_norm.argtypes = [vp] * 8 + [i32, f32, vp, vp, vp]
    lib.dora_residual_norm_workspace_size.restype = sz
    lib.dora_residual_norm_workspace_size.argtypes = [i64, i32]
    lib.dora_residual_norm_backward.restype = ctypes.c_int
    lib.dora_residual_norm_backward.argtypes = [vp] * 9 + [i32, f32] + [vp] * 9 + [sz, vp]
    lib.dora_status_string.restype = ctypes.c_char_p
    lib.dora_status_string.argtypes = [ctypes.c_int]
    lib.addresses = tuple(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name, _ in _ENTRIES)
    if _native_call is None:
        try:
            from ._host_call import (call as _native_call, describe as _native_describe, rows as _native_rows,
                                     spans as _native_spans, vectors as _native_vectors, written as _native_written)
        except ImportError as e:  # not built, or for another Python or torch
            warnings.warn(f"calls are marshalled by ctypes, about 5 us slower each: {e}; build the native marshalling "
                          "with `python -m paper_2609_34325_amd.build`")
            _native_call = _native_spans = _native_rows = _native_vectors = _native_written = _leave_to_ctypes
            _native_describe = _leave_to_ctypes
    if path is None:
        _lib = lib
    return lib


def _call(name: str, stream, *args) -> None:
    """Check the tensors of one entry point and enqueue it on `stream`.  args:
    every argument but the stream, tensors as they are.  Raises DoraError for
    a negative status."""
    lib = _lib or load_library()
    which = _INDEX[name]
    rc = NotImplemented
    if torch.cuda.is_initialized():  # else there is no tensor on the GPU
        st = torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else _stream(stream)
        rc = _native_call(which, lib.addresses[which], *args, st)
    if rc is NotImplemented:  # an argument that the native path leaves to these checks
        spec = _ENTRIES[which][1]
        rc = getattr(lib, name)(*(a if s is None or (a is None and s[0] in _OPTIONAL) else _dev(a, s[0], s[1])
                                  for a, s in zip(args, spec)), _stream(stream))
    if rc != DORA_OK:
        raise DoraError(name, rc)


def dora_status_string(code: int) -> str:
    return load_library().dora_status_string(int(code)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return DORA_BF16
    if t.dtype == torch.float32:
        return DORA_F32
    raise TypeError(f"unsupported dtype {t.dtype}; expected bfloat16 or float32")


def _dev(t: torch.Tensor, name: str, dtype=None) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _check(fn: str, code: int) -> None:
    if code != DORA_OK:
        raise DoraError(fn, code)


def new_status(device=None) -> torch.Tensor:
    """A zeroed int32 device status word."""
    return torch.zeros(1, dtype=torch.int32, device=device or "cuda")


def _select_pack_args(scores, keep, tokens, cu_in, N, idx_out, cu_out, packed_out, cap_rows, dev_status):
    B = int(keep.shape[0])
    if cu_in is None:
        if tokens.dim() != 3:
            raise ValueError("dense tokens must be [B,N,C]")
        N = int(tokens.shape[1])
        C = int(tokens.shape[2])
        total_in = B * N
        if tuple(scores.shape) != (B, N):
            raise ValueError("scores must be [B,N]")
    else:
        if tokens.dim() != 2:
            raise ValueError("packed tokens must be [total_in,C]")
        if N is None:
            raise ValueError("packed input needs N (an upper bound on segment lengths)")
        C = int(tokens.shape[1])
        total_in = int(tokens.shape[0])
        if scores.dim() != 1 or int(scores.shape[0]) < total_in:
            raise ValueError("packed scores must be [total_in]")
        if tuple(cu_in.shape) != (B + 1,):
            raise ValueError("cu_in must be [B+1]")
    dev = tokens.device
    if cap_rows is None:
        cap_rows = int(packed_out.shape[0]) if packed_out is not None else B * int(N)
    if idx_out is None:
        idx_out = torch.empty(cap_rows, dtype=torch.int32, device=dev)
    if cu_out is None:
        cu_out = torch.empty(B + 1, dtype=torch.int32, device=dev)
    if packed_out is None:
        packed_out = torch.empty((cap_rows, C), dtype=tokens.dtype, device=dev)
    if dev_status is None:
        dev_status = new_status(dev)
    if packed_out.dtype != tokens.dtype or int(packed_out.shape[-1]) != C:
        raise ValueError("packed_out must match the tokens' dtype and C")
    if int(idx_out.numel()) < cap_rows or int(packed_out.shape[0]) < cap_rows:
        raise ValueError("outputs smaller than cap_rows")
    args = [scores, keep, tokens, cu_in, total_in, B, int(N), C, _dtype_code(tokens), idx_out, cu_out, packed_out,
            int(cap_rows)]
    return args, (idx_out, cu_out, packed_out, dev_status)


def dora_select_pack(scores: torch.Tensor, keep: torch.Tensor, tokens: torch.Tensor,
                     cu_in: Optional[torch.Tensor] = None, N: Optional[int] = None,
                     idx_out: Optional[torch.Tensor] = None,
                     cu_out: Optional[torch.Tensor] = None,
                     packed_out: Optional[torch.Tensor] = None,
                     cap_rows: Optional[int] = None,
                     dev_status: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Keep CLS + the keep-1 highest keep-scores per image, pack the kept rows.

    Dense input: scores [B,N] fp32, tokens [B,N,C].  Packed input (a cascaded
    round): scores [total_in], tokens [total_in,C], cu_in [B+1] and N = an
    upper bound on the segment lengths.  keep: int32 [B] (counts CLS).
    Outputs (allocated if not given; capacity defaults to B*N rows so no
    host synchronisation is needed): idx [cap], cu [B+1], packed [cap,C],
    dev_status [1].  Returns (idx_out, cu_out, packed_out, dev_status).
    """
    args, outs = _select_pack_args(scores, keep, tokens, cu_in, N, idx_out, cu_out, packed_out,
                                   cap_rows, dev_status)
    _call("dora_select_pack", stream, *args, outs[3])
    return outs


def dora_select_pack_plan(scores: torch.Tensor, keep: torch.Tensor, tokens: torch.Tensor,
                          H: int, max_seqlen: int, total: int, workspace: torch.Tensor,
                          cu_in: Optional[torch.Tensor] = None, N: Optional[int] = None,
                          idx_out: Optional[torch.Tensor] = None,
                          cu_out: Optional[torch.Tensor] = None,
                          packed_out: Optional[torch.Tensor] = None,
                          cap_rows: Optional[int] = None,
                          dev_status: Optional[torch.Tensor] = None,
                          stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """dora_select_pack plus the attention plan of the packed output in `workspace`
    (for dora_varlen_attn_execute with cu_seqlens = cu_out, H heads, max_seqlen
    and total Q/K/V rows)."""
    args, outs = _select_pack_args(scores, keep, tokens, cu_in, N, idx_out, cu_out, packed_out,
                                   cap_rows, dev_status)
    _call("dora_select_pack_plan", stream, *args, int(H), int(max_seqlen), int(total), workspace,
          workspace.numel() * workspace.element_size(), outs[3])
    return outs


def dora_select_pack_residual(scores: torch.Tensor, keep: torch.Tensor, h: torch.Tensor, a: torch.Tensor,
                              cu_in: Optional[torch.Tensor] = None, N: Optional[int] = None,
                              idx_out: Optional[torch.Tensor] = None,
                              cu_out: Optional[torch.Tensor] = None,
                              packed_out: Optional[torch.Tensor] = None,
                              cap_rows: Optional[int] = None,
                              dev_status: Optional[torch.Tensor] = None,
                              stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """dora_select_pack of the attention residual h + a: the kept rows of the
    sum, each element rounded once to h's dtype.  a has h's shape and dtype."""
    if a.shape != h.shape or a.dtype != h.dtype:
        raise ValueError("a must have h's shape and dtype")
    args, outs = _select_pack_args(scores, keep, h, cu_in, N, idx_out, cu_out, packed_out,
                                   cap_rows, dev_status)
    args.insert(3, a)
    _call("dora_select_pack_residual", stream, *args, outs[3])
    return outs


def dora_actor_gate(p_gate: torch.Tensor, M: int, N: int, cu_in: Optional[torch.Tensor] = None,
                    on_rank: Optional[torch.Tensor] = None, on_list: Optional[torch.Tensor] = None,
                    n_on: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                    stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gate decisions and the ordered list of gate-on images.  p_gate: fp32 [B];
    N tokens per image (CLS included) or cu_in [B+1]; M budget-head outputs.
    Returns (on_rank [B], on_list [B], n_on [1], dev_status)."""
    B = int(p_gate.shape[0])
    dev = p_gate.device
    if cu_in is not None and tuple(cu_in.shape) != (B + 1,):
        raise ValueError("cu_in must be [B+1]")
    on_rank = torch.empty(B, dtype=torch.int32, device=dev) if on_rank is None else on_rank
    on_list = torch.empty(B, dtype=torch.int32, device=dev) if on_list is None else on_list
    n_on = torch.empty(1, dtype=torch.int32, device=dev) if n_on is None else n_on
    dev_status = new_status(dev) if dev_status is None else dev_status
    for t, name in ((on_rank, "on_rank"), (on_list, "on_list")):
        if t.numel() < B:
            raise ValueError(f"{name} needs {B} entries")
    _call("dora_actor_gate", stream, p_gate, cu_in, B, int(N), int(M), on_rank, on_list, n_on, dev_status)
    return on_rank, on_list, n_on, dev_status


def dora_actor_decode(budget_logits: torch.Tensor, on_rank: torch.Tensor, N: int,
                      removal_scores: Optional[torch.Tensor] = None, cu_in: Optional[torch.Tensor] = None,
                      keep_out: Optional[torch.Tensor] = None, scores_out: Optional[torch.Tensor] = None,
                      dev_status: Optional[torch.Tensor] = None,
                      stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """Keep counts from the budget logits [rows, M] (row r = gate-on image r)
    and, if removal_scores is given, keep-scores = -removal_scores in the same
    layout.  Returns (keep [B], keep-scores or None, dev_status)."""
    B = int(on_rank.shape[0])
    dev = on_rank.device
    if budget_logits.dim() != 2:
        raise ValueError("budget_logits must be [rows, M]")
    rows, M = int(budget_logits.shape[0]), int(budget_logits.shape[1])
    keep_out = torch.empty(B, dtype=torch.int32, device=dev) if keep_out is None else keep_out
    if removal_scores is not None and scores_out is None:
        scores_out = torch.empty_like(removal_scores)
    if (removal_scores is None) != (scores_out is None):
        raise ValueError("removal_scores and scores_out go together")
    if removal_scores is not None and scores_out.shape != removal_scores.shape:
        raise ValueError("scores_out must have removal_scores' shape")
    if cu_in is None:
        total_in = B * int(N)
        if removal_scores is not None and tuple(removal_scores.shape) != (B, int(N)):
            raise ValueError("dense removal_scores must be [B,N]")
    else:
        if tuple(cu_in.shape) != (B + 1,):
            raise ValueError("cu_in must be [B+1]")
        total_in = int(removal_scores.shape[0]) if removal_scores is not None else 0
    dev_status = new_status(dev) if dev_status is None else dev_status
    _call("dora_actor_decode", stream, budget_logits if rows > 0 else None, rows, M, removal_scores, cu_in, total_in,
          B, int(N), on_rank, keep_out, scores_out, dev_status)
    return keep_out, scores_out, dev_status


def _numel(t) -> int:
    return t.numel() if isinstance(t, torch.Tensor) else 0  # anything else is refused with the other arguments


def _pl_geometry(scores, B, cu_in, N):
    if cu_in is None:
        if scores.dim() != 2 or int(scores.shape[0]) != B:
            raise ValueError("dense scores must be [B,N]")
        return int(scores.shape[1]), B * int(scores.shape[1])
    if tuple(cu_in.shape) != (B + 1,) or scores.dim() != 1:
        raise ValueError("packed scores must be [total_in] with cu_in [B+1]")
    if N is None:
        raise ValueError("packed input needs N (an upper bound on segment lengths)")
    return int(N), int(scores.shape[0])


def dora_pl_sample(scores: torch.Tensor, gumbel: torch.Tensor, k: torch.Tensor,
                   cu_in: Optional[torch.Tensor] = None, N: Optional[int] = None,
                   order_out: Optional[torch.Tensor] = None, cu_order_out: Optional[torch.Tensor] = None,
                   logprob_out: Optional[torch.Tensor] = None, cap: Optional[int] = None,
                   dev_status: Optional[torch.Tensor] = None, stream=None):
    """Gumbel-top-k Plackett-Luce draws of k[b] visual tokens per image (removal
    scores + noise), in drawing order, and their ordered log-probability.
    Returns (order [cap], cu_order [B+1], logprob [B], dev_status)."""
    B = int(k.shape[0])
    N, total_in = _pl_geometry(scores, B, cu_in, N)
    if gumbel.shape != scores.shape:
        raise ValueError("gumbel must have the scores' shape")
    dev = scores.device
    cap = (int(order_out.numel()) if order_out is not None else B * max(N - 1, 1)) if cap is None else cap
    order_out = torch.empty(cap, dtype=torch.int32, device=dev) if order_out is None else order_out
    cu_order_out = torch.empty(B + 1, dtype=torch.int32, device=dev) if cu_order_out is None else cu_order_out
    logprob_out = torch.empty(B, dtype=torch.float32, device=dev) if logprob_out is None else logprob_out
    dev_status = new_status(dev) if dev_status is None else dev_status
    if order_out.numel() < cap:
        raise ValueError("order_out smaller than cap")
    _call("dora_pl_sample", stream, scores, gumbel, k, cu_in, total_in, B, N, order_out, cu_order_out, logprob_out,
          int(cap), dev_status)
    return order_out, cu_order_out, logprob_out, dev_status


def dora_pl_logprob(scores: torch.Tensor, order: torch.Tensor, cu_order: torch.Tensor,
                    cu_in: Optional[torch.Tensor] = None, N: Optional[int] = None,
                    logprob_out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                    stream=None):
    """Ordered log-probability of given draws (order, cu_order) under scores.
    Images whose draws lie past the end of order are reported
    (DORA_DEV_KEEP_RANGE).  Returns (logprob [B], dev_status)."""
    B = int(cu_order.shape[0]) - 1
    N, total_in = _pl_geometry(scores, B, cu_in, N)
    dev = scores.device
    logprob_out = torch.empty(B, dtype=torch.float32, device=dev) if logprob_out is None else logprob_out
    dev_status = new_status(dev) if dev_status is None else dev_status
    _call("dora_pl_logprob_cap", stream, scores, order, cu_order, _numel(order), cu_in, total_in, B, N, logprob_out,
          dev_status)
    return logprob_out, dev_status


def dora_lc1_readout_workspace_size(B: int, C: int) -> int:
    return int(load_library().dora_lc1_readout_workspace_size(int(B), int(C)))


def new_lc1_workspace(B: int, C: int, device=None) -> torch.Tensor:
    """A workspace for dora_lc1_readout (no required contents)."""
    n = dora_lc1_readout_workspace_size(B, C)
    if n == 0:
        raise DoraError("dora_lc1_readout_workspace_size", DORA_ERR_SHAPE)
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def dora_lc1_readout(x: torch.Tensor, cu_seqlens: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor,
                     eps: float = 1e-6, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, single: bool = False,
                     dev_status: Optional[torch.Tensor] = None, stream=None):
    """LayerNorm of each packed sequence's CLS row next to the mean LayerNorm of
    its other rows: x [total, C] bf16/fp32, cu_seqlens [B+1] -> out fp32 [B, 2C].
    With a workspace (a new one when None) a sequence's rows may be
    split over several workgroups; single=True passes none (one workgroup per
    sequence).  Returns (out, dev_status)."""
    if x.dim() != 2:
        raise ValueError("x must be [total, C]")
    B = int(cu_seqlens.shape[0]) - 1
    total, C = int(x.shape[0]), int(x.shape[1])
    out = torch.empty((B, 2 * C), dtype=torch.float32, device=x.device) if out is None else out
    dev_status = new_status(x.device) if dev_status is None else dev_status
    if tuple(out.shape) != (B, 2 * C):
        raise ValueError("out must be [B, 2C]")
    if not single and workspace is None:
        workspace = new_lc1_workspace(B, C, x.device)
    ws, ws_bytes = (None, 0) if single else (workspace, workspace.numel() * workspace.element_size())
    _call("dora_lc1_readout", stream, x, cu_seqlens, total, B, C, _dtype_code(x), gamma, beta, float(eps), out, ws,
          ws_bytes, dev_status)
    return out, dev_status


def dora_trajectory_flops(tokens: torch.Tensor, d: int, N0: int, patch: int, M: Optional[int] = None,
                          mlp_ratio: int = 4, in_chans: int = 3, classes: int = 1000, head_inputs: int = 1,
                          actor: bool = True, flops_out: Optional[torch.Tensor] = None,
                          total_out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                          stream=None):
    """FLOPs per image along realised token trajectories tokens [L+1, B] (int32).
    Returns (flops [B] int64, total [1] int64, dev_status)."""
    if tokens.dim() != 2:
        raise ValueError("tokens must be [L+1, B]")
    L, B = int(tokens.shape[0]) - 1, int(tokens.shape[1])
    cfg = FlopsConfig(int(d), L, int(N0), int(patch), int(in_chans), int(classes), int(head_inputs),
                      int(mlp_ratio), int((N0 - 4) // 2 if M is None else M), int(bool(actor)))
    dev = tokens.device
    flops_out = torch.empty(B, dtype=torch.int64, device=dev) if flops_out is None else flops_out
    total_out = torch.empty(1, dtype=torch.int64, device=dev) if total_out is None else total_out
    dev_status = new_status(dev) if dev_status is None else dev_status
    _call("dora_trajectory_flops", stream, tokens, B, ctypes.addressof(cfg), flops_out, total_out, dev_status)
    return flops_out, total_out, dev_status


def dora_varlen_attn_workspace_size(B: int, H: int, max_seqlen: int) -> int:
    return int(load_library().dora_varlen_attn_workspace_size(int(B), int(H), int(max_seqlen)))


def new_workspace(B: int, H: int, max_seqlen: int, device=None) -> torch.Tensor:
    n = dora_varlen_attn_workspace_size(B, H, max_seqlen)
    if n == 0:
        raise DoraError("dora_varlen_attn_workspace_size", DORA_ERR_SHAPE)
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def dora_varlen_attn_plan(cu_seqlens: torch.Tensor, H: int, max_seqlen: int, total: int,
                          workspace: torch.Tensor, dev_status: torch.Tensor, stream=None) -> None:
    B = int(cu_seqlens.shape[0]) - 1
    _call("dora_varlen_attn_plan", stream, cu_seqlens, B, int(H), int(max_seqlen), int(total), workspace,
          workspace.numel() * workspace.element_size(), dev_status)


def _attn_args(q, k, v, cu_seqlens, out):
    if q.dim() != 3 or q.shape != k.shape or q.shape != v.shape:
        raise ValueError("q, k, v must share the shape [total, H, 64]")
    if q.dtype != k.dtype or q.dtype != v.dtype:
        raise TypeError("q, k, v must share one dtype")
    total, H, D = (int(x) for x in q.shape)
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must match q")
    return total, H, D, out


def dora_varlen_attn_execute(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                             cu_seqlens: torch.Tensor, max_seqlen: int, workspace: torch.Tensor,
                             out: Optional[torch.Tensor] = None, softmax_scale: float = 0.0,
                             dev_status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    total, H, D, out = _attn_args(q, k, v, cu_seqlens, out)
    if dev_status is None:
        dev_status = new_status(q.device)
    B = int(cu_seqlens.shape[0]) - 1
    _call("dora_varlen_attn_execute", stream, q, k, v, cu_seqlens, B, H, D, int(max_seqlen), total, float(softmax_scale),
          _dtype_code(q), out, workspace, workspace.numel() * workspace.element_size(), dev_status)
    return out


def dora_varlen_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                     max_seqlen: int, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, softmax_scale: float = 0.0,
                     dev_status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """softmax(scale * Q K^T) V inside each packed sequence; q/k/v/out [total, H, 64]."""
    total, H, D, out = _attn_args(q, k, v, cu_seqlens, out)
    B = int(cu_seqlens.shape[0]) - 1
    if workspace is None:
        workspace = new_workspace(B, H, max_seqlen, q.device)
    if dev_status is None:
        dev_status = new_status(q.device)
    _call("dora_varlen_attn", stream, q, k, v, cu_seqlens, B, H, D, int(max_seqlen), total, float(softmax_scale),
          _dtype_code(q), out, workspace, workspace.numel() * workspace.element_size(), dev_status)
    return out


def dora_varlen_attn_noalloc(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                             max_seqlen: int, out: torch.Tensor, softmax_scale: float = 0.0,
                             dev_status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dora_varlen_attn with the library's static per-GPU workspace: no device
    allocation in the call (out and dev_status must be given).  Calls that
    overlap in time on one GPU race on that workspace."""
    if out is None or dev_status is None:
        raise ValueError("dora_varlen_attn_noalloc allocates nothing: pass out and dev_status")
    lib = load_library()
    total, H, D, out = _attn_args(q, k, v, cu_seqlens, out)
    B = int(cu_seqlens.shape[0]) - 1
    rc = lib.dora_varlen_attn_noalloc(
        _dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(cu_seqlens, "cu_seqlens", torch.int32),
        B, H, D, int(max_seqlen), total, float(softmax_scale), _dtype_code(q), _dev(out, "out"),
        _dev(dev_status, "dev_status", torch.int32), _stream(stream))
    _check("dora_varlen_attn_noalloc", rc)
    return out


def _in_stream(stream):
    """The context of a given stream: what a call allocates and clears belongs to
    the stream that it runs on."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _rows(t: torch.Tensor, name: str):
    """Address, leading dimension, sizes, type and device of rows whose elements
    are adjacent."""
    got = (_native_rows or _leave_to_ctypes)(t)
    if got is not NotImplemented:
        return got
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.layout != torch.strided or t.is_nested:
        raise ValueError(f"{name} must be a strided tensor, not a sparse or nested one")
    if t.dim() != 2:
        raise ValueError(f"{name} must be [T, V]")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    T, V = t.shape
    ld, one = t.stride()
    if T <= 1:
        ld = V
    if (V > 1 and one != 1) or ld < V:
        raise ValueError(f"{name} must have adjacent elements in each row, and rows apart")
    return t.data_ptr(), ld, T, V, _dtype_code(t), t.get_device()


def _vectors(names, device: int, *sized) -> None:
    """The tensors of a call (n, tensor, n, tensor, ...) are vectors of n elements
    (n < 0: any tensor) on the device, the current one, whose stream runs it."""
    if (_native_vectors or _leave_to_ctypes)(device, *sized) is NotImplemented:
        for name, n, t in zip(names, sized[::2], sized[1::2]):
            if t is None:
                continue
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch tensor")
            if n >= 0 and tuple(t.shape) != (n,):
                raise ValueError(f"{name} must be [{n}]")
            if t.get_device() != device:
                raise ValueError(f"tensors on devices {device} and {t.get_device()} (-1: the host): {name}")
    if device >= 0 and device != torch._C._cuda_getDevice():
        raise ValueError(f"tensors on device {device}, which is not the current one")


def _written(*outputs) -> None:
    """Tensors (or lists of them) that a call wrote by their addresses: autograd
    refuses a backward pass that saved one of them, as after torch's own
    in-place operators."""
    if (_native_written or _leave_to_ctypes)(*outputs) is NotImplemented:
        for t in outputs:
            torch.autograd.graph.increment_version(t)


def _bytes(workspace: Optional[torch.Tensor]) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def _new_bytes(fn: str, n: int, device) -> torch.Tensor:
    if n == 0:
        raise DoraError(fn, DORA_ERR_SHAPE)
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def dora_policy_workspace_size(T: int, V: int) -> int:
    return int(load_library().dora_policy_workspace_size(int(T), int(V)))


def new_policy_workspace(T: int, V: int, device=None) -> torch.Tensor:
    """A workspace for dora_policy_loss and dora_action_logprob (no required contents)."""
    return _new_bytes("dora_policy_workspace_size", dora_policy_workspace_size(T, V), device)


def dora_action_logprob(logits: torch.Tensor, actions: torch.Tensor, weight: Optional[torch.Tensor] = None,
                        legal: Optional[torch.Tensor] = None, logprob_out: Optional[torch.Tensor] = None,
                        entropy_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        single: bool = False, dev_status: Optional[torch.Tensor] = None, stream=None):
    """Log-probability of each row's action, and the entropy of its choice.

    logits: [T, V] bf16 or fp32, elements of a row adjacent, rows any distance
    apart; actions: int32 [T]; legal: int32 [T], the first legal[t] choices are
    open; weight: fp32 [T], rows of weight 0 are padding (results 0).  With a
    workspace (a new one when None) few long rows may be split over several
    workgroups; single=True passes none.  Returns (logprob [T], entropy [T],
    dev_status)."""
    if stream is not None:
        with _in_stream(stream):
            return dora_action_logprob(logits, actions, weight, legal, logprob_out, entropy_out, workspace, single,
                                       dev_status)
    address, ld, T, V, code, device = _rows(logits, "logits")
    dev = logits.device
    logprob_out = torch.empty(T, dtype=torch.float32, device=dev) if logprob_out is None else logprob_out
    entropy_out = torch.empty(T, dtype=torch.float32, device=dev) if entropy_out is None else entropy_out
    if single:
        workspace = None
    elif workspace is None:
        workspace = new_policy_workspace(T, V, dev)
    dev_status = new_status(dev) if dev_status is None else dev_status
    _vectors(("actions", "legal", "weight", "logprob_out", "entropy_out", "workspace", "dev_status"), device,
             T, actions, T, legal, T, weight, T, logprob_out, T, entropy_out, -1, workspace, -1, dev_status)
    _call("dora_action_logprob", None, address, ld, actions, legal, weight, T, V, code, logprob_out, entropy_out,
          workspace, _bytes(workspace), dev_status)
    _written(logprob_out, entropy_out)
    return logprob_out, entropy_out, dev_status


def dora_policy_loss(logits: torch.Tensor, actions: torch.Tensor, old_logprob: torch.Tensor, advantage: torch.Tensor,
                     ref_logprob: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                     legal: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2,
                     kl_coef: float = 0.0, entropy_coef: float = 0.0, dlogits: Optional[torch.Tensor] = None,
                     logprob_out: Optional[torch.Tensor] = None, stats_out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None, stream=None):
    """The clipped policy loss of T decisions and its gradient.

    logits, actions, weight and legal as for dora_action_logprob; old_logprob,
    advantage and ref_logprob (needed for kl_coef != 0): fp32 [T].  The loss is
    the sum over rows of weight * (-min(r A, clip(r) A) + kl_coef * kl -
    entropy_coef * entropy); for a mean, weight is 1 / count.  dlogits may be
    the logits themselves; logits.backward(dlogits) carries it on.  Returns
    (dlogits [T, V], logprob [T], stats [6], dev_status); stats holds the sums
    of loss, gain, kl, entropy, clipped share and weight."""
    if stream is not None:
        with _in_stream(stream):
            return dora_policy_loss(logits, actions, old_logprob, advantage, ref_logprob, weight, legal, clip_low,
                                    clip_high, kl_coef, entropy_coef, dlogits, logprob_out, stats_out, workspace,
                                    dev_status)
    address, ld, T, V, code, device = _rows(logits, "logits")
    dev = logits.device
    dlogits = torch.empty((T, V), dtype=logits.dtype, device=dev) if dlogits is None else dlogits
    grad, ld_grad, *like = _rows(dlogits, "dlogits")
    if like != [T, V, code, device]:
        raise ValueError("dlogits must have the logits' shape, type and device")
    logprob_out = torch.empty(T, dtype=torch.float32, device=dev) if logprob_out is None else logprob_out
    stats_out = torch.empty(6, dtype=torch.float32, device=dev) if stats_out is None else stats_out
    workspace = new_policy_workspace(T, V, dev) if workspace is None else workspace
    dev_status = new_status(dev) if dev_status is None else dev_status
    _vectors(("actions", "legal", "old_logprob", "ref_logprob", "advantage", "weight", "logprob_out", "stats_out",
              "workspace", "dev_status"), device, T, actions, T, legal, T, old_logprob, T, ref_logprob, T, advantage,
             T, weight, T, logprob_out, 6, stats_out, -1, workspace, -1, dev_status)
    _call("dora_policy_loss", None, address, ld, actions, legal, old_logprob, ref_logprob, advantage, weight, T, V,
          code, float(clip_low), float(clip_high), float(kl_coef), float(entropy_coef), grad, ld_grad, logprob_out,
          stats_out, workspace, _bytes(workspace), dev_status)
    _written(dlogits, logprob_out, stats_out)
    return dlogits, logprob_out, stats_out, dev_status


def dora_pl_policy_workspace_size(B: int) -> int:
    return int(load_library().dora_pl_policy_workspace_size(int(B)))


def new_pl_policy_workspace(B: int, device=None) -> torch.Tensor:
    """A workspace for dora_pl_policy_loss (no required contents)."""
    return _new_bytes("dora_pl_policy_workspace_size", dora_pl_policy_workspace_size(B), device)


def dora_pl_policy_loss(scores: torch.Tensor, order: torch.Tensor, cu_order: torch.Tensor, old_logprob: torch.Tensor,
                        advantage: torch.Tensor, ref_logprob: Optional[torch.Tensor] = None,
                        weight: Optional[torch.Tensor] = None, cu_in: Optional[torch.Tensor] = None,
                        N: Optional[int] = None, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                        dscores: Optional[torch.Tensor] = None, logprob_out: Optional[torch.Tensor] = None,
                        stats_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        dev_status: Optional[torch.Tensor] = None, stream=None):
    """The clipped policy loss of ordered Plackett-Luce draws and its gradient
    with respect to the removal scores: scores, order, cu_order, cu_in and N as
    for dora_pl_logprob, the rest as for dora_policy_loss, one entry per image.
    Returns (dscores in the scores' layout, logprob [B], stats [6],
    dev_status)."""
    if stream is not None:
        with _in_stream(stream):
            return dora_pl_policy_loss(scores, order, cu_order, old_logprob, advantage, ref_logprob, weight, cu_in, N,
                                       clip_low, clip_high, kl_coef, dscores, logprob_out, stats_out, workspace,
                                       dev_status)
    B = int(cu_order.shape[0]) - 1
    N, total_in = _pl_geometry(scores, B, cu_in, N)
    dev = scores.device
    dscores = torch.empty_like(scores) if dscores is None else dscores
    if dscores.shape != scores.shape:
        raise ValueError("dscores must be of the scores' shape")
    logprob_out = torch.empty(B, dtype=torch.float32, device=dev) if logprob_out is None else logprob_out
    stats_out = torch.empty(6, dtype=torch.float32, device=dev) if stats_out is None else stats_out
    workspace = new_pl_policy_workspace(B, dev) if workspace is None else workspace
    dev_status = new_status(dev) if dev_status is None else dev_status
    _vectors(("old_logprob", "ref_logprob", "advantage", "weight", "logprob_out", "stats_out", "order", "cu_order",
              "cu_in", "dscores", "workspace", "dev_status"), scores.get_device(), B, old_logprob, B, ref_logprob,
             B, advantage, B, weight, B, logprob_out, 6, stats_out, -1, order, B + 1, cu_order, B + 1, cu_in,
             -1, dscores, -1, workspace, -1, dev_status)
    _call("dora_pl_policy_loss_cap", None, scores, order, cu_order, _numel(order), cu_in, total_in, old_logprob,
          ref_logprob, advantage, weight, B, N, float(clip_low), float(clip_high), float(kl_coef), dscores, logprob_out,
          stats_out, workspace, _bytes(workspace), dev_status)
    _written(dscores, logprob_out, stats_out)
    return dscores, logprob_out, stats_out, dev_status


def dora_grad_clip_workspace_size(n: int) -> int:
    return int(load_library().dora_grad_clip_workspace_size(int(n)))


def new_grad_clip_workspace(n: int, device=None) -> torch.Tensor:
    """A workspace for dora_grad_clip over n tensors (no required contents)."""
    return _new_bytes("dora_grad_clip_workspace_size", dora_grad_clip_workspace_size(n), device)


def _spans(tensors, name: str):
    """The tensors' spans and the device that holds them."""
    tensors = list(tensors)
    spans = (Span * len(tensors))()
    if not tensors:
        raise ValueError(f"{name} is empty")
    load_library()
    device = _native_spans(tensors, ctypes.addressof(spans))
    if device is NotImplemented:
        for i, t in enumerate(tensors):
            spans[i] = Span(_dev(t, f"{name}[{i}]"), t.numel(), _dtype_code(t), 0)
        device = tensors[0].get_device()
        _vectors([f"{name}[{i}]" for i in range(len(tensors))], device, *(x for t in tensors for x in (-1, t)))
    return spans, device


def dora_grad_clip(grads, max_norm: float, out=None, eps: float = 1e-6, norm_out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None):
    """Scale gradient tensors so that their global norm is at most max_norm.

    grads: contiguous bf16 or fp32 tensors, types may be mixed; out: tensors of
    the same sizes and types, or None: in place.  Every tensor is multiplied by
    min(1, max_norm / (norm + eps)), or 1 with max_norm = infinity, where in
    place only the norm is formed.  Returns (out, norm [1] fp32)."""
    if stream is not None:
        with _in_stream(stream):
            return dora_grad_clip(grads, max_norm, out, eps, norm_out, workspace)
    grads = list(grads)
    spans, device = _spans(grads, "grads")
    out_spans = None
    if out is not None:
        out = list(out)
        if len(out) != len(grads):
            raise ValueError("out must have a tensor for each of grads")
        out_spans, out_device = _spans(out, "out")
        if out_device != device:
            raise ValueError(f"tensors on devices {device} and {out_device}")
    dev = grads[0].device
    norm_out = torch.empty(1, dtype=torch.float32, device=dev) if norm_out is None else norm_out
    workspace = new_grad_clip_workspace(len(grads), dev) if workspace is None else workspace
    _vectors(("norm_out", "workspace"), device, 1, norm_out, -1, workspace)
    _call("dora_grad_clip", None, ctypes.addressof(spans), 0 if out_spans is None else ctypes.addressof(out_spans),
          len(grads), float(max_norm), float(eps), norm_out, workspace, _bytes(workspace))
    scaled = grads if out is None else out
    _written([] if out is None and max_norm == math.inf else scaled, norm_out)
    return scaled, norm_out


def _describe(names, *tensors):
    """Descriptions (dora_rows) of tensors [rows, heads, dim] or [rows, dim], the
    address of each (0 for None) and their device, which is the current one."""
    load_library()
    rows = (Rows * len(tensors))()
    at = ctypes.addressof(rows)
    device = _native_describe(at, *tensors)
    if device is NotImplemented:
        device = -1
        for i, (name, t) in enumerate(zip(names, tensors)):
            if t is None:
                continue
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch tensor")
            if t.layout != torch.strided or t.is_nested:
                raise ValueError(f"{name} must be a strided tensor, not a sparse or nested one")
            if t.dim() not in (2, 3):
                raise ValueError(f"{name} must be [rows, dim] or [rows, heads, dim]")
            if not t.is_cuda:
                raise ValueError(f"{name} must be on the GPU")
            if t.shape[-1] > 1 and t.stride(-1) != 1:
                raise ValueError(f"{name} must have adjacent elements in each row")
            if max(t.shape[1:]) > 0x7FFFFFFF:
                raise ValueError(f"{name} is too wide")
            if device >= 0 and t.get_device() != device:
                raise ValueError(f"tensors on devices {device} and {t.get_device()}: {name}")
            device = t.get_device()
            heads = int(t.shape[1]) if t.dim() == 3 else 1
            rows[i] = Rows(t.data_ptr(), t.shape[0], heads, t.shape[-1], t.stride(0), t.stride(1) if t.dim() == 3 else 0,
                           _dtype_code(t), 0)
    if device >= 0 and device != torch._C._cuda_getDevice():
        raise ValueError(f"tensors on device {device}, which is not the current one")
    size = ctypes.sizeof(Rows)
    return rows, [0 if t is None else at + i * size for i, t in enumerate(tensors)], device


def _like(t: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of t's shape and type."""
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _heads(names, *tensors) -> None:
    for name, t in zip(names, tensors):
        if t is not None and not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch tensor")
        if t is not None and t.dim() != 3:
            raise ValueError(f"{name} must be [rows, heads, dim]")


def rope_frequencies(R: int, base: float = 10000.0, factor: float = 1.0, trained: Optional[int] = None,
                     few: float = 1.0, many: float = 32.0, device=None) -> torch.Tensor:
    """Angles a position for dora_rope: float64 [R / 2], base^(-2 i / R).

    For contexts `factor` times the `trained` length, pairs are interpolated
    (divided by factor) where they turn fewer than `few` times in that length,
    left alone where more than `many` times, and blended linearly between; all
    are interpolated without `trained`."""
    if R < 2 or R % 2 or base <= 0 or factor <= 0 or (trained is not None and (trained < 1 or few >= many)):
        raise ValueError("R must be even, base and factor positive, trained at least 1 and few below many")
    freq = torch.tensor(float(base), dtype=torch.float64) ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R)
    if factor != 1.0:
        keep = 0.0
        if trained is not None:
            keep = ((trained * freq / (2 * math.pi) - few) / (many - few)).clamp(0.0, 1.0)
        freq = freq * keep + freq / factor * (1.0 - keep)
    return freq.to(device or "cuda")


def dora_rope(q: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, k: Optional[torch.Tensor] = None,
              interleaved: bool = False, inverse: bool = False, scale: float = 1.0, q_out: Optional[torch.Tensor] = None,
              k_out: Optional[torch.Tensor] = None, stream=None):
    """Rotary positions of q [rows, H, D] and k [rows, Hk, D] (bf16 or fp32, any
    strides between rows and heads).

    positions: int32 [rows] or [rows, axes], each axis for its share of the pairs
    in turn; freq: float64 [R / 2], radians per position (rope_frequencies); the
    first R elements of each head are turned, in pairs (i, i + R / 2) or,
    interleaved, (2 i, 2 i + 1), and multiplied by scale.  inverse turns back:
    the gradient.  q_out and k_out may be q and k.  Returns (q_out, k_out)."""
    if stream is not None:
        with _in_stream(stream):
            return dora_rope(q, positions, freq, k, interleaved, inverse, scale, q_out, k_out)
    _heads(("q", "k"), q, k)
    if k is None and k_out is not None:
        raise ValueError("k_out goes with k")
    for name, t in (("positions", positions), ("freq", freq)):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch tensor")
    axes = 1 if positions.dim() == 1 else int(positions.shape[-1])
    if positions.dim() not in (1, 2) or int(positions.shape[0]) != int(q.shape[0]) or freq.dim() != 1:
        raise ValueError("positions must be [rows] or [rows, axes], freq [R / 2]")
    if freq.dtype != torch.float64:
        raise TypeError(f"freq must be {torch.float64}, got {freq.dtype}")
    q_out = _like(q) if q_out is None else q_out
    k_out = _like(k) if k is not None and k_out is None else k_out
    rows, at, device = _describe(("q", "k", "q_out", "k_out"), q, k, q_out, k_out)
    _vectors(("positions", "freq"), device, -1, positions, -1, freq)
    _call("dora_rope", None, at[0], at[1], positions, axes, freq, 2 * freq.numel(), int(bool(interleaved)),
          int(bool(inverse)), float(scale), at[2], at[3])
    _written(q_out) if k_out is None else _written(q_out, k_out)
    return q_out, k_out


def dora_grouped_attn_workspace_size(B: int, H: int, Hk: int, D: int, max_q: int, total_q: int, total_k: int) -> int:
    return int(load_library().dora_grouped_attn_workspace_size(B, H, Hk, D, max_q, total_q, total_k))


def dora_grouped_attn_backward_workspace_size(B: int, H: int, Hk: int, D: int, max_q: int, total_q: int,
                                              total_k: int) -> int:
    return int(load_library().dora_grouped_attn_backward_workspace_size(B, H, Hk, D, max_q, total_q, total_k))


def new_grouped_attn_workspace(B: int, H: int, Hk: int, D: int, max_q: int, total_q: int, total_k: int,
                               backward: bool = False, device=None) -> torch.Tensor:
    """A workspace for dora_grouped_attn, and with `backward` for its backward pass too (no required contents)."""
    sizes = (int(B), int(H), int(Hk), int(D), int(max_q), int(total_q), int(total_k))
    n = dora_grouped_attn_workspace_size(*sizes)
    if backward:
        n = max(n, dora_grouped_attn_backward_workspace_size(*sizes))
    return _new_bytes("dora_grouped_attn_workspace_size", n, device)


def _sequences(cu_q, cu_k):
    if not isinstance(cu_q, torch.Tensor) or cu_q.dim() != 1 or cu_q.numel() < 2:
        raise ValueError("cu_q must be [B + 1]")
    return int(cu_q.shape[0]) - 1, cu_q if cu_k is None else cu_k


def dora_grouped_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, max_q: int,
                      cu_k: Optional[torch.Tensor] = None, causal: bool = False, softmax_scale: float = 0.0,
                      out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, keep_lse: bool = True,
                      workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None, stream=None,
                      max_k: int = 0):
    """softmax(scale q k^T) v inside packed sequences with grouped heads.

    q: [total_q, H, D]; k, v: [total_k, Hk, D], H a multiple of Hk, D 32, 64 or
    128, bf16 or fp32, any strides of 16 bytes; cu_q, cu_k (cu_q when None):
    int32 [B + 1]; max_q: no sequence has more queries.  causal: query i of nq
    sees the keys j <= i + nk - nq, so one new token sees all.  max_k: no
    sequence has more keys (0: not known); short lists then take one launch.
    Returns (out [total_q, H, D], lse [total_q, H] fp32 or None without keep_lse,
    dev_status)."""
    if stream is not None:
        with _in_stream(stream):
            return dora_grouped_attn(q, k, v, cu_q, max_q, cu_k, causal, softmax_scale, out, lse_out, keep_lse,
                                     workspace, dev_status, max_k=max_k)
    _heads(("q", "k", "v"), q, k, v)
    B, cu_k = _sequences(cu_q, cu_k)
    dev = q.device
    out = _like(q) if out is None else out
    total_q, H, D = q.shape
    if lse_out is None and keep_lse:
        lse_out = torch.empty((total_q, H), dtype=torch.float32, device=dev)
    if lse_out is not None and lse_out.shape != q.shape[:2]:
        raise ValueError("lse_out must be [total_q, H]")
    if workspace is None:
        workspace = new_grouped_attn_workspace(B, H, k.shape[1], D, max_q, total_q, k.shape[0], device=dev)
    dev_status = new_status(dev) if dev_status is None else dev_status
    rows, at, device = _describe(("q", "k", "v", "out"), q, k, v, out)
    _vectors(("cu_q", "cu_k", "lse_out", "workspace", "dev_status"), device, B + 1, cu_q, B + 1, cu_k, -1, lse_out,
             -1, workspace, -1, dev_status)
    _call("dora_grouped_attn", None, at[0], at[1], at[2], cu_q, cu_k, B, int(max_q), int(max_k),
          int(bool(causal)), float(softmax_scale), at[3], lse_out, workspace, _bytes(workspace), dev_status)
    _written(out) if lse_out is None else _written(out, lse_out)
    return out, lse_out, dev_status


def dora_grouped_attn_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                               out: torch.Tensor, lse: torch.Tensor, cu_q: torch.Tensor, max_q: int,
                               cu_k: Optional[torch.Tensor] = None, causal: bool = False, softmax_scale: float = 0.0,
                               dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                               dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                               dev_status: Optional[torch.Tensor] = None, stream=None):
    """Gradients of dora_grouped_attn from the output's, dout: out and lse as the
    forward call returned them, the other arguments as it had them.  dq, dk and
    dv may be slices of one tensor.  Returns (dq, dk, dv, dev_status)."""
    if stream is not None:
        with _in_stream(stream):
            return dora_grouped_attn_backward(dout, q, k, v, out, lse, cu_q, max_q, cu_k, causal, softmax_scale, dq, dk,
                                              dv, workspace, dev_status)
    _heads(("q", "k", "v"), q, k, v)
    B, cu_k = _sequences(cu_q, cu_k)
    dev = q.device
    dq, dk, dv = (_like(t) if g is None else g for t, g in ((q, dq), (k, dk), (v, dv)))
    total_q, H, D = q.shape
    if not isinstance(lse, torch.Tensor) or lse.shape != q.shape[:2]:
        raise ValueError("lse must be [total_q, H]")
    if workspace is None:
        n = dora_grouped_attn_backward_workspace_size(B, H, k.shape[1], D, int(max_q), total_q, k.shape[0])
        workspace = _new_bytes("dora_grouped_attn_backward_workspace_size", n, dev)
    dev_status = new_status(dev) if dev_status is None else dev_status
    rows, at, device = _describe(("dout", "q", "k", "v", "out", "dq", "dk", "dv"), dout, q, k, v, out, dq, dk, dv)
    _vectors(("lse", "cu_q", "cu_k", "workspace", "dev_status"), device, -1, lse, B + 1, cu_q, B + 1, cu_k, -1, workspace,
             -1, dev_status)
    _call("dora_grouped_attn_backward", None, *at[:5], lse, cu_q, cu_k, B, int(max_q), int(bool(causal)),
          float(softmax_scale), *at[5:], workspace, _bytes(workspace), dev_status)
    _written(dq, dk, dv)
    return dq, dk, dv, dev_status


def dora_residual_norm_workspace_size(T: int, C: int) -> int:
    return int(load_library().dora_residual_norm_workspace_size(int(T), int(C)))


def new_residual_norm_workspace(T: int, C: int, device=None) -> torch.Tensor:
    """A workspace for dora_residual_norm_backward (no required contents)."""
    return _new_bytes("dora_residual_norm_workspace_size", dora_residual_norm_workspace_size(T, C), device)


_NORM_KINDS = {"layer": DORA_NORM_LAYER, "rms": DORA_NORM_RMS}


def _norm_kind(kind: str) -> int:
    if kind not in _NORM_KINDS:
        raise ValueError(f"kind must be 'layer' or 'rms', not {kind!r}")
    return _NORM_KINDS[kind]


def _matrix(t, name: str):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must be [T, C]")
    return int(t.shape[0]), int(t.shape[1])


def dora_residual_norm(x: torch.Tensor, a: Optional[torch.Tensor], gamma: torch.Tensor,
                       beta: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                       gate: Optional[torch.Tensor] = None, post_gamma: Optional[torch.Tensor] = None,
                       post_beta: Optional[torch.Tensor] = None, kind: str = "layer", eps: float = 1e-6,
                       h_out: Optional[torch.Tensor] = None, y_out: Optional[torch.Tensor] = None, stream=None):
    """h = x + gate scale u and y = norm(h), u the branch's output a or (with
    post_gamma) its norm.

    x, a: [T, C] bf16 or fp32, C at most 8192, rows a multiple of 16 bytes and any
    distance of such apart; a None: the norm of x alone.  gamma, beta, scale (layer
    scale), post_gamma, post_beta: fp32 [C]; gate: fp32 [T], 0 drops a row's branch.
    kind: "layer" or "rms".  h_out and y_out may be x or a.  Returns (h, y); h is x
    itself without a."""
    if stream is not None:
        with _in_stream(stream):
            return dora_residual_norm(x, a, gamma, beta, scale, gate, post_gamma, post_beta, kind, eps, h_out, y_out)
    T, C = _matrix(x, "x")
    code = _norm_kind(kind)
    h_out = _like(x) if h_out is None and a is not None else h_out
    y_out = _like(x) if y_out is None else y_out
    rows, at, device = _describe(("x", "a", "h_out", "y_out"), x, a, h_out, y_out)
    _vectors(_NORM, device, C, gamma, C, beta, C, scale, T, gate, C, post_gamma, C, post_beta)
    _call("dora_residual_norm", None, at[0], at[1], gamma, beta, scale, gate, post_gamma, post_beta, code, float(eps),
          at[2], at[3])
    _written(y_out) if h_out is None else _written(h_out, y_out)
    return x if h_out is None else h_out, y_out


class ResidualNormGrads(NamedTuple):
    """Gradients of dora_residual_norm's arguments; None where it had none."""
    dx: torch.Tensor
    da: Optional[torch.Tensor]
    dgamma: torch.Tensor
    dbeta: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dpost_gamma: Optional[torch.Tensor]
    dpost_beta: Optional[torch.Tensor]


def dora_residual_norm_backward(dy: Optional[torch.Tensor], h: torch.Tensor, a: Optional[torch.Tensor],
                                gamma: torch.Tensor, beta: Optional[torch.Tensor] = None,
                                scale: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                                post_gamma: Optional[torch.Tensor] = None, post_beta: Optional[torch.Tensor] = None,
                                dh: Optional[torch.Tensor] = None, kind: str = "layer", eps: float = 1e-6,
                                dx: Optional[torch.Tensor] = None, da: Optional[torch.Tensor] = None,
                                dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None,
                                dscale: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                                dpost_gamma: Optional[torch.Tensor] = None, dpost_beta: Optional[torch.Tensor] = None,
                                workspace: Optional[torch.Tensor] = None, stream=None) -> ResidualNormGrads:
    """Gradients of dora_residual_norm from those of y (dy) and of h (dh; either
    may be None), for the h that it returned.  The branch's gradient is dx itself
    where it has neither scale, gate nor norm (and da is None).  dx and da may be
    dy, dh, h or a.  The parameters' gradients are fp32 in their shapes."""
    if stream is not None:
        with _in_stream(stream):
            return dora_residual_norm_backward(dy, h, a, gamma, beta, scale, gate, post_gamma, post_beta, dh, kind, eps, dx,
                                               da, dgamma, dbeta, dscale, dgate, dpost_gamma, dpost_beta, workspace)
    T, C = _matrix(h, "h")
    code = _norm_kind(kind)
    dx = _like(h) if dx is None else dx
    same = a is not None and da is None and scale is None and gate is None and post_gamma is None
    if a is not None and da is None and not same:
        da = _like(h)
    workspace = new_residual_norm_workspace(T, C, h.device) if workspace is None else workspace
    grads = [dgamma, dbeta, dscale, dgate, dpost_gamma, dpost_beta]
    sizes = (C, C, C, T, C, C)
    for i, (t, name) in enumerate(zip((gamma, beta, scale, gate, post_gamma, post_beta), _NORM_GRADS)):
        if t is None and grads[i] is not None:
            raise ValueError(f"{name} without {name[1:]}")
        if t is not None and grads[i] is None:
            grads[i] = torch.empty(sizes[i], dtype=torch.float32, device=h.device)
    rows, at, device = _describe(("dy", "dh", "h", "a", "dx", "da"), dy, dh, h, a, dx, da)
    if same:  # not read, but a's gradient has its sizes and type
        if a.shape != h.shape or a.dtype != h.dtype:
            raise DoraError("dora_residual_norm_backward", DORA_ERR_SHAPE if a.shape != h.shape else DORA_ERR_DTYPE)
        at[3] = 0
    _vectors(_NORM + ("workspace",) + _NORM_GRADS, device, C, gamma, C, beta, C, scale, T, gate, C, post_gamma, C,
             post_beta, -1, workspace, *(x for pair in zip(sizes, grads) for x in pair))
    _call("dora_residual_norm_backward", None, *at[:4], gamma, scale, gate, post_gamma, post_beta, code,
          float(eps), at[4], at[5], *grads, workspace, _bytes(workspace))
    _written(*(t for t in (dx, da, *grads) if t is not None))
    return ResidualNormGrads(dx, dx if same else da, *grads)
