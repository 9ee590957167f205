"""Binding of libdetox.so (ctypes; for the worker-side operators a compiled module): argument marshalling only.

Every function has the name and the meaning of the C entry point in include/detox.h.  Tensors are
torch CUDA tensors used as device memory; matrices may be column-sliced views (the row stride is
passed as `ld`).  Output and workspace buffers are created here when the caller passes none.  There
is no CPU path: if the library is not built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdetox.so")

AGG_NONE, AGG_MEAN, AGG_COORD_MEDIAN, AGG_MULTIKRUM, AGG_BULYAN, AGG_TRIMMED_MEAN, AGG_GEOMETRIC_MEDIAN, AGG_SIGN_MAJORITY = range(8)
MAX_ROWS, MAX_R = 1024, 15

EXPORTS = (
    "detox_status_string", "detox_vote_workspace_bytes", "detox_vote", "detox_vote_noalloc", "detox_hier_mean",
    "detox_vote_hier_mean",
    "agg_coord_median_workspace_bytes", "agg_coord_median", "agg_trimmed_mean", "agg_sign_majority", "agg_geometric_median_workspace_bytes", "agg_geometric_median", "agg_multikrum_workspace_bytes", "agg_multikrum",
    "agg_bulyan_workspace_bytes", "agg_bulyan", "detox_aggregate_workspace_bytes", "detox_aggregate",
    "detox_selftest_bounded_wait", "agg_pairwise_sqdist_workspace_bytes", "agg_pairwise_sqdist",
    "detox_kernel_launch_count", "detox_vote_hier_mean_many", "detox_tc_split_mode", "detox_tc_repeated_passes",
    "detox_checkpoint_pack", "detox_checkpoint_unpack", "detox_rmsnorm", "detox_rmsnorm_backward_workspace_bytes",
    "detox_rmsnorm_backward", "detox_gated_workspace_bytes", "detox_gated", "detox_gated_backward_workspace_bytes",
    "detox_gated_backward", "detox_gated_expired_waits", "detox_gated_wait_limit",
    "detox_embedding", "detox_embedding_backward_workspace_bytes", "detox_embedding_backward", "detox_token_logp",
    "detox_token_logp_backward", "detox_policy_loss_workspace_bytes", "detox_policy_loss",
    "detox_preference_loss_workspace_bytes", "detox_preference_loss", "detox_adamw",
)


class DetoxError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {status_string(code)} (status {code})")


class PipelineDesc(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int32), ("r", ctypes.c_int32), ("d", ctypes.c_int64),
        ("members", ctypes.POINTER(ctypes.c_int32)),
        ("a0", ctypes.c_int32), ("n_sets", ctypes.c_int32),
        ("set_offsets", ctypes.POINTER(ctypes.c_int32)), ("set_members", ctypes.POINTER(ctypes.c_int32)),
        ("a1", ctypes.c_int32), ("f", ctypes.c_int32), ("m_sel", ctypes.c_int32),
        ("gm_iters", ctypes.c_int32), ("gm_eps", ctypes.c_float),
    ]


class GatedDesc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
        ("tokens", ctypes.c_int64), ("in_dim", ctypes.c_int64), ("hidden", ctypes.c_int64),
        ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64),
        ("XQ", ctypes.c_void_p), ("ldxq", ctypes.c_int64), ("XE", ctypes.c_void_p), ("ldxe", ctypes.c_int64),
        ("Wg", ctypes.c_void_p), ("ldwg", ctypes.c_int64), ("Wu", ctypes.c_void_p), ("ldwu", ctypes.c_int64),
        ("GQ", ctypes.c_void_p), ("GE", ctypes.c_void_p), ("UQ", ctypes.c_void_p), ("UE", ctypes.c_void_p),
        ("ldq", ctypes.c_int64), ("lde", ctypes.c_int64),
    ]


class PolicyDesc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("index", ctypes.c_int32), ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64),
        ("Z", ctypes.c_void_p), ("ldz", ctypes.c_int64), ("y", ctypes.c_void_p), ("old_logp", ctypes.c_void_p),
        ("advantage", ctypes.c_void_p), ("ref_logp", ctypes.c_void_p), ("weight", ctypes.c_void_p),
        ("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float), ("kl_coef", ctypes.c_float), ("scale", ctypes.c_float),
        ("grad_scale", ctypes.c_float),
    ]


class PreferenceDesc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("index", ctypes.c_int32), ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64),
        ("pairs", ctypes.c_int64), ("Z", ctypes.c_void_p), ("ldz", ctypes.c_int64), ("y", ctypes.c_void_p),
        ("offsets", ctypes.c_void_p), ("ref", ctypes.c_void_p), ("beta", ctypes.c_float), ("smoothing", ctypes.c_float),
        ("scale", ctypes.c_float), ("grad_scale", ctypes.c_float),
    ]


class AdamWTensor(ctypes.Structure):
    _fields_ = [
        ("P", ctypes.c_void_p), ("G", ctypes.c_void_p), ("master", ctypes.c_void_p), ("M", ctypes.c_void_p), ("ME", ctypes.c_void_p),
        ("V", ctypes.c_void_p), ("VE", ctypes.c_void_p), ("n", ctypes.c_int64), ("p_dtype", ctypes.c_int32),
        ("g_dtype", ctypes.c_int32), ("weight_decay", ctypes.c_float), ("key", ctypes.c_uint32),
    ]


class AdamWDesc(ctypes.Structure):
    _fields_ = [
        ("bits", ctypes.c_int32), ("seed", ctypes.c_uint32), ("lr", ctypes.c_double), ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("grad_scale", ctypes.c_float), ("step", ctypes.c_int64),
        ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p),
    ]


_lib = None
_vp, _i64, _int, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
_ip = ctypes.POINTER(ctypes.c_int32)


def load() -> ctypes.CDLL:
    """Load libdetox.so (built in-tree by paper_1907_12205_b200.build).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_1907_12205_b200.build` "
                          "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    lib.detox_status_string.restype = ctypes.c_char_p
    lib.detox_status_string.argtypes = [_int]
    lib.detox_vote_workspace_bytes.restype = _sz
    lib.detox_vote_workspace_bytes.argtypes = [_int, _int]
    lib.detox_vote.argtypes = [_vp, _i64, _int, _int, _i64, _ip, _vp, _i64, _vp, _vp, _sz, _vp]
    lib.detox_vote_noalloc.argtypes = [_vp, _i64, _int, _int, _i64, _ip, _vp, _i64, _vp, _vp]
    lib.detox_vote_hier_mean.argtypes = [_vp, _i64, _int, _int, _i64, _ip, _ip, _ip, _int, _vp, _i64, _vp, _vp, _sz, _vp]
    lib.detox_hier_mean.argtypes = [_vp, _i64, _int, _i64, _ip, _ip, _int, _vp, _i64, _vp]
    for name in ("agg_coord_median", "agg_multikrum", "agg_bulyan"):
        fn = getattr(lib, name + "_workspace_bytes")
        fn.restype = _sz
        fn.argtypes = [_int, _i64]
    lib.agg_coord_median.argtypes = [_vp, _i64, _int, _i64, _vp, _vp, _sz, _vp]
    lib.agg_trimmed_mean.argtypes = [_vp, _i64, _int, _i64, _int, _vp, _vp]
    lib.agg_geometric_median_workspace_bytes.restype = _sz
    lib.agg_geometric_median_workspace_bytes.argtypes = [_int, _i64]
    lib.agg_geometric_median.argtypes = [_vp, _i64, _int, _i64, _int, ctypes.c_float, _vp, _vp, _sz, _vp]
    lib.agg_sign_majority.argtypes = [_vp, _i64, _int, _i64, _vp, _vp]
    lib.agg_multikrum.argtypes = [_vp, _i64, _int, _i64, _int, _int, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.agg_bulyan.argtypes = [_vp, _i64, _int, _i64, _int, _vp, _vp, _vp, _sz, _vp]
    lib.detox_aggregate_workspace_bytes.restype = _sz
    lib.detox_aggregate_workspace_bytes.argtypes = [ctypes.POINTER(PipelineDesc)]
    lib.detox_aggregate.argtypes = [ctypes.POINTER(PipelineDesc), _vp, _i64, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.detox_selftest_bounded_wait.argtypes = [_vp, _i64, _vp]
    lib.agg_pairwise_sqdist_workspace_bytes.restype = _sz
    lib.agg_pairwise_sqdist_workspace_bytes.argtypes = [_int, _i64]
    lib.agg_pairwise_sqdist.argtypes = [_vp, _i64, _int, _i64, _vp, _vp, _sz, _vp]
    lib.detox_vote_hier_mean_many.argtypes = [_vp, _i64, _i64, _int, _int, _vp, _ip, _int, _vp, _i64, _vp, _vp]
    lib.detox_tc_split_mode.argtypes = [_int]
    lib.detox_tc_split_mode.restype = _int
    lib.detox_tc_repeated_passes.restype = ctypes.c_ulonglong
    lib.detox_tc_repeated_passes.argtypes = []
    lib.detox_kernel_launch_count.restype = ctypes.c_ulonglong
    lib.detox_kernel_launch_count.argtypes = []
    lib.detox_checkpoint_pack.argtypes = [_int, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp]
    lib.detox_checkpoint_unpack.argtypes = [_int, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _i64, _vp]
    lib.detox_rmsnorm.argtypes = [_int, _vp, _i64, _vp, _i64, _vp, _i64, _i64, ctypes.c_float, _vp, _i64, _vp, _i64, _vp,
                                  _i64, _vp, _i64, _vp, _vp]
    lib.detox_rmsnorm_backward_workspace_bytes.restype = _sz
    lib.detox_rmsnorm_backward_workspace_bytes.argtypes = [_i64, _i64]
    lib.detox_rmsnorm_backward.argtypes = [_int, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _i64, _vp, _vp,
                                           _sz, _vp]
    for name in ("detox_gated", "detox_gated_backward"):
        fn = getattr(lib, name + "_workspace_bytes")
        fn.restype = _sz
        fn.argtypes = [ctypes.POINTER(GatedDesc)]
    lib.detox_gated_expired_waits.restype = ctypes.c_ulonglong
    lib.detox_gated_expired_waits.argtypes = [_ip, _int]
    lib.detox_gated_wait_limit.restype = _i64
    lib.detox_gated_wait_limit.argtypes = [_i64]
    lib.detox_gated.argtypes = [ctypes.POINTER(GatedDesc), _vp, _i64, _vp, _sz, _vp]
    lib.detox_gated_backward.argtypes = [ctypes.POINTER(GatedDesc), _vp, _i64, _vp, _i64, _vp, _vp, _i64, _int, _vp, _sz, _vp]
    _f = ctypes.c_float
    lib.detox_embedding.argtypes = [_int, _vp, _i64, _i64, _i64, _int, _vp, _i64, _f, _vp, _i64, _vp]
    lib.detox_embedding_backward_workspace_bytes.restype = _sz
    lib.detox_embedding_backward_workspace_bytes.argtypes = [_i64, _i64, _i64]
    lib.detox_embedding_backward.argtypes = [_int, _vp, _i64, _int, _vp, _i64, _i64, _i64, _f, _vp, _i64, _int, _int, _vp, _sz, _vp]
    lib.detox_token_logp.argtypes = [_int, _vp, _i64, _i64, _i64, _int, _vp, _f, _vp, _vp, _vp]
    lib.detox_token_logp_backward.argtypes = [_int, _vp, _i64, _i64, _i64, _int, _vp, _f, _vp, _vp, _vp, _i64, _vp]
    lib.detox_policy_loss_workspace_bytes.restype = _sz
    lib.detox_policy_loss_workspace_bytes.argtypes = [_i64]
    lib.detox_policy_loss.argtypes = [ctypes.POINTER(PolicyDesc), _vp, _vp, _vp, _i64, _vp, _sz, _vp]
    lib.detox_preference_loss_workspace_bytes.restype = _sz
    lib.detox_preference_loss_workspace_bytes.argtypes = [_i64, _i64]
    lib.detox_preference_loss.argtypes = [ctypes.POINTER(PreferenceDesc), _vp, _vp, _vp, _vp, _i64, _vp, _sz, _vp]
    lib.detox_adamw.argtypes = [ctypes.POINTER(AdamWDesc), ctypes.POINTER(AdamWTensor), _i64, _vp]
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().detox_status_string(int(code)).decode()


def _check(code: int, what: str):
    if code != 0:
        raise DetoxError(code, what)


def _mat(X: torch.Tensor):
    if not (isinstance(X, torch.Tensor) and X.is_cuda and X.dtype == torch.float32 and X.dim() == 2):
        raise TypeError("expected a 2-D float32 CUDA tensor")
    if X.shape[1] > 1 and X.stride(1) != 1:
        raise ValueError("rows must be contiguous")
    ld = X.stride(0) if X.shape[0] > 1 else max(X.stride(0), X.shape[1])
    return X.data_ptr(), int(ld), int(X.shape[0]), int(X.shape[1])


def _host_i32(a: Sequence[int]) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _stream(stream) -> int:
    if stream is None:   # the current stream's handle, without a Stream object around it (3.2 -> 0.3 us a call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_object(stream):
    if hasattr(stream, "cuda_stream"):
        return stream
    return torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()


def _made_for_stream(fn):
    """With a stream given, it is the current one during the call, so that outputs and workspace are made for it: blocks of
    another stream's pool may still be in use there, or (the workspace, at the call's return) be used there again."""
    at = list(inspect.signature(fn).parameters).index("stream")

    @functools.wraps(fn)
    def call(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return fn(*args, **kw)
        with torch.cuda.stream(_stream_object(stream)):
            return fn(*args, **kw)

    return call


def _ws(nbytes: int, ws: Optional[torch.Tensor], device):
    if ws is None:
        ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    elif ws.device != device:
        raise TypeError(f"ws: expected a tensor on {device}, got one on {ws.device}")
    elif not ws.is_contiguous():
        raise ValueError("ws: expected a contiguous tensor")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def read_status(ws: torch.Tensor, stream=None) -> int:
    """The device status word of a finished call: the first int32 of the workspace that was passed to agg_multikrum,
    agg_bulyan or detox_aggregate.  Synchronises the stream.  0, or 5 (DETOX_ERR_TIMEOUT) when a bounded device-side
    wait ran out and the call's outputs are not valid."""
    (torch.cuda.current_stream() if stream is None else stream).synchronize()
    return int(ws[:4].view(torch.int32).item())


def check_status(ws: torch.Tensor, what: str = "device status", stream=None):
    """Raises DetoxError if the device status word of a finished call is not 0 (synchronises the stream)."""
    _check(read_status(ws, stream), what)


@_made_for_stream
def detox_selftest_bounded_wait(limit_cycles: int = 100_000, status: Optional[torch.Tensor] = None, stream=None):
    """Runs the library's bounded wait on a barrier that nothing completes; returns the int32 status tensor, which
    reads 5 (DETOX_ERR_TIMEOUT) once the stream has been synchronised."""
    if status is None:
        status = torch.empty(1, dtype=torch.int32, device="cuda")
    _check(load().detox_selftest_bounded_wait(status.data_ptr(), int(limit_cycles), _stream(stream)),
           "detox_selftest_bounded_wait")
    return status


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def detox_vote_workspace_bytes(n: int, r: int) -> int:
    return int(load().detox_vote_workspace_bytes(n, r))


@_made_for_stream
def detox_vote(X, r: int, members, Z: Optional[torch.Tensor] = None, winner: Optional[torch.Tensor] = None,
               want_Z: bool = True, ws: Optional[torch.Tensor] = None, stream=None):
    """Majority vote per node group.  Returns (Z or None, winner)."""
    lib = load()
    xp, ld, n, d = _mat(X)
    mem = _host_i32(members)
    if Z is None and want_Z:
        ldz = (d + 31) // 32 * 32
        Z = torch.empty((n // max(r, 1), ldz), dtype=torch.float32, device=X.device)[:, :d]
    if winner is None:
        winner = torch.empty(max(n // max(r, 1), 1), dtype=torch.int32, device=X.device)[: n // max(r, 1)]
    zp, ldz = (None, 0) if Z is None else (Z.data_ptr(), Z.stride(0) if Z.shape[0] > 1 else max(Z.stride(0), d))
    ws, wp, wb = _ws(lib.detox_vote_workspace_bytes(n, r), ws, X.device)
    _check(lib.detox_vote(xp, ld, n, r, d, mem.ctypes.data_as(_ip), zp, ldz, winner.data_ptr(), wp, wb,
                          _stream(stream)), "detox_vote")
    return Z, winner


NOALLOC_MAX_GROUPS = 256


def detox_vote_noalloc(X, r: int, members, Z: torch.Tensor, winner: torch.Tensor, stream=None):
    """detox_vote for callers that cannot allocate: the scratch is a fixed array inside the library,
    and Z (or None) and winner must be passed in, so neither the library nor this wrapper allocates
    device memory.  At most NOALLOC_MAX_GROUPS node groups.  Calls that overlap on the GPU race on
    the shared scratch; the first call on a device should come before any stream capture."""
    lib = load()
    xp, ld, n, d = _mat(X)
    mem = _host_i32(members)
    zp, ldz = (None, 0) if Z is None else (Z.data_ptr(), Z.stride(0) if Z.shape[0] > 1 else max(Z.stride(0), d))
    _check(lib.detox_vote_noalloc(xp, ld, n, r, d, mem.ctypes.data_as(_ip), zp, ldz, winner.data_ptr(),
                                  _stream(stream)), "detox_vote_noalloc")
    return Z, winner


@_made_for_stream
def detox_hier_mean(Z, set_offsets, set_members, M: Optional[torch.Tensor] = None, stream=None):
    lib = load()
    zp, ldz, G, d = _mat(Z)
    so, sm = _host_i32(set_offsets), _host_i32(set_members)
    S = len(so) - 1
    if M is None:
        ldm = (d + 31) // 32 * 32
        M = torch.empty((max(S, 1), ldm), dtype=torch.float32, device=Z.device)[:S, :d]
    ldm = M.stride(0) if M.shape[0] > 1 else max(M.stride(0), d)
    _check(lib.detox_hier_mean(zp, ldz, G, d, so.ctypes.data_as(_ip), sm.ctypes.data_as(_ip), S, M.data_ptr(), ldm,
                               _stream(stream)), "detox_hier_mean")
    return M


@_made_for_stream
def detox_vote_hier_mean(X, r: int, members, set_offsets, set_members, M: Optional[torch.Tensor] = None,
                         winner: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Vote and mean over each vote set in one pass.  Returns (M [S, d], winner [G])."""
    lib = load()
    xp, ld, n, d = _mat(X)
    mem, so, sm = _host_i32(members), _host_i32(set_offsets), _host_i32(set_members)
    S = len(so) - 1
    if M is None:
        ldm = (d + 31) // 32 * 32
        M = torch.empty((max(S, 1), ldm), dtype=torch.float32, device=X.device)[:S, :d]
    ldm = M.stride(0) if M.shape[0] > 1 else max(M.stride(0), d)
    if winner is None:
        winner = torch.empty(max(n // max(r, 1), 1), dtype=torch.int32, device=X.device)[: n // max(r, 1)]
    ws, wp, wb = _ws(lib.detox_vote_workspace_bytes(n, r), ws, X.device)
    _check(lib.detox_vote_hier_mean(xp, ld, n, r, d, mem.ctypes.data_as(_ip), so.ctypes.data_as(_ip),
                                    sm.ctypes.data_as(_ip), S, M.data_ptr(), ldm, winner.data_ptr(), wp, wb,
                                    _stream(stream)), "detox_vote_hier_mean")
    return M, winner


@_made_for_stream
def detox_vote_hier_mean_many(X, r: int, members_dev: torch.Tensor, set_offsets=None, M: Optional[torch.Tensor] = None,
                              winner: Optional[torch.Tensor] = None, stream=None):
    """Vote and set means for very many nodes with short vectors.  members_dev: int32 CUDA tensor [n];
    set_offsets: host, in groups (None: votes only).  Returns (M [S, d] or None, winner [n / r])."""
    lib = load()
    xp, ld, n, d = _mat(X)
    if not (members_dev.is_cuda and members_dev.dtype == torch.int32 and members_dev.numel() == n):
        raise TypeError("members_dev: int32 CUDA tensor with one entry per node")
    G = n // max(r, 1)
    if winner is None:
        winner = torch.empty(max(G, 1), dtype=torch.int32, device=X.device)[:G]
    so, S, mp, ldm = None, 0, None, 0
    if set_offsets is not None:
        so = _host_i32(set_offsets)
        S = len(so) - 1
        if M is None:
            M = torch.empty((max(S, 1), (d + 31) // 32 * 32), dtype=torch.float32, device=X.device)[:S, :d]
        mp, ldm = M.data_ptr(), (M.stride(0) if M.shape[0] > 1 else max(M.stride(0), d))
    _check(lib.detox_vote_hier_mean_many(xp, ld, n, r, d, members_dev.data_ptr(),
                                         None if so is None else so.ctypes.data_as(_ip), S, mp, ldm, winner.data_ptr(),
                                         _stream(stream)), "detox_vote_hier_mean_many")
    return M, winner


def agg_coord_median_workspace_bytes(m: int, d: int) -> int:
    return int(load().agg_coord_median_workspace_bytes(m, d))


@_made_for_stream
def agg_coord_median(X, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    lib = load()
    xp, ld, m, d = _mat(X)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=X.device)
    _check(lib.agg_coord_median(xp, ld, m, d, out.data_ptr(), _ptr(ws), 0 if ws is None else ws.numel(),
                                _stream(stream)), "agg_coord_median")
    return out


@_made_for_stream
def agg_trimmed_mean(X, trim: int, out: Optional[torch.Tensor] = None, stream=None):
    """Coordinate-wise mean after dropping the `trim` smallest and `trim` largest values."""
    lib = load()
    xp, ld, m, d = _mat(X)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=X.device)
    _check(lib.agg_trimmed_mean(xp, ld, m, d, trim, out.data_ptr(), _stream(stream)), "agg_trimmed_mean")
    return out


@_made_for_stream
def agg_sign_majority(X, out: Optional[torch.Tensor] = None, stream=None):
    """Coordinate-wise sign(sum of signs): -1, 0 or +1 per coordinate."""
    lib = load()
    xp, ld, m, d = _mat(X)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=X.device)
    _check(lib.agg_sign_majority(xp, ld, m, d, out.data_ptr(), _stream(stream)), "agg_sign_majority")
    return out


@_made_for_stream
def agg_geometric_median(X, iters: int = 32, eps: float = 1e-12, out: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None, stream=None):
    """Geometric median of at most 32 rows by `iters` Weiszfeld iterations started at the mean."""
    lib = load()
    xp, ld, m, d = _mat(X)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=X.device)
    ws, wp, wb = _ws(lib.agg_geometric_median_workspace_bytes(m, d), ws, X.device)
    _check(lib.agg_geometric_median(xp, ld, m, d, iters, eps, out.data_ptr(), wp, wb, _stream(stream)),
           "agg_geometric_median")
    return out


SPLIT_AUTO, SPLIT_TF32 = 0, 1


def tc_split_mode(mode: int = -1) -> int:
    """Sets which operand split the tensor-core distance pass tries first (SPLIT_AUTO: fp16 pairs, SPLIT_TF32);
    returns the previous mode; without an argument only queries."""
    return int(load().detox_tc_split_mode(int(mode)))


def tc_repeated_passes() -> int:
    """Calls on the current device whose tensor-core distance pass had to be repeated so far (synchronises)."""
    return int(load().detox_tc_repeated_passes())


def kernel_launch_count() -> int:
    """Kernels launched by the library in this process so far."""
    return int(load().detox_kernel_launch_count())


def agg_pairwise_sqdist_workspace_bytes(m: int, d: int) -> int:
    return int(load().agg_pairwise_sqdist_workspace_bytes(m, d))


@_made_for_stream
def agg_pairwise_sqdist(X, D: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Squared distances between the rows: D [m, m] float64, symmetric, zero diagonal."""
    lib = load()
    xp, ld, m, d = _mat(X)
    if D is None:
        D = torch.empty((m, m), dtype=torch.float64, device=X.device)
    ws, wp, wb = _ws(lib.agg_pairwise_sqdist_workspace_bytes(m, d), ws, X.device)
    _check(lib.agg_pairwise_sqdist(xp, ld, m, d, D.data_ptr(), wp, wb, _stream(stream)), "agg_pairwise_sqdist")
    return D


def agg_multikrum_workspace_bytes(m: int, d: int) -> int:
    return int(load().agg_multikrum_workspace_bytes(m, d))


@_made_for_stream
def agg_multikrum(X, f: int, m_sel: int, out: Optional[torch.Tensor] = None, sel: Optional[torch.Tensor] = None,
                  scores: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Returns (out [d] float32, sel [m_sel] int32 ascending, scores [m] float64)."""
    lib = load()
    xp, ld, m, d = _mat(X)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=X.device)
    if sel is None:
        sel = torch.empty(max(m_sel, 1), dtype=torch.int32, device=X.device)[: max(m_sel, 0)]
    if scores is None:
        scores = torch.empty(m, dtype=torch.float64, device=X.device)
    ws, wp, wb = _ws(lib.agg_multikrum_workspace_bytes(m, d), ws, X.device)
    _check(lib.agg_multikrum(xp, ld, m, d, f, m_sel, out.data_ptr(), sel.data_ptr(), scores.data_ptr(), wp, wb,
                             _stream(stream)), "agg_multikrum")
    return out, sel, scores


def agg_bulyan_workspace_bytes(m: int, d: int) -> int:
    return int(load().agg_bulyan_workspace_bytes(m, d))


@_made_for_stream
def agg_bulyan(X, f: int, out: Optional[torch.Tensor] = None, sel: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None, stream=None):
    """Returns (out [d] float32, sel [m - 2f] int32 in selection order)."""
    lib = load()
    xp, ld, m, d = _mat(X)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=X.device)
    if sel is None:
        sel = torch.empty(max(m - 2 * f, 1), dtype=torch.int32, device=X.device)[: max(m - 2 * f, 0)]
    ws, wp, wb = _ws(lib.agg_bulyan_workspace_bytes(m, d), ws, X.device)
    _check(lib.agg_bulyan(xp, ld, m, d, f, out.data_ptr(), sel.data_ptr(), wp, wb, _stream(stream)), "agg_bulyan")
    return out, sel


class Pipeline:
    """Holds the host-side description of one DETOX configuration (Algorithm 1 + Algorithm 2)."""

    def __init__(self, n: int, r: int, d: int, members, a0: int = AGG_NONE, set_offsets=None, set_members=None,
                 a1: int = AGG_COORD_MEDIAN, f: int = 0, m_sel: int = 1, gm_iters: int = 32, gm_eps: float = 1e-12):
        self.members = _host_i32(members)
        self.set_offsets = None if set_offsets is None else _host_i32(set_offsets)
        self.set_members = None if set_members is None else _host_i32(set_members)
        self.desc = PipelineDesc()
        self.desc.n, self.desc.r, self.desc.d = n, r, d
        self.desc.members = self.members.ctypes.data_as(_ip)
        self.desc.a0 = a0
        self.desc.n_sets = 0 if self.set_offsets is None else len(self.set_offsets) - 1
        self.desc.set_offsets = None if self.set_offsets is None else self.set_offsets.ctypes.data_as(_ip)
        self.desc.set_members = None if self.set_members is None else self.set_members.ctypes.data_as(_ip)
        self.desc.a1, self.desc.f, self.desc.m_sel = a1, f, m_sel
        self.desc.gm_iters, self.desc.gm_eps = gm_iters, gm_eps
        self.n, self.r, self.d, self.a0, self.a1, self.f, self.m_sel = n, r, d, a0, a1, f, m_sel

    @property
    def G(self) -> int:
        return self.n // self.r

    @property
    def rows_into_a1(self) -> int:
        return self.desc.n_sets if self.a0 != AGG_NONE else self.G

    @property
    def n_selected(self) -> int:
        if self.a0 in (AGG_MULTIKRUM, AGG_BULYAN):      # chosen inside every vote set, concatenated in set order
            sizes = np.diff(self.set_offsets)
            if self.a0 == AGG_BULYAN:
                return int(sum(k - 2 * self.f for k in sizes))
            return int(sum(self.m_sel if self.m_sel > 0 else max(k - self.f, 1) for k in sizes))
        if self.a1 == AGG_MULTIKRUM:
            return self.m_sel
        if self.a1 == AGG_BULYAN:
            return self.rows_into_a1 - 2 * self.f
        return 0

    def workspace_bytes(self) -> int:
        return int(load().detox_aggregate_workspace_bytes(ctypes.byref(self.desc)))


def detox_aggregate_workspace_bytes(pipe: Pipeline) -> int:
    return pipe.workspace_bytes()


@_made_for_stream
def detox_aggregate(pipe: Pipeline, X, out: Optional[torch.Tensor] = None, winner: Optional[torch.Tensor] = None,
                    sel: Optional[torch.Tensor] = None, sel_workers: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, stream=None):
    """Vote -> A_0 -> A_1.  Returns dict(out, winner, sel, sel_workers).

    sel lists the rows chosen by the Krum-type stage: rows that entered A_1 when A_1 is Multi-Krum / Bulyan;
    vote (group) indices, set after set, when A_0 is Multi-Krum / Bulyan.  sel_workers gives the same rows
    as worker ids whenever sel indexes votes."""
    lib = load()
    xp, ld, n, d = _mat(X)
    if n != pipe.n or d != pipe.d:
        raise ValueError("X does not match the pipeline description")
    dev = X.device
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=dev)
    if winner is None:
        winner = torch.empty(pipe.G, dtype=torch.int32, device=dev)
    k = pipe.n_selected
    if k > 0 and sel is None:
        sel = torch.empty(k, dtype=torch.int32, device=dev)
    if k > 0 and sel_workers is None and pipe.a0 != AGG_MEAN:
        sel_workers = torch.empty(k, dtype=torch.int32, device=dev)
    need = pipe.workspace_bytes()
    if need == 0:
        raise DetoxError(1, "detox_aggregate_workspace_bytes")
    ws, wp, wb = _ws(need, ws, dev)
    _check(lib.detox_aggregate(ctypes.byref(pipe.desc), xp, ld, out.data_ptr(), winner.data_ptr(), _ptr(sel),
                               _ptr(sel_workers), wp, wb, _stream(stream)), "detox_aggregate")
    return dict(out=out, winner=winner, sel=sel, sel_workers=sel_workers)


# ------------------------------------------------------------------------------------------------------------------
# The worker's side: norm, 8-bit checkpoints, gated projections.  With `stream` a call makes its outputs and its workspace for
# that stream, as it would under torch.cuda.stream(stream).  No graph is recorded: tensors that require grad are refused outside
# torch.no_grad().

DTYPE_FLOAT, DTYPE_HALF, DTYPE_BFLOAT = range(3)
ACT_SILU, ACT_GELU, ACT_RELU = range(3)
KEEP_BLOCK = 128
_DTYPE = {torch.float32: DTYPE_FLOAT, torch.float16: DTYPE_HALF, torch.bfloat16: DTYPE_BFLOAT}


class RmsNorm(NamedTuple):
    """What detox_rmsnorm leaves; None where it was not asked for."""
    sum: Optional[torch.Tensor]
    y: Optional[torch.Tensor]
    q: Optional[torch.Tensor]
    e: Optional[torch.Tensor]
    rstd: torch.Tensor


class Kept(NamedTuple):
    """g and u of a gated pair of projections in the 8-bit form: values [2, tokens, hidden], scales [2, tokens, blocks]."""
    q: torch.Tensor
    e: torch.Tensor

    @property
    def gq(self):
        return self.q[0]

    @property
    def ge(self):
        return self.e[0]

    @property
    def uq(self):
        return self.q[1]

    @property
    def ue(self):
        return self.e[1]


_worker_module = None


def _worker():
    """The compiled module that checks tensors, makes outputs and calls the library for the functions below (a call's
    marshalling in Python took 10 to 40 us, more than the small kernels).  Raises if it is not built."""
    global _worker_module
    if _worker_module is None:
        load()
        from . import _worker as module
        module.set_error(DetoxError)
        _worker_module = module
    return _worker_module


def _handle(stream):
    return stream if stream is None or isinstance(stream, int) else stream.cuda_stream


def detox_checkpoint_pack(x: torch.Tensor, out=None, stream=None):
    """Rows in the 8-bit form: (q, e), float8_e4m3fn values and float8_e8m0fnu scales, one for each block of KEEP_BLOCK
    columns of a row.  out: such a pair to write into."""
    q, e = (None, None) if out is None else out
    return (_worker_module or _worker()).checkpoint_pack(x, q, e, _handle(stream))


def detox_checkpoint_unpack(q: torch.Tensor, e: torch.Tensor, dtype=torch.bfloat16, out: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """The way back from detox_checkpoint_pack: rows of `dtype`."""
    return (_worker_module or _worker()).checkpoint_unpack(q, e, _dtype_code(dtype), out, _handle(stream))


def detox_rmsnorm(x: torch.Tensor, w: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  want_y: bool = True, want_q: bool = False, sum_out: Optional[torch.Tensor] = None, stream=None) -> RmsNorm:
    """s = x + residual, y = s / rms(s) * w.  want_q: y also (want_y=False: only) in the 8-bit form.  The sum comes back
    when there is a residual, in sum_out when given (which may be x or residual itself)."""
    return RmsNorm._make((_worker_module or _worker()).rmsnorm(x, w, residual, eps, want_y, want_q, sum_out, _handle(stream)))


def detox_rmsnorm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(load().detox_rmsnorm_backward_workspace_bytes(rows, cols))


def detox_rmsnorm_backward(dy: torch.Tensor, s: torch.Tensor, w: torch.Tensor, rstd: torch.Tensor,
                           ds: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                           dw: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Gradients of detox_rmsnorm: (dx, dw).  s: the sum of the forward pass (its x when there was no residual); ds: the
    gradient that reaches the sum by its other uses.  dx is also the residual's gradient; dw is fp32."""
    return (_worker_module or _worker()).rmsnorm_backward(dy, s, w, rstd, ds, dx, dw, ws, _handle(stream))


def _gated_inputs(x, kept: Optional[Kept]):
    """x (a matrix, or its 8-bit form as a pair) and kept, as the module takes them."""
    x, xe = (x, None) if isinstance(x, torch.Tensor) else x
    q, e = (None, None) if kept is None else kept
    return x, xe, q, e


def detox_gated_workspace_bytes(x, wg, wu, act: int = ACT_SILU, kept: Optional[Kept] = None) -> int:
    x, xe, q, e = _gated_inputs(x, kept)
    return _worker().gated_workspace_bytes(x, xe, wg, wu, act, q, e, False)


def detox_gated(x, wg: torch.Tensor, wu: torch.Tensor, act: int = ACT_SILU, keep: bool = False,
                h: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """h = act(x wg^T) * (x wu^T).  x: a matrix, or its 8-bit form as a pair (q, e).  keep=True returns (h, Kept): g and u
    in the 8-bit form for the backward pass."""
    x, xe = (x, None) if isinstance(x, torch.Tensor) else x
    h, q, e = (_worker_module or _worker()).gated(x, xe, wg, wu, act, None, None, keep, h, ws, _handle(stream))
    return (h, Kept(q, e)) if keep else h


def detox_gated_backward_workspace_bytes(x, wg, wu, act: int = ACT_SILU, kept: Optional[Kept] = None) -> int:
    x, xe, q, e = _gated_inputs(x, kept)
    return _worker().gated_workspace_bytes(x, xe, wg, wu, act, q, e, True)


def detox_gated_backward(dh: torch.Tensor, x, wg: torch.Tensor, wu: torch.Tensor, act: int = ACT_SILU,
                         kept: Optional[Kept] = None, dx: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
                         dwu: Optional[torch.Tensor] = None, dw_dtype=None, ws: Optional[torch.Tensor] = None, stream=None):
    """Gradients of detox_gated: (dx, dwg, dwu).  kept: what the forward pass kept; without it g and u are computed again.
    x as in detox_gated.  The weight gradients have the weights' type, or float32 with dw_dtype (or buffers of it, such as
    pieces of a gradient's row).  In float16 the gradients of g and u have to stay below 65504 and well above 2^-25: scale dh."""
    x, xe, q, e = _gated_inputs(x, kept)
    return (_worker_module or _worker()).gated_backward(x, xe, wg, wu, act, q, e, dh, dx, dwg, dwu,
                                                        -1 if dw_dtype is None else _dtype_code(dw_dtype), ws, _handle(stream))


class ExpiredWait(NamedTuple):
    """What the first expired wait of the gated products waited for (include/detox.h, detox_gated_expired_waits)."""
    form: int
    ctas: int
    columns: int
    split: int
    rank: int
    barrier: int
    index: int
    tile: int


def gated_expired_waits(clear: bool = False):
    """(count, ExpiredWait or None): the waits of the gated products that ran out on the current device since the count was last
    cleared.  Synchronises the device.  Also tells of calls that made their own workspace and with it their status word."""
    first = (ctypes.c_int32 * 8)()
    n = int(load().detox_gated_expired_waits(first, int(clear)))
    return n, (ExpiredWait(*first) if n else None)


def gated_wait_limit(clocks: int = -1) -> int:
    """Sets the limit of the gated products' waits in SM clocks (0: by the product's length); returns the one before.  The
    default argument only asks."""
    return int(load().detox_gated_wait_limit(int(clocks)))


# ------------------------------------------------------------------------------------------------------------------
# Around the sublayer: the token embedding, the losses over logits, and the optimizer's step on the server.

LOGITS_MAX_COLS = 262144


def detox_embedding(tokens: torch.Tensor, w: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """Rows of the table w [vocab, cols], scaled: [tokens, cols].  tokens: a vector of int32 or int64; a negative one is padding (a
    row of zeros), one beyond the vocabulary gives a row of NaN."""
    return (_worker_module or _worker()).embedding(tokens, w, scale, out, _handle(stream))


def detox_embedding_backward_workspace_bytes(rows: int, vocab: int, cols: int) -> int:
    return int(load().detox_embedding_backward_workspace_bytes(rows, vocab, cols))


def detox_embedding_backward(dy: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0, dw: Optional[torch.Tensor] = None,
                             dw_dtype=None, accumulate: bool = False, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of the table, [vocab, cols], the rows of equal tokens added in a fixed order.  It has dy's type, or float32 with dw_dtype (or
    a dw of it, such as a piece of a gradient's row).  accumulate: add to dw, as for a table that is the output head too; rows of tokens
    that do not occur are left alone."""
    return (_worker_module or _worker()).embedding_backward(dy, tokens, vocab, scale, dw, -1 if dw_dtype is None else _dtype_code(dw_dtype),
                                                            accumulate, ws, _handle(stream))


class TokenLogp(NamedTuple):
    """Log-probabilities of the chosen tokens, and the rows' log-sum-exp for the backward pass (None where it was not wanted)."""
    logp: torch.Tensor
    lse: Optional[torch.Tensor]


def detox_token_logp(z: torch.Tensor, y: torch.Tensor, scale: float = 1.0, stream=None, want_lse: bool = True) -> TokenLogp:
    """logp[t] = log softmax(scale z[t])[y[t]] for logits z [tokens, vocab], and lse[t] = log sum exp(scale z[t]).  y < 0: no token was chosen
    there, and logp is 0; its lse is that of every other row.  want_lse=False: logp alone, and rows without a chosen token are not read."""
    return TokenLogp._make((_worker_module or _worker()).token_logp(z, y, scale, want_lse, _handle(stream)))


def detox_token_logp_backward(dlogp: torch.Tensor, z: torch.Tensor, y: torch.Tensor, lse: torch.Tensor, scale: float = 1.0,
                              dz: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of the logits for a gradient of detox_token_logp's logp.  dz may be z itself."""
    return (_worker_module or _worker()).token_logp_backward(dlogp, z, y, lse, scale, dz, _handle(stream))


class PolicyLoss(NamedTuple):
    """What detox_policy_loss leaves.  stats: loss, and the weighted sums of the policy's term, of the KL term and of the clipped tokens; dz is
    None where no gradient was wanted."""
    stats: torch.Tensor
    logp: torch.Tensor
    dz: Optional[torch.Tensor]

    @property
    def loss(self):
        return self.stats[0]

    @property
    def pg(self):
        return self.stats[1]

    @property
    def kl(self):
        return self.stats[2]

    @property
    def clipped(self):
        return self.stats[3]


def detox_policy_loss_workspace_bytes(rows: int) -> int:
    return int(load().detox_policy_loss_workspace_bytes(rows))


def detox_policy_loss(z: torch.Tensor, y: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor,
                      ref_logp: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                      clip_high: float = 0.2, kl_coef: float = 0.0, scale: float = 1.0, want_grad: bool = True, grad_scale: float = 1.0,
                      dz: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None) -> PolicyLoss:
    """The clipped policy loss sum of weight (pg + kl_coef kl) over the tokens, and with want_grad grad_scale times its gradient by the logits, from
    one pass over them.  weight: such as mask / number of tokens (default 1 / rows); rows of weight 0 or without a chosen token (y < 0)
    are not read and have zero gradients.  dz may be z itself."""
    return PolicyLoss._make((_worker_module or _worker()).policy_loss(z, y, old_logp, advantage, ref_logp, weight, clip_low, clip_high,
                                                                      kl_coef, scale, want_grad, grad_scale, dz, ws, _handle(stream)))


class PreferenceLoss(NamedTuple):
    """What detox_preference_loss leaves: loss [1], margin [pairs], sums of logp [2 pairs], and the logits' gradient (or None)."""
    loss: torch.Tensor
    margin: torch.Tensor
    sums: torch.Tensor
    dz: Optional[torch.Tensor]


def detox_preference_loss_workspace_bytes(rows: int, pairs: int) -> int:
    return int(load().detox_preference_loss_workspace_bytes(rows, pairs))


def detox_preference_loss(z: torch.Tensor, y: torch.Tensor, offsets: torch.Tensor, ref: torch.Tensor, beta: float = 0.1,
                          smoothing: float = 0.0, scale: float = 1.0, want_grad: bool = True, grad_scale: float = 1.0,
                          dz: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None) -> PreferenceLoss:
    """Mean loss of pairs of packed sequences, preferred and other in turn: offsets [2 pairs + 1] int32 bounds their rows, ref [2 pairs] holds
    their sums of logp under the reference policy.  Rows with y < 0 (prompts) and rows of no sequence count nothing.  dz may be z itself."""
    return PreferenceLoss._make((_worker_module or _worker()).preference_loss(z, y, offsets, ref, beta, smoothing, scale, want_grad,
                                                                              grad_scale, dz, ws, _handle(stream)))


def detox_adamw_state(params: Sequence[torch.Tensor], bits: int = 32):
    """New states for detox_adamw, all zeros: (m, v), lists of float32 tensors, or with bits=8 of pairs (values, scales)."""
    if bits not in (8, 32):
        raise ValueError(f"bits: expected 8 or 32, got {bits}")

    def state(p):
        if bits == 32:
            return torch.zeros(p.shape, dtype=torch.float32, device=p.device)
        q = torch.zeros(p.numel(), dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
        e = torch.ones(-(-p.numel() // KEEP_BLOCK), dtype=torch.uint8, device=p.device).view(torch.float8_e8m0fnu)   # 2^-126, a zero block's
        return q, e

    return [state(p) for p in params], [state(p) for p in params]


def detox_adamw(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m: Sequence, v: Sequence, step, lr, beta1: float = 0.9,
                beta2: float = 0.999, eps: float = 1e-8, weight_decay=0.0, masters: Optional[Sequence] = None, grad_scale: float = 1.0,
                seed: int = 0, stream=None) -> None:
    """One AdamW step over all tensors, in place.  step counts from 1; step and lr may be CUDA tensors of one int64 and one float32, which the
    step reads when it runs (so a captured one can be replayed).  m, v: as detox_adamw_state makes them; in 8 bits v holds the root, and both
    are rounded at random with bits that follow from seed, step, a tensor's place in the list and the entry.  weight_decay: a number, or one
    for each tensor.  masters: float32 copies of the params (or None for some), which then are what is stepped.  eps: at least 1e-18, with 8-bit states 1e-15."""
    (_worker_module or _worker()).adamw(params, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, masters, grad_scale, seed,
                                        _handle(stream))


def _dtype_code(dtype) -> int:
    if dtype not in _DTYPE:
        raise TypeError(f"expected float32, float16 or bfloat16, got {dtype}")
    return _DTYPE[dtype]
