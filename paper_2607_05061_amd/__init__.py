"""KVpop future-attention target on MI355X (gfx950).

A thin ctypes binding over the in-tree ``libkvpop.so`` (C ABI in ``include/kvpop.h``).
Every function here only marshals arguments: it checks tensor placement, dtype and
layout, derives the dimensions, allocates with PyTorch the outputs (and scratch) that
the caller does not pass, and calls the C entry point of the same name on the current
HIP stream or on ``stream``. All arithmetic runs in the library's HIP kernels; there is
no fallback.

Outputs that a call allocates belong to the current stream, as every torch result does;
a caller that passes another ``stream`` orders the two streams itself, or passes outputs.
Scratch comes from the memory of the stream that the kernels run on.

Quantities (KVpop App. D.1): for query head qh and key position t,

    lse[b, qh, d] = log sum_{t <= d} exp(scale <q_d, k_t> + bias_t)       (pass 1)
    out[b, qh, t] = sum_{d = t + window}^{min(T - 1, t + horizon)}
                    exp(scale <q_d, k_t> + bias_t - lse[b, qh, d])       (pass 2)

with query head qh reading KV head qh // (Hq // Hkv); horizon < 0 = no limit.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Any, NamedTuple, Optional, Tuple

__all__ = [
    "KVPOP_OK", "KVPOP_EINVAL", "KVPOP_EUNSUPPORTED", "KVPOP_EHIP", "KvpopDims", "KvpopError",
    "lib", "lib_path", "kvpop_row_lse", "kvpop_future_attn_from_lse", "kvpop_future_attn_target",
    "kvpop_future_attn_scores", "kvpop_strerror", "kvpop_abi_version", "KVPOP_AGG_MAX", "KVPOP_AGG_MEAN",
    "KvpopTopkDims", "kvpop_running_topk", "kvpop_running_topk_workspace_size", "kvpop_sparse_attn_fwd",
    "kvpop_running_topk_noalloc", "KVPOP_ETOOBIG", "KVPOP_NOALLOC_SCRATCH_BYTES", "kvpop_future_attn_bands",
    "KVPOP_CACHE_INT8", "KVPOP_CACHE_E4M3", "KvpopCache", "KvpopCacheC", "KvpopRowsC", "KvpopAppendC", "KvpopRetainC",
    "kvpop_cache_empty", "kvpop_cache_append", "kvpop_cache_attn", "kvpop_cache_attn_workspace_size",
    "kvpop_retain_prompt", "kvpop_retain_step",
]

KVPOP_OK = 0
KVPOP_EINVAL = 1
KVPOP_EUNSUPPORTED = 2
KVPOP_EHIP = 3
KVPOP_ETOOBIG = 4
KVPOP_NOALLOC_SCRATCH_BYTES = 32 << 20
KVPOP_AGG_MAX = 0
KVPOP_AGG_MEAN = 1
KVPOP_CACHE_INT8 = 0
KVPOP_CACHE_E4M3 = 1
ABI_VERSION = 3

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB: Optional[ctypes.CDLL] = None


class KvpopDims(ctypes.Structure):
    """Mirror of ``kvpop_dims`` in include/kvpop.h."""
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("seq_len", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]


class KvpopTopkDims(ctypes.Structure):
    """Mirror of ``kvpop_topk_dims`` in include/kvpop.h."""
    _fields_ = [("batch", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("seq_len", ctypes.c_int32)]


class KvpopCacheC(ctypes.Structure):
    """Mirror of ``kvpop_cache`` in include/kvpop_cache.h."""
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_kv_heads", "head_dim", "format", "page_size", "n_pages",
                                              "max_pages")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "k_exp", "v_exp", "page_table")]


class KvpopRowsC(ctypes.Structure):
    """Mirror of ``kvpop_rows`` in include/kvpop_cache.h."""
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_t", ctypes.c_int64)]


class KvpopAppendC(ctypes.Structure):
    """Mirror of ``kvpop_append`` in include/kvpop_cache.h."""
    _fields_ = [("n_tokens", ctypes.c_int32), ("n_entries", ctypes.c_int32), ("k", KvpopRowsC), ("v", KvpopRowsC),
                ("held", ctypes.c_void_p), ("count", ctypes.c_void_p), ("start", ctypes.c_void_p),
                ("src", ctypes.c_void_p), ("pos0", ctypes.c_void_p), ("cos", ctypes.c_void_p),
                ("sin", ctypes.c_void_p), ("n_positions", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("adjacent", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("q", KvpopRowsC),
                ("q_out", ctypes.c_void_p)]


class KvpopRetainC(ctypes.Structure):
    """Mirror of ``kvpop_retain`` in include/kvpop_cache.h."""
    _fields_ = [("batch", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("slots", ctypes.c_int32),
                ("pos", ctypes.c_void_p), ("prio", ctypes.c_void_p), ("held", ctypes.c_void_p)]


class KvpopError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__("%s failed with status %d: %s" % (where, status, kvpop_strerror(status)))
        self.status = status


def lib_path() -> str:
    return os.environ.get("KVPOP_LIB", os.path.join(_PKG_DIR, "libkvpop.so"))


def lib() -> ctypes.CDLL:
    """Load the built library (raises if it has not been built)."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError("libkvpop.so not found at %s: build it with "
                               "`python -m paper_2607_05061_amd.build`" % path)
        L = ctypes.CDLL(path)
        try:
            _set_types(L)
        except AttributeError as e:  # a library of an older build has fewer entry points
            raise RuntimeError("libkvpop.so at %s is not the one this binding was written for (%s): rebuild it with "
                               "`python -m paper_2607_05061_amd.build`" % (path, e)) from None
        _LIB = L
    return _LIB


def _set_types(L: ctypes.CDLL):
    """Checks the library's version and sets its entry points' types."""
    L.kvpop_abi_version.argtypes = []
    L.kvpop_abi_version.restype = ctypes.c_int
    if L.kvpop_abi_version() != ABI_VERSION:
        raise RuntimeError("libkvpop ABI version %d, binding expects %d" % (L.kvpop_abi_version(), ABI_VERSION))
    P, I32, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
    D = ctypes.POINTER(KvpopDims)
    L.kvpop_row_lse.argtypes = [D, P, P, P, P, P]
    L.kvpop_row_lse.restype = ctypes.c_int
    L.kvpop_future_attn_from_lse.argtypes = [D, P, P, P, P, I32, I32, P, P]
    L.kvpop_future_attn_from_lse.restype = ctypes.c_int
    L.kvpop_future_attn_bands.argtypes = [D, P, P, P, P, I32, ctypes.POINTER(I32), ctypes.POINTER(I32),
                                          ctypes.POINTER(P), P]
    L.kvpop_future_attn_bands.restype = ctypes.c_int
    L.kvpop_future_attn_target.argtypes = [D, P, P, P, I32, I32, P, P, P]
    L.kvpop_future_attn_target.restype = ctypes.c_int
    L.kvpop_future_attn_scores.argtypes = [D, P, P, P, P, I32, I32, I32, F, I32, P, P, P]
    L.kvpop_future_attn_scores.restype = ctypes.c_int
    L.kvpop_internal_scores_spread.argtypes = [D, I32, I32]
    L.kvpop_internal_scores_spread.restype = ctypes.c_int
    L.kvpop_running_topk_workspace_size.argtypes = [ctypes.POINTER(KvpopTopkDims)]
    L.kvpop_running_topk_workspace_size.restype = ctypes.c_size_t
    L.kvpop_running_topk.argtypes = [ctypes.POINTER(KvpopTopkDims), P, P, I32, I32, I32, P, P, P, P, P, P,
                                     ctypes.c_size_t, P]
    L.kvpop_running_topk.restype = ctypes.c_int
    L.kvpop_running_topk_noalloc.argtypes = [ctypes.POINTER(KvpopTopkDims), P, P, I32, I32, I32, P, P, P, P, P,
                                             P]
    L.kvpop_running_topk_noalloc.restype = ctypes.c_int
    L.kvpop_sparse_attn_fwd.argtypes = [ctypes.POINTER(KvpopDims), P, P, P, P, P, P, P, P]
    L.kvpop_sparse_attn_fwd.restype = ctypes.c_int
    # Structures go by address: a ctypes mirror by reference, or its packed bytes.
    C = R = S = P
    L.kvpop_cache_append.argtypes = [C, P, P]
    L.kvpop_cache_append.restype = ctypes.c_int
    L.kvpop_cache_attn_workspace_size.argtypes = [C, I32, I32]
    L.kvpop_cache_attn_workspace_size.restype = ctypes.c_size_t
    L.kvpop_cache_attn.argtypes = [C, I32, I32, F, R, P, P, P, P, P, ctypes.c_size_t, P]
    L.kvpop_cache_attn.restype = ctypes.c_int
    L.kvpop_retain_prompt.argtypes = [S, I32, P, P, P, P, P]
    L.kvpop_retain_prompt.restype = ctypes.c_int
    L.kvpop_retain_step.argtypes = [S, P, P, P, I32, I32, I32, P, P]
    L.kvpop_retain_step.restype = ctypes.c_int
    L.kvpop_strerror.argtypes = [ctypes.c_int]
    L.kvpop_strerror.restype = ctypes.c_char_p


def kvpop_strerror(status: int) -> str:
    return lib().kvpop_strerror(int(status)).decode()


def kvpop_abi_version() -> int:
    return int(lib().kvpop_abi_version())


# ---------------------------------------------------------------------------
# torch-tensor marshalling
# ---------------------------------------------------------------------------

def _torch():
    import torch  # noqa: WPS433 (PyTorch only provides device memory and streams)
    return torch


def _dims(q, k, scale: float) -> KvpopDims:
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q must be [B, Hq, T, D] and k [B, Hkv, T, D]")
    B, Hq, T, D = q.shape
    if k.shape[0] != B or k.shape[2] != T or k.shape[3] != D:
        raise ValueError("q %s and k %s disagree on B, T or D" % (tuple(q.shape), tuple(k.shape)))
    return KvpopDims(B, Hq, k.shape[1], T, D, float(scale))


def _check_tensor(x, name: str, dtype, device):
    torch = _torch()
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if x.device.type != "cuda" or (device is not None and x.device != device):
        raise ValueError("%s must be on the GPU device of q" % name)
    if x.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, x.dtype))
    if not x.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _stream_ptr(stream, device) -> int:
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return int(s.cuda_stream)


def _on_launch_stream(stream, device):
    """A context with the stream that the kernels run on as torch's current one: scratch that
    a call drops on return is allocated in it, so that the caching allocator orders the work
    before and after the call on that memory. ``stream`` is any object with a handle."""
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif not isinstance(stream, torch.cuda.Stream):
        h = int(stream.cuda_stream)
        stream = torch.cuda.ExternalStream(h, device=device) if h else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _check_workspace(workspace, need: int, device):
    """A caller's workspace: ``need`` bytes after each other (a view with strides may name as many elements
    and have less memory) on the device of the inputs."""
    if workspace.numel() * workspace.element_size() < need or workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must hold %d contiguous bytes on the device of the inputs" % need)


def _prep_inputs(q, k, key_bias):
    torch = _torch()
    _check_tensor(q, "q", torch.bfloat16, None)
    _check_tensor(k, "k", torch.bfloat16, q.device)
    if key_bias is not None:
        _check_tensor(key_bias, "key_bias", torch.float32, q.device)
        if key_bias.dim() != 1 or key_bias.shape[0] != q.shape[2]:
            raise ValueError("key_bias must be [T]")
    return q.data_ptr(), k.data_ptr(), (key_bias.data_ptr() if key_bias is not None else None)


def _prep_out(x, name, shape, device):
    torch = _torch()
    if x is None:
        return torch.empty(shape, dtype=torch.float32, device=device)
    _check_tensor(x, name, torch.float32, device)
    if tuple(x.shape) != tuple(shape):
        raise ValueError("%s must have shape %s" % (name, tuple(shape)))
    return x


def kvpop_row_lse(q, k, scale: float, key_bias=None, lse=None, stream=None):
    """Pass 1: dense causal row log-normaliser, fp32 [B, Hq, T] (eq. dense_lse_app)."""
    d = _dims(q, k, scale)
    qp, kp, bp = _prep_inputs(q, k, key_bias)
    lse = _prep_out(lse, "lse", (d.batch, d.n_q_heads, d.seq_len), q.device)
    st = lib().kvpop_row_lse(ctypes.byref(d), qp, kp, bp, lse.data_ptr(), _stream_ptr(stream, q.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_row_lse")
    return lse


def kvpop_future_attn_from_lse(q, k, lse, scale: float, window: int = 0, horizon: int = -1, key_bias=None,
                               out=None, stream=None):
    """Pass 2: per-key future mass from a given normaliser, fp32 [B, Hq, T] (eq. future_mass_app)."""
    torch = _torch()
    d = _dims(q, k, scale)
    qp, kp, bp = _prep_inputs(q, k, key_bias)
    _check_tensor(lse, "lse", torch.float32, q.device)
    if tuple(lse.shape) != (d.batch, d.n_q_heads, d.seq_len):
        raise ValueError("lse must be [B, Hq, T]")
    out = _prep_out(out, "out", (d.batch, d.n_q_heads, d.seq_len), q.device)
    st = lib().kvpop_future_attn_from_lse(ctypes.byref(d), qp, kp, bp, lse.data_ptr(), int(window), int(horizon),
                                          out.data_ptr(), _stream_ptr(stream, q.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_future_attn_from_lse")
    return out


def kvpop_future_attn_bands(q, k, lse, scale: float, bands, key_bias=None, outs=None, stream=None):
    """Pass 2 for one or two (window, horizon) bands from one normaliser in one sweep;
    returns a list of fp32 [B, Hq, T] masses, one per band."""
    torch = _torch()
    d = _dims(q, k, scale)
    qp, kp, bp = _prep_inputs(q, k, key_bias)
    _check_tensor(lse, "lse", torch.float32, q.device)
    shape = (d.batch, d.n_q_heads, d.seq_len)
    if tuple(lse.shape) != shape:
        raise ValueError("lse must be [B, Hq, T]")
    bands = [(int(a), int(b)) for a, b in bands]
    if not 1 <= len(bands) <= 2:
        raise ValueError("one or two bands")
    outs = [None] * len(bands) if outs is None else list(outs)
    if len(outs) != len(bands):
        raise ValueError("one output per band")
    outs = [_prep_out(o, "outs[%d]" % i, shape, q.device) for i, o in enumerate(outs)]
    n = len(bands)
    win = (ctypes.c_int32 * n)(*[b[0] for b in bands])
    hor = (ctypes.c_int32 * n)(*[b[1] for b in bands])
    ptr = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    st = lib().kvpop_future_attn_bands(ctypes.byref(d), qp, kp, bp, lse.data_ptr(), n, win, hor, ptr,
                                       _stream_ptr(stream, q.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_future_attn_bands")
    return outs


def kvpop_future_attn_target(q, k, scale: float, window: int = 0, horizon: int = -1, key_bias=None,
                             lse_ws=None, out=None, stream=None) -> Tuple["object", "object"]:
    """Both passes; returns (out, lse) where lse is the dense normaliser of pass 1."""
    d = _dims(q, k, scale)
    qp, kp, bp = _prep_inputs(q, k, key_bias)
    shape = (d.batch, d.n_q_heads, d.seq_len)
    lse_ws = _prep_out(lse_ws, "lse_ws", shape, q.device)
    out = _prep_out(out, "out", shape, q.device)
    st = lib().kvpop_future_attn_target(ctypes.byref(d), qp, kp, bp, int(window), int(horizon), lse_ws.data_ptr(),
                                        out.data_ptr(), _stream_ptr(stream, q.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_future_attn_target")
    return out, lse_ws


def kvpop_future_attn_scores(q, k, lse, scale: float, window: int = 0, horizon: int = -1, agg: str = "max",
                             eps: float = 1e-8, normalize: bool = True, key_bias=None, scores=None, out=None,
                             write_mass: bool = False, stream=None):
    """Pass 2 plus the target epilogue (App. D.4 step 5): per-KV-head scores
    log(agg_g m_bar + eps) - log N_t, fp32 [B, Hkv, T]. Returns (scores, out), where
    out holds the per-head masses if ``write_mass`` (or ``out``) is given, else None.
    Where that is faster the masses get an array of their own for the time of the call
    (B * Hq * T floats), but not while the stream is being captured: a captured call takes
    the faster form only with ``write_mass`` or ``out``."""
    torch = _torch()
    d = _dims(q, k, scale)
    qp, kp, bp = _prep_inputs(q, k, key_bias)
    _check_tensor(lse, "lse", torch.float32, q.device)
    if tuple(lse.shape) != (d.batch, d.n_q_heads, d.seq_len):
        raise ValueError("lse must be [B, Hq, T]")
    if agg not in ("max", "mean"):
        raise ValueError("agg must be 'max' or 'mean'")
    scores = _prep_out(scores, "scores", (d.batch, d.n_kv_heads, d.seq_len), q.device)
    if out is not None or write_mass:
        out = _prep_out(out, "out", (d.batch, d.n_q_heads, d.seq_len), q.device)
    # On a small problem with a long band the library spreads the query heads over the
    # GPU if it can write the masses: give it room, except under capture, whose replays
    # would write to it after it is freed.
    mass, L, dims = out, lib(), ctypes.byref(d)
    if mass is None and L.kvpop_internal_scores_spread(dims, int(window), int(horizon)):
        if stream is None and q.device.index == torch.cuda.current_device():  # no context: a small call's time is host time
            if not torch.cuda.is_current_stream_capturing():
                mass = torch.empty(lse.shape, dtype=torch.float32, device=q.device)
        else:
            with _on_launch_stream(stream, q.device):
                if not torch.cuda.is_current_stream_capturing():
                    mass = torch.empty(lse.shape, dtype=torch.float32, device=q.device)
    st = L.kvpop_future_attn_scores(dims, qp, kp, bp, lse.data_ptr(), int(window), int(horizon),
                                    KVPOP_AGG_MAX if agg == "max" else KVPOP_AGG_MEAN, float(eps),
                                    int(bool(normalize)), mass.data_ptr() if mass is not None else None,
                                    scores.data_ptr(), _stream_ptr(stream, q.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_future_attn_scores")
    return scores, out


def kvpop_running_topk_workspace_size(batch: int, n_heads: int, seq_len: int) -> int:
    d = KvpopTopkDims(batch, n_heads, seq_len)
    return int(lib().kvpop_running_topk_workspace_size(ctypes.byref(d)))


def kvpop_running_topk(scores, sinks: int, window: int, topk: int, log_gamma=None, labels: bool = True,
                       evict: bool = False, workspace=None, stream=None):
    """Ranks, running cutoffs and (optionally) teacher labels and boundary tokens, and
    token eviction queries, for scores [B, H, T] (App. B.3, App. C). Returns a dict of
    int32 tensors."""
    torch = _torch()
    _check_tensor(scores, "scores", torch.float32, None)
    if scores.dim() != 3:
        raise ValueError("scores must be [B, H, T]")
    B, H, T = scores.shape
    if log_gamma is not None:
        _check_tensor(log_gamma, "log_gamma", torch.float32, scores.device)
        if tuple(log_gamma.shape) != (H,):
            raise ValueError("log_gamma must be [H]")
    need = kvpop_running_topk_workspace_size(B, H, T)
    if need == 0:
        raise ValueError("invalid dimensions")
    if workspace is None:
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=scores.device)
        else:
            with _on_launch_stream(stream, scores.device):
                workspace = torch.empty(need, dtype=torch.uint8, device=scores.device)
    else:
        _check_workspace(workspace, need, scores.device)
    out = {n: torch.empty((B, H, T), dtype=torch.int32, device=scores.device) for n in ("rank", "cutoff")}
    if labels:
        out["label"] = torch.empty((B, H, T), dtype=torch.int32, device=scores.device)
        out["boundary"] = torch.empty((B, H, T), dtype=torch.int32, device=scores.device)
    if evict:
        out["evict"] = torch.empty((B, H, T), dtype=torch.int32, device=scores.device)
    d = KvpopTopkDims(B, H, T)
    st = lib().kvpop_running_topk(ctypes.byref(d), scores.data_ptr(),
                                  log_gamma.data_ptr() if log_gamma is not None else None, int(sinks), int(window),
                                  int(topk), out["rank"].data_ptr(), out["cutoff"].data_ptr(),
                                  out["label"].data_ptr() if labels else None,
                                  out["boundary"].data_ptr() if labels else None,
                                  out["evict"].data_ptr() if evict else None, workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _stream_ptr(stream, scores.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_running_topk")
    return out


def kvpop_running_topk_noalloc(scores, sinks: int, window: int, topk: int, log_gamma=None, labels: bool = True,
                               evict: bool = False, out=None, stream=None):
    """kvpop_running_topk without a workspace: the library's own per-GPU scratch array
    serves instead (see include/kvpop.h). ``out`` may hold preallocated int32 [B, H, T]
    outputs ("rank", "cutoff" and, as requested, "label", "boundary", "evict"), so that
    the call itself allocates nothing; missing ones are allocated here."""
    torch = _torch()
    _check_tensor(scores, "scores", torch.float32, None)
    if scores.dim() != 3:
        raise ValueError("scores must be [B, H, T]")
    B, H, T = scores.shape
    if log_gamma is not None:
        _check_tensor(log_gamma, "log_gamma", torch.float32, scores.device)
        if tuple(log_gamma.shape) != (H,):
            raise ValueError("log_gamma must be [H]")
    names = ["rank", "cutoff"] + (["label", "boundary"] if labels else []) + (["evict"] if evict else [])
    res = {}
    for n in names:
        x = (out or {}).get(n)
        if x is None:
            x = torch.empty((B, H, T), dtype=torch.int32, device=scores.device)
        else:
            _check_tensor(x, n, torch.int32, scores.device)
            if tuple(x.shape) != (B, H, T):
                raise ValueError("%s must be [B, H, T]" % n)
        res[n] = x
    d = KvpopTopkDims(B, H, T)
    ptr = lambda n: res[n].data_ptr() if n in res else None  # noqa: E731
    st = lib().kvpop_running_topk_noalloc(ctypes.byref(d), scores.data_ptr(),
                                          log_gamma.data_ptr() if log_gamma is not None else None, int(sinks),
                                          int(window), int(topk), ptr("rank"), ptr("cutoff"), ptr("label"),
                                          ptr("boundary"), ptr("evict"), _stream_ptr(stream, scores.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_running_topk_noalloc")
    return res


def kvpop_sparse_attn_fwd(q, k, v, evict, scale: float, key_bias=None, o=None, lse=None, stream=None):
    """Running top-k sparse attention forward (Sec. 3.2, App. C): key t of KV head h is
    kept by query q iff t <= q < evict[b, h, t]. Returns (o bf16 [B, Hq, T, D],
    lse fp32 [B, Hq, T])."""
    torch = _torch()
    d = _dims(q, k, scale)
    qp, kp, bp = _prep_inputs(q, k, key_bias)
    _check_tensor(v, "v", torch.bfloat16, q.device)
    if tuple(v.shape) != tuple(k.shape):
        raise ValueError("v must have the shape of k")
    _check_tensor(evict, "evict", torch.int32, q.device)
    if tuple(evict.shape) != (d.batch, d.n_kv_heads, d.seq_len):
        raise ValueError("evict must be [B, Hkv, T]")
    if o is None:
        o = torch.empty(tuple(q.shape), dtype=torch.bfloat16, device=q.device)
    else:
        _check_tensor(o, "o", torch.bfloat16, q.device)
        if tuple(o.shape) != tuple(q.shape):
            raise ValueError("o must have the shape of q")
    lse = _prep_out(lse, "lse", (d.batch, d.n_q_heads, d.seq_len), q.device)
    st = lib().kvpop_sparse_attn_fwd(ctypes.byref(d), qp, kp, v.data_ptr(), bp, evict.data_ptr(), o.data_ptr(),
                                     lse.data_ptr(), _stream_ptr(stream, q.device))
    if st != KVPOP_OK:
        raise KvpopError(st, "kvpop_sparse_attn_fwd")
    return o, lse


# ---------------------------------------------------------------------------
# The compact cache (include/kvpop_cache.h)
# ---------------------------------------------------------------------------

class KvpopCache(NamedTuple):
    """A pool of 8-bit pages and the page lists of B sequences of H KV heads.

    k_pages, v_pages: int8 or float8_e4m3fn [n_pages, P, D], P 16, 32, 64 or 128, D 64 or
    128; k_exp, v_exp: int8 [n_pages], a page's values are code * 2 ** exp; page_table:
    int32 [B, H, max_pages], slot j of a list is row j % P of entry j // P."""
    k_pages: Any
    v_pages: Any
    k_exp: Any
    v_exp: Any
    page_table: Any


def kvpop_cache_empty(batch: int, n_kv_heads: int, tokens: int, head_dim: int, page_size: int = 64,
                      dtype=None, device="cuda") -> KvpopCache:
    """A cache with room for ``tokens`` tokens in each list, its pages dealt to the lists in
    order. dtype: torch.int8 (the default) or torch.float8_e4m3fn."""
    torch = _torch()
    if page_size not in (16, 32, 64, 128) or head_dim not in (64, 128):
        raise ValueError("page_size must be 16, 32, 64 or 128, and head_dim 64 or 128")
    if batch < 1 or n_kv_heads < 1 or tokens < 1:
        raise ValueError("batch, n_kv_heads and tokens must be positive")
    if dtype not in (None, torch.int8, torch.float8_e4m3fn):
        raise TypeError("dtype must be int8 or float8_e4m3fn")
    per = -(-tokens // page_size)
    n = batch * n_kv_heads * per
    dtype = torch.int8 if dtype is None else dtype
    pages = [torch.zeros((n, page_size, head_dim), dtype=torch.int8, device=device).view(dtype) for _ in range(2)]
    exps = [torch.zeros(n, dtype=torch.int8, device=device) for _ in range(2)]
    table = torch.arange(n, dtype=torch.int32, device=device).view(batch, n_kv_heads, per)
    return KvpopCache(pages[0], pages[1], exps[0], exps[1], table)


# The mirrors' fields in order, for calls that pack them at once.
_CACHE_PACK = struct.Struct("7i4x5P")
_ROWS_PACK = struct.Struct("P3q")
_APPEND_PACK = struct.Struct("2i P3q P3q 7P 4i P3q P")
_RETAIN_PACK = struct.Struct("3i4x3P")


def _need(ok: bool, text: str):
    if not ok:
        raise ValueError(text)


def _ptr(x, name: str, dtype, shape, dev: int) -> int:
    """The address of a contiguous tensor of this type and shape on GPU ``dev``; 0 for None."""
    if x is None:
        return 0
    try:
        if x.dtype is dtype and x.get_device() == dev and x.shape == shape and x.is_contiguous():
            return x.data_ptr()
    except AttributeError:
        pass
    _check_tensor(x, name, dtype, _torch().device("cuda", dev))
    raise ValueError("%s must be %s" % (name, list(shape)))


def _cache_parts(torch, cache):
    """A cache checked: (packed kvpop_cache, B, H, D, GPU index)."""
    k, v, ke, ve, table = cache
    i8 = torch.int8
    dtype = getattr(k, "dtype", None)
    if dtype is not i8 and dtype is not torch.float8_e4m3fn:
        raise TypeError("k_pages must be int8 or float8_e4m3fn")
    if not k.is_cuda:
        _check_tensor(k, "k_pages", dtype, None)
    _need(k.dim() == 3, "k_pages must be [n_pages, P, D]")
    dev = k.get_device()
    shape = k.shape
    n, P, D = shape
    _need(getattr(table, "shape", None) is not None and len(table.shape) == 3, "page_table must be [B, H, max_pages]")
    B, H, per = table.shape
    packed = _CACHE_PACK.pack(B, H, D, KVPOP_CACHE_INT8 if dtype is i8 else KVPOP_CACHE_E4M3, P, n, per,
                              _ptr(k, "k_pages", dtype, shape, dev), _ptr(v, "v_pages", dtype, shape, dev),
                              _ptr(ke, "k_exp", i8, (n,), dev), _ptr(ve, "v_exp", i8, (n,), dev),
                              _ptr(table, "page_table", torch.int32, (B, H, per), dev))
    return packed, B, H, D, dev


def _rows(torch, x, name: str, B: int, heads, N, D: int, dev: int):
    """A bf16 tensor [B, heads, N, D] (heads, N None: any), strided but for its last dimension:
    (address, strides of its first three), its heads and its tokens."""
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if x.get_device() != dev:
        raise ValueError("%s must be on the GPU device of the cache" % name)
    if x.dtype is not torch.bfloat16:
        raise TypeError("%s must be %s, got %s" % (name, torch.bfloat16, x.dtype))
    shape = x.shape
    if len(shape) != 4 or shape[0] != B or shape[3] != D or (heads or shape[1]) != shape[1] or (N or shape[2]) != shape[2]:
        raise ValueError("%s must be [B, heads, N, D] = %s, got %s" % (name, [B, heads, N, D], list(shape)))
    sb, sh, st, sd = x.stride()
    if sd != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    # The stride of a dimension of one element means nothing.
    _, h, n, _ = shape
    return (x.data_ptr(), sb if B > 1 else 0, sh if h > 1 else 0, st if n > 1 else 0), h, n


def _current(torch, dev: int):
    """(handle of GPU ``dev``'s current stream, current GPU). torch's own short ways, 0.2 us where the
    public ones take 1.4; those serve where a version of torch lacks the others."""
    try:
        return torch._C._cuda_getCurrentRawStream(dev), torch._C._cuda_getDevice()
    except AttributeError:
        return int(torch.cuda.current_stream(dev).cuda_stream), torch.cuda.current_device()


def _call(torch, f, dev: int, stream, *args):
    """Calls entry point ``f`` on ``stream`` or the current one of GPU ``dev``, which is made the current
    device: the default stream's handle is that of whichever device is current."""
    handle, current = _current(torch, dev)
    if stream is not None:
        handle = int(stream.cuda_stream)
    if dev == current:
        st = f(*args, handle)
    else:
        with torch.cuda.device(dev):
            st = f(*args, handle)
    if st != KVPOP_OK:
        raise KvpopError(st, f.__name__)


def kvpop_cache_append(cache: KvpopCache, k, v, held, count=None, start=None, src=None, q=None, rotary=None,
                       pos0=None, adjacent: bool = False, q_out=None, stream=None):
    """New keys and values into the lists' pages, the keys (and queries) turned by their
    positions. k, v: bf16 [B, H, N, D] (any strides that are multiples of 8); held: int32
    [B, H], the lists' lengths after the call; count: int32 [B, H], how many tokens each list takes
    (None: all); start: int32 [B, H], the first slot written, negative for none (None: held -
    count); src: int32 [B, H, M], which tokens (None: 0, 1, ...); rotary: (cos, sin), fp32
    [positions, R / 2] each; pos0: int32 [B], the position of token 0 (None: 0); adjacent: pairs
    (2 j, 2 j + 1) instead of (j, j + R / 2). With q (bf16 [B, Hq, N, D]) returns it rotated,
    bf16 [B, Hq, N, D] contiguous; else None. include/kvpop_cache.h has the exponents' rule."""
    torch = _torch()
    i32, bf16 = torch.int32, torch.bfloat16
    c, B, H, D, dev = _cache_parts(torch, cache)
    kr, _, N = _rows(torch, k, "k", B, H, None, D, dev)
    vr, _, _ = _rows(torch, v, "v", B, H, N, D, dev)
    M = N
    if src is not None:
        M = src.shape[-1] if src.dim() == 3 else 0
    lists = (B, H)
    cos = sin = n_positions = rot = 0
    if rotary is not None:
        t_cos, t_sin = rotary
        _need(len(getattr(t_cos, "shape", ())) == 2, "cos and sin must be [positions, R / 2]")
        n_positions, rot = t_cos.shape
        cos = _ptr(t_cos, "cos", torch.float32, (n_positions, rot), dev)
        sin = _ptr(t_sin, "sin", torch.float32, (n_positions, rot), dev)
    qr, Hq, qo = (0, 0, 0, 0), 0, 0
    if q is not None:
        qr, Hq, _ = _rows(torch, q, "q", B, None, N, D, dev)
        if q_out is None:
            q_out = torch.empty((B, Hq, N, D), dtype=bf16, device=q.device)
        qo = _ptr(q_out, "q_out", bf16, (B, Hq, N, D), dev)
    elif q_out is not None:
        raise ValueError("q_out without q")
    a = _APPEND_PACK.pack(N, M, *kr, *vr, _ptr(held, "held", i32, lists, dev), _ptr(count, "count", i32, lists, dev),
                          _ptr(start, "start", i32, lists, dev), _ptr(src, "src", i32, (B, H, M), dev),
                          _ptr(pos0, "pos0", i32, (B,), dev), cos, sin, n_positions, 2 * rot, 1 if adjacent else 0, Hq,
                          *qr, qo)
    _call(torch, lib().kvpop_cache_append, dev, stream, c, a)
    return q_out


def kvpop_cache_attn_workspace_size(cache: KvpopCache, n_q_heads: int, n_tokens: int) -> int:
    """Bytes of workspace of a kvpop_cache_attn call with q [B, n_q_heads, n_tokens, D]."""
    return int(lib().kvpop_cache_attn_workspace_size(_cache_parts(_torch(), cache)[0], n_q_heads, n_tokens))


def kvpop_cache_attn(q, cache: KvpopCache, held, scale: float, q_lens=None, o=None, lse=None, workspace=None,
                     stream=None):
    """Attention of the newest queries q (bf16 [B, Hq, N, D]) over the lists: query i of the n =
    q_lens[b] (None: N) of a sequence sees the slots below held[b, h] - (n - 1 - i), so several
    queries at once are for lists that their tokens were added to at the end. Returns
    (o bf16 [B, Hq, N, D], lse fp32 [B, Hq, N]); rows from n on, and queries that see
    nothing, get 0 and -inf."""
    torch = _torch()
    i32 = torch.int32
    c, B, H, D, dev = _cache_parts(torch, cache)
    qr, Hq, N = _rows(torch, q, "q", B, None, None, D, dev)
    if o is None:
        o = torch.empty((B, Hq, N, D), dtype=torch.bfloat16, device=q.device)
    if lse is None:
        lse = torch.empty((B, Hq, N), dtype=torch.float32, device=q.device)
    need = lib().kvpop_cache_attn_workspace_size(c, Hq, N)
    if workspace is None:
        if need:
            if stream is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            else:
                with _on_launch_stream(stream, q.device):
                    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    else:
        _check_workspace(workspace, need, q.device)
    _call(torch, lib().kvpop_cache_attn, dev, stream, c, Hq, N, float(scale), _ROWS_PACK.pack(*qr),
          _ptr(held, "held", i32, (B, H), dev), _ptr(q_lens, "q_lens", i32, (B,), dev),
          _ptr(o, "o", torch.bfloat16, (B, Hq, N, D), dev), _ptr(lse, "lse", torch.float32, (B, Hq, N), dev),
          workspace.data_ptr() if workspace is not None else 0, need)
    return o, lse


def kvpop_retain_prompt(evict, scores, budget: int, log_gamma=None, lens=None, pos=None, prio=None, held=None,
                        stream=None):
    """The tokens that a prompt's end keeps, from kvpop_running_topk's evict and its scores
    (both [B, H, T]): (pos int32 [B, H, budget], prio fp32 [B, H, budget], held int32 [B, H]),
    ascending positions, then -1 and -inf. lens: int32 [B], the prompts' lengths (None: T)."""
    torch = _torch()
    i32, f32 = torch.int32, torch.float32
    _check_tensor(scores, "scores", f32, None)
    _need(scores.dim() == 3, "scores must be [B, H, T]")
    device, dev = scores.device, scores.get_device()
    B, H, T = scores.shape
    S = int(budget)
    _need(S >= 1, "budget must be positive")
    if pos is None:
        pos = torch.empty((B, H, S), dtype=i32, device=device)
    if prio is None:
        prio = torch.empty((B, H, S), dtype=f32, device=device)
    if held is None:
        held = torch.empty((B, H), dtype=i32, device=device)
    st = _RETAIN_PACK.pack(B, H, S, _ptr(pos, "pos", i32, (B, H, S), dev), _ptr(prio, "prio", f32, (B, H, S), dev),
                           _ptr(held, "held", i32, (B, H), dev))
    _call(torch, lib().kvpop_retain_prompt, dev, stream, st, T, _ptr(evict, "evict", i32, (B, H, T), dev), scores.data_ptr(),
          _ptr(log_gamma, "log_gamma", f32, (H,), dev), _ptr(lens, "lens", i32, (B,), dev))
    return pos, prio, held


def kvpop_retain_step(scores, q_pos, pos, prio, held, sinks: int, window: int, topk: int, log_gamma=None,
                      slot=None, stream=None):
    """The running top-k for single tokens: which slot (int32 [B, H], -1 for none) the
    token at q_pos (int32 [B], negative for an idle sequence) takes in each list of at most sinks
    + window + topk tokens. scores: fp32 [B, H], of the token at q_pos - window, which leaves
    the protected window. Updates pos, prio ([B, H, S]) and held ([B, H]) in place."""
    torch = _torch()
    i32, f32 = torch.int32, torch.float32
    _check_tensor(pos, "pos", i32, None)
    shape = pos.shape
    _need(len(shape) == 3, "pos must be [B, H, S]")
    dev = pos.get_device()
    B, H, S = shape
    lists = (B, H)
    if slot is None:
        slot = torch.empty(lists, dtype=i32, device=pos.device)
    st = _RETAIN_PACK.pack(B, H, S, pos.data_ptr(), _ptr(prio, "prio", f32, shape, dev), _ptr(held, "held", i32, lists, dev))
    _call(torch, lib().kvpop_retain_step, dev, stream, st, _ptr(scores, "scores", f32, lists, dev),
          _ptr(log_gamma, "log_gamma", f32, (H,), dev), _ptr(q_pos, "q_pos", i32, (B,), dev), int(sinks), int(window),
          int(topk), _ptr(slot, "slot", i32, lists, dev))
    return slot
