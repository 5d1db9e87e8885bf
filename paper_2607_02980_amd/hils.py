"""ctypes binding of libhils.so -- argument marshalling only.

The entry points keep the C names (``hils_prefill_fwd``, ``hils_decode_fwd``,
``hils_decode_fwd_noalloc``, ``hils_decode_paged_fwd``, ``hils_bwd``,
``hils_landmark_fwd``, ``hils_landmark_bwd``, ``hils_q8_append``,
``hils_q8_landmark_fwd``, ``hils_decode_q8_fwd``, ``hils_cache_evict``,
``hils_prefill_paged_fwd``, ``hils_cache_reserve``, ``hils_cache_fork``,
``hils_cache_free``, ``hils_cache_compact``, ``hils_workspace_size``, ``hils_prefill_record_cap``, ``hils_last_error``, ``hils_version``).
They take torch tensors already resident on the GPU, check dtype, shape,
device and contiguity, allocate missing outputs and the workspace with
``torch.empty`` and pass raw pointers plus the current HIP stream.  Every step
of the computation runs in the library's HIP kernels; there is no fallback:
if ``libhils.so`` is missing or fails to load, importing this module raises.
"""
from __future__ import annotations

import ctypes
import operator
import os
from dataclasses import dataclass

import torch

# HILS_LIB names another build of the same sources (the sanitizer build of the
# host code, libhils_san.so); by default the in-tree libhils.so
_LIB_PATH = os.environ.get("HILS_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhils.so")

HILS_F32, HILS_BF16 = 0, 1
HILS_OK, HILS_ERR_INVALID, HILS_ERR_UNSUPPORTED, HILS_ERR_WORKSPACE, HILS_ERR_HIP = range(5)
HILS_FLAG_GIVEN_IDX = 1
HILS_FLAG_SHARED_LMK_QUERY = 2
HILS_FLAG_HEAD_NORM_SELECT = 4
HILS_FLAG_UNION_PACKING = 8
HILS_OP_PREFILL, HILS_OP_DECODE, HILS_OP_BWD, HILS_OP_LANDMARK = 0, 1, 2, 3
HILS_OP_DECODE_Q8, HILS_OP_Q8_APPEND, HILS_OP_Q8_LANDMARK, HILS_OP_CACHE_EVICT = 4, 5, 6, 7
HILS_OP_PREFILL_PAGED, HILS_OP_CACHE_RESERVE, HILS_OP_CACHE_FORK, HILS_OP_CACHE_FREE, HILS_OP_CACHE_COMPACT = 8, 9, 10, 11, 12


class HilsError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"hils error {code}: {msg}")
        self.code = code


class hils_params(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("Hq", ctypes.c_int), ("Hkv", ctypes.c_int), ("Hl", ctypes.c_int),
                ("N", ctypes.c_int), ("L", ctypes.c_int), ("d", ctypes.c_int), ("chunk", ctypes.c_int),
                ("topk", ctypes.c_int), ("window", ctypes.c_int), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int), ("flags", ctypes.c_uint)]


class hils_pool(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_bytes", ctypes.c_size_t)]


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run `python -m paper_2607_02980_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    P = ctypes.POINTER(hils_params)
    lib.hils_version.restype = ctypes.c_int
    lib.hils_last_error.restype = ctypes.c_char_p
    lib.hils_workspace_size.argtypes = [P, ctypes.c_int, ctypes.POINTER(sz)]
    lib.hils_prefill_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hils_decode_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hils_decode_paged_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp, vp, vp, vp, sz, vp]
    lib.hils_decode_fwd_noalloc.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.hils_bwd.argtypes = [P] + [vp] * 17 + [sz, vp]
    lib.hils_landmark_fwd.argtypes = [P, vp, vp, vp, vp, vp]
    lib.hils_landmark_bwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    ci = ctypes.c_int
    lib.hils_q8_append.argtypes = [P, vp, vp, vp, vp, vp, vp, ci, vp, vp, vp]
    lib.hils_q8_landmark_fwd.argtypes = [P, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp]
    lib.hils_decode_q8_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hils_cache_evict.argtypes = [P, vp, vp, vp, vp, vp, ci, ci, ci, vp, vp, vp, vp, vp, vp]
    lib.hils_prefill_paged_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hils_cache_reserve.argtypes = [P, vp, vp, ci, vp, vp, vp, ci, vp, vp, vp, vp, vp]
    lib.hils_cache_fork.argtypes = [P, vp, ci, vp, vp, ci, vp, vp, vp, vp, vp]
    lib.hils_cache_free.argtypes = [P, vp, vp, vp, ci, vp, vp, ci, vp, vp, vp, vp, vp]
    lib.hils_cache_compact.argtypes = [P, vp, vp, ci, vp, vp, ci, vp, vp, vp, vp, vp, vp]
    lib.hils_prefill_record_cap.argtypes = [sz]
    lib.hils_prefill_record_cap.restype = sz
    lib.hils_timing_enable.argtypes = [ctypes.c_int]
    lib.hils_timing_read.argtypes = [ctypes.c_char_p, sz, ctypes.POINTER(ctypes.c_float),
                                     ctypes.POINTER(ctypes.c_int), ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    for f in (lib.hils_workspace_size, lib.hils_prefill_fwd, lib.hils_decode_fwd, lib.hils_decode_fwd_noalloc,
              lib.hils_bwd,
              lib.hils_landmark_fwd, lib.hils_landmark_bwd, lib.hils_q8_append, lib.hils_q8_landmark_fwd,
              lib.hils_decode_q8_fwd, lib.hils_cache_evict, lib.hils_prefill_paged_fwd, lib.hils_cache_reserve,
              lib.hils_cache_fork, lib.hils_cache_free, lib.hils_cache_compact, lib.hils_timing_enable, lib.hils_timing_read):
        f.restype = ctypes.c_int
    return lib


LIB = _load()


@dataclass
class Params:
    """Python mirror of ``hils_params``."""
    B: int
    Hq: int
    Hkv: int
    N: int
    L: int
    d: int
    chunk: int = 64
    topk: int = 16
    window: int = 512
    scale: float | None = None
    dtype: str = "bf16"
    Hl: int = 0
    flags: int = 0

    def c(self) -> hils_params:
        return hils_params(self.B, self.Hq, self.Hkv, self.Hl or self.Hq, self.N, self.L, self.d, self.chunk,
                           self.topk, self.window, float(self.scale if self.scale is not None else self.d ** -0.5),
                           HILS_BF16 if self.dtype == "bf16" else HILS_F32, self.flags)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32


def hils_version() -> int:
    return LIB.hils_version()


def hils_prefill_record_cap(nbytes: int = 0) -> int:
    """Set (nbytes > 0) and/or read the chunk-major prefill's cap on the per-slot
    records of one segment of rows; returns the previous cap."""
    return int(LIB.hils_prefill_record_cap(int(nbytes)))


def hils_last_error() -> str:
    return LIB.hils_last_error().decode()


def _check(rc: int):
    if rc != HILS_OK:
        raise HilsError(rc, hils_last_error())


def hils_workspace_size(p: Params, op: int) -> int:
    n = ctypes.c_size_t(0)
    cp = p.c()
    _check(LIB.hils_workspace_size(ctypes.byref(cp), op, ctypes.byref(n)))
    return n.value


def _ptr(t, name, shape=None, dtype=None, required=True):
    if t is None:
        if required:
            raise ValueError(f"{name} is required")
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _workspace(p: Params, op: int, workspace):
    n = hils_workspace_size(p, op)
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    if workspace.numel() < n:
        raise ValueError(f"workspace has {workspace.numel()} bytes, {n} needed")
    return workspace, n


def _shapes(p: Params):
    nc = p.L // p.chunk
    Hl = p.Hl or p.Hq
    return {"q": (p.B, p.Hq, p.N, p.d), "kv": (p.B, p.Hkv, p.L, p.d), "lmk": (p.B, Hl, nc, p.d),
            "bias": (p.B, Hl, nc), "lse": (p.B, p.Hq, p.N), "idx": (p.B, p.Hkv, p.N, p.topk)}


def hils_prefill_fwd(p: Params, q, k, v, lmk, lmk_bias=None, q_route=None, out=None, lse=None, idx=None,
                     workspace=None):
    """Prefill forward.  Returns (out, lse, idx).  With ``p.flags & HILS_FLAG_GIVEN_IDX``
    the given ``idx`` is consumed instead of selected."""
    S, dt = _shapes(p), p.torch_dtype
    if out is None:
        out = torch.empty(S["q"], dtype=dt, device=q.device)
    if lse is None:
        lse = torch.empty(S["lse"], dtype=torch.float32, device=q.device)
    if idx is None:
        if p.flags & HILS_FLAG_GIVEN_IDX:
            raise ValueError("HILS_FLAG_GIVEN_IDX needs idx")
        idx = torch.empty(S["idx"], dtype=torch.int32, device=q.device)
    ws, n = _workspace(p, HILS_OP_PREFILL, workspace)
    cp = p.c()
    _check(LIB.hils_prefill_fwd(
        ctypes.byref(cp), _ptr(q, "q", S["q"], dt), _ptr(k, "k", S["kv"], dt), _ptr(v, "v", S["kv"], dt),
        _ptr(lmk, "lmk", S["lmk"], dt), _ptr(lmk_bias, "lmk_bias", S["bias"], torch.float32, False),
        _ptr(q_route, "q_route", S["q"], dt, False), _ptr(out, "out", S["q"], dt),
        _ptr(lse, "lse", S["lse"], torch.float32), _ptr(idx, "idx", S["idx"], torch.int32),
        _ptr(ws, "workspace"), n, _stream()))
    return out, lse, idx


def hils_decode_fwd(p: Params, q, k_cache, v_cache, lmk_cache, lmk_bias=None, q_route=None, seqlens=None,
                    out=None, lse=None, idx=None, workspace=None):
    """Decode forward, N >= 1 new queries per sequence (query n at seqlens[b] - N + n).
    Returns (out, lse, idx)."""
    S, dt = _shapes(p), p.torch_dtype
    if out is None:
        out = torch.empty(S["q"], dtype=dt, device=q.device)
    if lse is None:
        lse = torch.empty(S["lse"], dtype=torch.float32, device=q.device)
    if idx is None:
        if p.flags & HILS_FLAG_GIVEN_IDX:
            raise ValueError("HILS_FLAG_GIVEN_IDX needs idx")
        idx = torch.empty(S["idx"], dtype=torch.int32, device=q.device)
    ws, n = _workspace(p, HILS_OP_DECODE, workspace)
    cp = p.c()
    _check(LIB.hils_decode_fwd(
        ctypes.byref(cp), _ptr(q, "q", S["q"], dt), _ptr(k_cache, "k_cache", S["kv"], dt),
        _ptr(v_cache, "v_cache", S["kv"], dt), _ptr(lmk_cache, "lmk_cache", S["lmk"], dt),
        _ptr(lmk_bias, "lmk_bias", S["bias"], torch.float32, False), _ptr(q_route, "q_route", S["q"], dt, False),
        _ptr(seqlens, "seqlens", (p.B,), torch.int32, False), _ptr(out, "out", S["q"], dt),
        _ptr(lse, "lse", S["lse"], torch.float32), _ptr(idx, "idx", S["idx"], torch.int32),
        _ptr(ws, "workspace"), n, _stream()))
    return out, lse, idx


HILS_DECODE_NOALLOC_SCRATCH_BYTES = 64 << 20


def hils_decode_fwd_noalloc(p: Params, q, k_cache, v_cache, lmk_cache, lmk_bias=None, q_route=None, seqlens=None,
                            out=None, lse=None, idx=None):
    """hils_decode_fwd without a workspace: the library's fixed per-GPU array
    (HILS_DECODE_NOALLOC_SCRATCH_BYTES) serves as the workspace.  Outputs not
    given are allocated here with torch.empty (the C call itself allocates
    nothing).  Returns (out, lse, idx)."""
    S, dt = _shapes(p), p.torch_dtype
    if out is None:
        out = torch.empty(S["q"], dtype=dt, device=q.device)
    if lse is None:
        lse = torch.empty(S["lse"], dtype=torch.float32, device=q.device)
    if idx is None:
        if p.flags & HILS_FLAG_GIVEN_IDX:
            raise ValueError("HILS_FLAG_GIVEN_IDX needs idx")
        idx = torch.empty(S["idx"], dtype=torch.int32, device=q.device)
    cp = p.c()
    _check(LIB.hils_decode_fwd_noalloc(
        ctypes.byref(cp), _ptr(q, "q", S["q"], dt), _ptr(k_cache, "k_cache", S["kv"], dt),
        _ptr(v_cache, "v_cache", S["kv"], dt), _ptr(lmk_cache, "lmk_cache", S["lmk"], dt),
        _ptr(lmk_bias, "lmk_bias", S["bias"], torch.float32, False), _ptr(q_route, "q_route", S["q"], dt, False),
        _ptr(seqlens, "seqlens", (p.B,), torch.int32, False), _ptr(out, "out", S["q"], dt),
        _ptr(lse, "lse", S["lse"], torch.float32), _ptr(idx, "idx", S["idx"], torch.int32), _stream()))
    return out, lse, idx


def hils_decode_paged_fwd(p: Params, q, k_pages, v_pages, lmk_pages, block_table, bias_pages=None, q_route=None,
                          seqlens=None, out=None, lse=None, idx=None, workspace=None):
    """Decode forward over paged pools (one chunk per page): k/v_pages [P, Hkv, S, d],
    lmk_pages [P, Hl, d], bias_pages [P, Hl] f32, block_table [B, L/S] int32.
    Returns (out, lse, idx)."""
    S, dt = _shapes(p), p.torch_dtype
    P = k_pages.shape[0]
    Hl = p.Hl or p.Hq
    if out is None:
        out = torch.empty(S["q"], dtype=dt, device=q.device)
    if lse is None:
        lse = torch.empty(S["lse"], dtype=torch.float32, device=q.device)
    if idx is None:
        if p.flags & HILS_FLAG_GIVEN_IDX:
            raise ValueError("HILS_FLAG_GIVEN_IDX needs idx")
        idx = torch.empty(S["idx"], dtype=torch.int32, device=q.device)
    ws, n = _workspace(p, HILS_OP_DECODE, workspace)
    cp = p.c()
    _check(LIB.hils_decode_paged_fwd(
        ctypes.byref(cp), _ptr(q, "q", S["q"], dt), _ptr(k_pages, "k_pages", (P, p.Hkv, p.chunk, p.d), dt),
        _ptr(v_pages, "v_pages", (P, p.Hkv, p.chunk, p.d), dt), _ptr(lmk_pages, "lmk_pages", (P, Hl, p.d), dt),
        _ptr(bias_pages, "bias_pages", (P, Hl), torch.float32, False), _ptr(q_route, "q_route", S["q"], dt, False),
        _ptr(block_table, "block_table", (p.B, p.L // p.chunk), torch.int32), P,
        _ptr(seqlens, "seqlens", (p.B,), torch.int32, False), _ptr(out, "out", S["q"], dt),
        _ptr(lse, "lse", S["lse"], torch.float32), _ptr(idx, "idx", S["idx"], torch.int32),
        _ptr(ws, "workspace"), n, _stream()))
    return out, lse, idx


def hils_bwd(p: Params, dout, q, k, v, lmk, out, lse, idx, lmk_bias=None, q_route=None, want_dbias=True,
             workspace=None):
    """Backward with the selection fixed to ``idx``.  Returns dict(dq, dk, dv, dlmk, dlmk_bias, dq_route)."""
    S, dt = _shapes(p), p.torch_dtype
    dev = q.device
    dq = torch.empty(S["q"], dtype=dt, device=dev)
    dk = torch.empty(S["kv"], dtype=dt, device=dev)
    dv = torch.empty(S["kv"], dtype=dt, device=dev)
    dlmk = torch.empty(S["lmk"], dtype=dt, device=dev)
    dbias = torch.empty(S["bias"], dtype=torch.float32, device=dev) if want_dbias else None
    dqr = torch.empty(S["q"], dtype=dt, device=dev) if q_route is not None else None
    ws, n = _workspace(p, HILS_OP_BWD, workspace)
    cp = p.c()
    _check(LIB.hils_bwd(
        ctypes.byref(cp), _ptr(dout, "dout", S["q"], dt), _ptr(q, "q", S["q"], dt), _ptr(k, "k", S["kv"], dt),
        _ptr(v, "v", S["kv"], dt), _ptr(lmk, "lmk", S["lmk"], dt),
        _ptr(lmk_bias, "lmk_bias", S["bias"], torch.float32, False), _ptr(q_route, "q_route", S["q"], dt, False),
        _ptr(out, "out", S["q"], dt), _ptr(lse, "lse", S["lse"], torch.float32),
        _ptr(idx, "idx", S["idx"], torch.int32), _ptr(dq, "dq"), _ptr(dk, "dk"), _ptr(dv, "dv"),
        _ptr(dlmk, "dlmk"), _ptr(dbias, "dbias", required=False), _ptr(dqr, "dq_route", required=False),
        _ptr(ws, "workspace"), n, _stream()))
    return {"dq": dq, "dk": dk, "dv": dv, "dlmk": dlmk, "dlmk_bias": dbias, "dq_route": dqr}


def _lq_shape(p: Params, S):
    return (p.Hl or p.Hq, p.d) if p.flags & HILS_FLAG_SHARED_LMK_QUERY else S["lmk"]


def hils_landmark_fwd(p: Params, lq, k, lmk=None, lmk_bias=None):
    """Landmark compression (Prop. 3.1): lq [B, Hl, L/S, d] landmark queries (or
    [Hl, d] under HILS_FLAG_SHARED_LMK_QUERY) and k [B, Hkv, L, d] ->
    (lmk [B, Hl, L/S, d], lmk_bias [B, Hl, L/S] float32)."""
    S, dt = _shapes(p), p.torch_dtype
    dev = k.device
    lmk = torch.empty(S["lmk"], dtype=dt, device=dev) if lmk is None else lmk
    lmk_bias = torch.empty(S["bias"], dtype=torch.float32, device=dev) if lmk_bias is None else lmk_bias
    cp = p.c()
    _check(LIB.hils_landmark_fwd(ctypes.byref(cp), _ptr(lq, "lq", _lq_shape(p, S), dt), _ptr(k, "k", S["kv"], dt),
                                 _ptr(lmk, "lmk", S["lmk"], dt), _ptr(lmk_bias, "lmk_bias", S["bias"], torch.float32),
                                 _stream()))
    return lmk, lmk_bias


def hils_landmark_bwd(p: Params, lq, k, dlmk, dlmk_bias=None, dlq=None, dk=None, workspace=None):
    """Backward of hils_landmark_fwd -> (dlq [B, Hl, L/S, d] (or [Hl, d] under
    HILS_FLAG_SHARED_LMK_QUERY), dk [B, Hkv, L, d])."""
    S, dt = _shapes(p), p.torch_dtype
    dev = k.device
    lqs = _lq_shape(p, S)
    dlq = torch.empty(lqs, dtype=dt, device=dev) if dlq is None else dlq
    dk = torch.empty(S["kv"], dtype=dt, device=dev) if dk is None else dk
    ws, n = _workspace(p, HILS_OP_LANDMARK, workspace)
    cp = p.c()
    _check(LIB.hils_landmark_bwd(ctypes.byref(cp), _ptr(lq, "lq", lqs, dt), _ptr(k, "k", S["kv"], dt),
                                 _ptr(dlmk, "dlmk", S["lmk"], dt),
                                 _ptr(dlmk_bias, "dlmk_bias", S["bias"], torch.float32, False),
                                 _ptr(dlq, "dlq", lqs, dt), _ptr(dk, "dk", S["kv"], dt), _ptr(ws, "workspace"), n,
                                 _stream()))
    return dlq, dk


# ---- the 8-bit cache: k_pages [P, Hkv, S, d], v_pages [P, Hkv, d, S] and lmk_pages [P, Hl, d] are
# torch.float8_e4m3fn, kv_scale [P, Hkv, 2] and bias_pages [P, Hl] float32, block_table [B, L/S] int32.
# A single-token step of a small batch takes the GPU about as long as these checks take the host, so
# each tensor is looked at once and its address passed as an int.

_F8, _F32, _I32 = torch.float8_e4m3fn, torch.float32, torch.int32
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _address(t, name, shape, dtype, dev):
    """The address of a contiguous tensor of this shape and type on device number dev."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _ptr(t, name, shape, dtype)  # says what is wrong
    raise ValueError(f"{name} is on {t.device}, expected cuda:{dev}")


def _gpu(t, name):
    """Number of the device that a call runs on: its first tensor's."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    return t.get_device()


def _pages(t, name):
    """Pages of a pool."""
    if not isinstance(t, torch.Tensor) or t.dim() == 0:
        raise ValueError(f"{name} must be a GPU tensor")
    return t.shape[0]


def _int(x, name):
    """A whole number that the C call takes as an int (ctypes would drop its higher bits)."""
    x = operator.index(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name}={x} does not fit in 32 bits")
    return x


def _run(fn, dev, *args):
    """The C call on device dev (made current for it) and that device's current stream."""
    if dev == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        _check(rc)


def hils_window_pieces(window: int) -> int:
    """Chunks that a window of this many tokens reaches into, at most: the window entries of ``weights``."""
    return (window + 62) // 64 + 1


def hils_q8_append(p: Params, k_new, v_new, k_pages, v_pages, kv_scale, block_table, seqlens=None, newlens=None):
    """Write new tokens into the 8-bit cache: sequence b's first newlens[b] rows of k_new, v_new
    [B, Hkv, N, d] go to its last newlens[b] positions (seqlens counts them).  Changes k_pages,
    v_pages and kv_scale in place and returns them."""
    dev, dt, B, H, d, S = _gpu(k_new, "k_new"), p.torch_dtype, p.B, p.Hkv, p.d, p.chunk
    new, n = (B, H, p.N, d), _pages(k_pages, "k_pages")
    _run(LIB.hils_q8_append, dev, ctypes.byref(p.c()), _address(k_new, "k_new", new, dt, dev),
         _address(v_new, "v_new", new, dt, dev), _address(k_pages, "k_pages", (n, H, S, d), _F8, dev),
         _address(v_pages, "v_pages", (n, H, d, S), _F8, dev), _address(kv_scale, "kv_scale", (n, H, 2), _F32, dev),
         _address(block_table, "block_table", (B, p.L // S), _I32, dev), n,
         None if seqlens is None else _address(seqlens, "seqlens", (B,), _I32, dev),
         None if newlens is None else _address(newlens, "newlens", (B,), _I32, dev))
    return k_pages, v_pages, kv_scale


def hils_q8_landmark_fwd(p: Params, lq, k_pages, kv_scale, block_table, lmk_pages, bias_pages, seqlens=None,
                         newlens=None):
    """Landmark rows and biases of the chunks that each sequence's last newlens[b] tokens completed, from
    the stored keys: lq [B, Hl, (N + S - 1) // S, d] (one query per completed chunk) or [Hl, d] under
    HILS_FLAG_SHARED_LMK_QUERY.  Changes lmk_pages and bias_pages in place and returns them."""
    dev, B, H, Hl, d, S = _gpu(lq, "lq"), p.B, p.Hkv, p.Hl or p.Hq, p.d, p.chunk
    n, lqs = _pages(k_pages, "k_pages"), (Hl, d) if p.flags & HILS_FLAG_SHARED_LMK_QUERY else (B, Hl, (p.N + S - 1) // S, d)
    _run(LIB.hils_q8_landmark_fwd, dev, ctypes.byref(p.c()), _address(lq, "lq", lqs, p.torch_dtype, dev),
         _address(k_pages, "k_pages", (n, H, S, d), _F8, dev), _address(kv_scale, "kv_scale", (n, H, 2), _F32, dev),
         _address(block_table, "block_table", (B, p.L // S), _I32, dev), n,
         None if seqlens is None else _address(seqlens, "seqlens", (B,), _I32, dev),
         None if newlens is None else _address(newlens, "newlens", (B,), _I32, dev),
         _address(lmk_pages, "lmk_pages", (n, Hl, d), _F8, dev), _address(bias_pages, "bias_pages", (n, Hl), _F32, dev))
    return lmk_pages, bias_pages


def hils_decode_q8_fwd(p: Params, q, k_pages, v_pages, kv_scale, lmk_pages, block_table, bias_pages=None, q_route=None,
                       seqlens=None, out=None, lse=None, idx=None, weights=None, want_weights=True, workspace=None):
    """Decode forward over the 8-bit cache, N >= 1 new queries per sequence.  Returns (out, lse, idx, weights);
    weights [B, Hkv, N, K + hils_window_pieces(W)] float32 (None without want_weights): each selected chunk's
    and window piece's attention weight, summed over the group's heads."""
    dev, dt, B, Hq, H, N, d, S = _gpu(q, "q"), p.torch_dtype, p.B, p.Hq, p.Hkv, p.N, p.d, p.chunk
    n, Hl, qs, K = _pages(k_pages, "k_pages"), p.Hl or p.Hq, (B, Hq, N, d), p.topk
    on = q.device
    if out is None:
        out = torch.empty(qs, dtype=dt, device=on)
    if lse is None:
        lse = torch.empty((B, Hq, N), dtype=_F32, device=on)
    if idx is None:
        if p.flags & HILS_FLAG_GIVEN_IDX:
            raise ValueError("HILS_FLAG_GIVEN_IDX needs idx")
        idx = torch.empty((B, H, N, K), dtype=_I32, device=on)
    wshape = (B, H, N, K + hils_window_pieces(p.window))
    if weights is None and want_weights:
        weights = torch.empty(wshape, dtype=_F32, device=on)
    if workspace is None:
        workspace = torch.empty(max(1, hils_workspace_size(p, HILS_OP_DECODE_Q8)), dtype=torch.uint8, device=on)
    nbytes = workspace.numel() if isinstance(workspace, torch.Tensor) else 0  # the library says if that is too little
    _run(LIB.hils_decode_q8_fwd, dev, ctypes.byref(p.c()), _address(q, "q", qs, dt, dev),
         _address(k_pages, "k_pages", (n, H, S, d), _F8, dev), _address(v_pages, "v_pages", (n, H, d, S), _F8, dev),
         _address(kv_scale, "kv_scale", (n, H, 2), _F32, dev), _address(lmk_pages, "lmk_pages", (n, Hl, d), _F8, dev),
         None if bias_pages is None else _address(bias_pages, "bias_pages", (n, Hl), _F32, dev),
         None if q_route is None else _address(q_route, "q_route", qs, dt, dev),
         _address(block_table, "block_table", (B, p.L // S), _I32, dev), n,
         None if seqlens is None else _address(seqlens, "seqlens", (B,), _I32, dev), _address(out, "out", qs, dt, dev),
         _address(lse, "lse", (B, Hq, N), _F32, dev), _address(idx, "idx", (B, H, N, K), _I32, dev),
         None if weights is None else _address(weights, "weights", wshape, _F32, dev),
         _address(workspace, "workspace", (nbytes,), torch.uint8, dev), nbytes)
    return out, lse, idx, weights


def hils_cache_evict(p: Params, acc, block_table, seqlens=None, budget=0, sink=0, max_evict=None, weights=None,
                     idx=None, acc_out=None, table_out=None, seqlens_out=None, freed=None, nfreed=None):
    """Add a decode call's weights (and idx) to the chunks' totals acc [B, L/S], then cut every sequence to
    ``budget`` candidate chunks by dropping those with the least totals, never the first ``sink``, at most
    max_evict (None: any number).  Returns (acc, block_table, seqlens, freed, nfreed), new tensors unless
    outputs are given (the inputs themselves for a call in place); the pages given up by sequence b are
    freed[b, :nfreed[b]]."""
    if weights is not None and idx is None:
        raise ValueError("weights needs idx")
    budget, sink, nc = _int(budget, "budget"), _int(sink, "sink"), p.L // p.chunk
    most = nc if max_evict is None else _int(max_evict, "max_evict")
    dev, B, on = _gpu(acc, "acc"), p.B, acc.device
    if acc_out is None:
        acc_out = torch.empty((B, nc), dtype=_F32, device=on)
    if table_out is None:
        table_out = torch.empty((B, nc), dtype=_I32, device=on)
    if seqlens_out is None:
        seqlens_out = torch.empty(B, dtype=_I32, device=on)
    if freed is None:
        freed = torch.empty((B, most), dtype=_I32, device=on)
    if nfreed is None:
        nfreed = torch.empty(B, dtype=_I32, device=on)
    _run(LIB.hils_cache_evict, dev, ctypes.byref(p.c()), _address(acc, "acc", (B, nc), _F32, dev),
         _address(block_table, "block_table", (B, nc), _I32, dev),
         None if seqlens is None else _address(seqlens, "seqlens", (B,), _I32, dev),
         None if weights is None else
         _address(weights, "weights", (B, p.Hkv, p.N, p.topk + hils_window_pieces(p.window)), _F32, dev),
         None if weights is None else _address(idx, "idx", (B, p.Hkv, p.N, p.topk), _I32, dev), budget, sink, most,
         _address(acc_out, "acc_out", (B, nc), _F32, dev), _address(table_out, "table_out", (B, nc), _I32, dev),
         _address(seqlens_out, "seqlens_out", (B,), _I32, dev), _address(freed, "freed", (B, most), _I32, dev),
         _address(nfreed, "nfreed", (B,), _I32, dev))
    return acc_out, table_out, seqlens_out, freed, nfreed


def hils_prefill_paged_fwd(p: Params, q, k_pages, v_pages, lmk_pages, block_table, bias_pages=None, q_route=None,
                           seqlens=None, newlens=None, out=None, lse=None, idx=None, workspace=None):
    """Attention of a chunk of new tokens over paged pools (as hils_decode_paged_fwd's): row n < newlens[b] of
    q [B, Hq, N, d] is the query at position seqlens[b] - newlens[b] + n; other rows are neither read nor
    written.  Returns (out, lse, idx)."""
    dev, dt, B, Hq, H, N, d, S = _gpu(q, "q"), p.torch_dtype, p.B, p.Hq, p.Hkv, p.N, p.d, p.chunk
    n, Hl, qs, K = _pages(k_pages, "k_pages"), p.Hl or p.Hq, (B, Hq, N, d), p.topk
    on = q.device
    if out is None:
        out = torch.empty(qs, dtype=dt, device=on)
    if lse is None:
        lse = torch.empty((B, Hq, N), dtype=_F32, device=on)
    if idx is None:
        if p.flags & HILS_FLAG_GIVEN_IDX:
            raise ValueError("HILS_FLAG_GIVEN_IDX needs idx")
        idx = torch.empty((B, H, N, K), dtype=_I32, device=on)
    if workspace is None:
        workspace = torch.empty(max(1, hils_workspace_size(p, HILS_OP_PREFILL_PAGED)), dtype=torch.uint8, device=on)
    nbytes = workspace.numel() if isinstance(workspace, torch.Tensor) else 0  # the library says if that is too little
    _run(LIB.hils_prefill_paged_fwd, dev, ctypes.byref(p.c()), _address(q, "q", qs, dt, dev),
         _address(k_pages, "k_pages", (n, H, S, d), dt, dev), _address(v_pages, "v_pages", (n, H, S, d), dt, dev),
         _address(lmk_pages, "lmk_pages", (n, Hl, d), dt, dev),
         None if bias_pages is None else _address(bias_pages, "bias_pages", (n, Hl), _F32, dev),
         None if q_route is None else _address(q_route, "q_route", qs, dt, dev),
         _address(block_table, "block_table", (B, p.L // S), _I32, dev), n,
         None if seqlens is None else _address(seqlens, "seqlens", (B,), _I32, dev),
         None if newlens is None else _address(newlens, "newlens", (B,), _I32, dev), _address(out, "out", qs, dt, dev),
         _address(lse, "lse", (B, Hq, N), _F32, dev), _address(idx, "idx", (B, H, N, K), _I32, dev),
         _address(workspace, "workspace", (nbytes,), torch.uint8, dev), nbytes)
    return out, lse, idx


# ---- the pages of a cache as a resource: block_table [B, L/S], seqlens [B] and page_refs [P] (how many table
# entries name a page; 0: free) are int32; pools are the tensors that the table indexes, [P, ...] of any type.


def _pool_list(pools, P, dev):
    """The pools as an array of hils_pool (an address and a page's bytes each), and how many they are."""
    flat = []
    for i, t in enumerate(pools):
        try:
            ok = t.get_device() == dev and t.shape[0] == P and t.is_contiguous()
        except (AttributeError, IndexError):
            ok = False
        if not ok:
            _gpu(t, f"pools[{i}]")
            raise ValueError(f"pools[{i}] must be a contiguous tensor of {P} pages on cuda:{dev}")
        flat.append(t.data_ptr())
        flat.append(t.nbytes // P)
    return (ctypes.c_size_t * len(flat))(*flat), len(flat) // 2


def _refs(page_refs):
    dev = _gpu(page_refs, "page_refs")
    if page_refs.dim() != 1 or not len(page_refs):
        raise ValueError(f"page_refs has shape {tuple(page_refs.shape)}, expected one dimension of at least one page")
    return dev, page_refs.shape[0]


def hils_cache_reserve(p: Params, block_table, page_refs, pools=(), seqlens=None, newlens=None, table_out=None,
                       refs_out=None, copied=None, counts=None):
    """Give every sequence pages for its last newlens[b] tokens (which seqlens counts), before they are written: a
    free page for each chunk that begins, a copy (in all ``pools``) of a begun page that others have too.
    Returns (block_table, page_refs, copied [B, 2], counts [2]); counts = (pages needed, free pages found), and
    nothing has been done unless both are equal.  In place if the outputs are the inputs."""
    dev, P = _refs(page_refs)
    shape, on = (p.B, p.L // p.chunk), page_refs.device
    if table_out is None:
        table_out = torch.empty(shape, dtype=_I32, device=on)
    if refs_out is None:
        refs_out = torch.empty(P, dtype=_I32, device=on)
    if copied is None:
        copied = torch.empty((p.B, 2), dtype=_I32, device=on)
    if counts is None:
        counts = torch.empty(2, dtype=_I32, device=on)
    arr, n = _pool_list(pools, P, dev)
    _run(LIB.hils_cache_reserve, dev, ctypes.byref(p.c()), _address(block_table, "block_table", shape, _I32, dev),
         _address(page_refs, "page_refs", (P,), _I32, dev), P,
         None if seqlens is None else _address(seqlens, "seqlens", (p.B,), _I32, dev),
         None if newlens is None else _address(newlens, "newlens", (p.B,), _I32, dev), arr, n,
         _address(table_out, "table_out", shape, _I32, dev), _address(refs_out, "refs_out", (P,), _I32, dev),
         _address(copied, "copied", (p.B, 2), _I32, dev), _address(counts, "counts", (2,), _I32, dev))
    return table_out, refs_out, copied, counts


def hils_cache_fork(p: Params, parent, block_table, page_refs, seqlens=None, table_out=None, seqlens_out=None,
                    refs_out=None):
    """Rows that go on from rows ``parent`` [rows] int32 (outside [0, B): empty rows): they share their pages.  Rows
    of the input that nobody goes on from are freed.  Returns (block_table [rows, L/S], seqlens [rows], page_refs);
    only the last may be written in place."""
    dev, P = _refs(page_refs)
    if not isinstance(parent, torch.Tensor) or parent.dim() != 1:
        raise ValueError("parent must be a GPU tensor of one dimension")
    rows, C, on = parent.shape[0], p.L // p.chunk, page_refs.device
    if table_out is None:
        table_out = torch.empty((rows, C), dtype=_I32, device=on)
    if seqlens_out is None:
        seqlens_out = torch.empty(rows, dtype=_I32, device=on)
    if refs_out is None:
        refs_out = torch.empty(P, dtype=_I32, device=on)
    _run(LIB.hils_cache_fork, dev, ctypes.byref(p.c()), _address(parent, "parent", (rows,), _I32, dev), rows,
         _address(block_table, "block_table", (p.B, C), _I32, dev), _address(page_refs, "page_refs", (P,), _I32, dev), P,
         None if seqlens is None else _address(seqlens, "seqlens", (p.B,), _I32, dev),
         _address(table_out, "table_out", (rows, C), _I32, dev), _address(seqlens_out, "seqlens_out", (rows,), _I32, dev),
         _address(refs_out, "refs_out", (P,), _I32, dev))
    return table_out, seqlens_out, refs_out


def hils_cache_free(p: Params, keep, block_table, page_refs, seqlens=None, pages=None, npages=None, table_out=None,
                    seqlens_out=None, refs_out=None):
    """Cut every sequence to its first keep[b] tokens and give up the pages past them, and those that ``pages``
    [B, M] with ``npages`` [B] list (``freed`` and ``nfreed`` of hils_cache_evict).  Returns (block_table, seqlens,
    page_refs); in place if the outputs are the inputs."""
    dev, P = _refs(page_refs)
    shape, on = (p.B, p.L // p.chunk), page_refs.device
    if pages is not None and (not isinstance(pages, torch.Tensor) or pages.dim() != 2):
        raise ValueError("pages must be a GPU tensor of two dimensions")
    most = 0 if pages is None else pages.shape[1]
    nlisted = None if npages is None else _address(npages, "npages", (p.B,), _I32, dev)
    if pages is not None and not most:  # lists of no entries have no address, so their counts are left out too
        nlisted = None
    if table_out is None:
        table_out = torch.empty(shape, dtype=_I32, device=on)
    if seqlens_out is None:
        seqlens_out = torch.empty(p.B, dtype=_I32, device=on)
    if refs_out is None:
        refs_out = torch.empty(P, dtype=_I32, device=on)
    _run(LIB.hils_cache_free, dev, ctypes.byref(p.c()), _address(keep, "keep", (p.B,), _I32, dev),
         None if pages is None else _address(pages, "pages", (p.B, most), _I32, dev), nlisted, most,
         _address(block_table, "block_table", shape, _I32, dev), _address(page_refs, "page_refs", (P,), _I32, dev), P,
         None if seqlens is None else _address(seqlens, "seqlens", (p.B,), _I32, dev),
         _address(table_out, "table_out", shape, _I32, dev), _address(seqlens_out, "seqlens_out", (p.B,), _I32, dev),
         _address(refs_out, "refs_out", (P,), _I32, dev))
    return table_out, seqlens_out, refs_out


def hils_cache_compact(p: Params, block_table, page_refs, pools=(), seqlens=None, table_out=None, refs_out=None,
                       new_page=None, moved=None, counts=None):
    """Move the used pages of all ``pools`` to the front, into the lowest free ones.  Returns (block_table, page_refs,
    new_page [P], moved [P], counts [2]): new_page[i] is where page i is now (-1: it was free), ``moved`` lists the
    pages that moved, counts = (pages in use, pages moved).  In place if the outputs are the inputs."""
    dev, P = _refs(page_refs)
    shape, on = (p.B, p.L // p.chunk), page_refs.device
    if table_out is None:
        table_out = torch.empty(shape, dtype=_I32, device=on)
    if refs_out is None:
        refs_out = torch.empty(P, dtype=_I32, device=on)
    if new_page is None:
        new_page = torch.empty(P, dtype=_I32, device=on)
    if moved is None:
        moved = torch.empty(P, dtype=_I32, device=on)
    if counts is None:
        counts = torch.empty(2, dtype=_I32, device=on)
    arr, n = _pool_list(pools, P, dev)
    _run(LIB.hils_cache_compact, dev, ctypes.byref(p.c()), _address(block_table, "block_table", shape, _I32, dev),
         _address(page_refs, "page_refs", (P,), _I32, dev), P,
         None if seqlens is None else _address(seqlens, "seqlens", (p.B,), _I32, dev), arr, n,
         _address(table_out, "table_out", shape, _I32, dev), _address(refs_out, "refs_out", (P,), _I32, dev),
         _address(new_page, "new_page", (P,), _I32, dev), _address(moved, "moved", (P,), _I32, dev),
         _address(counts, "counts", (2,), _I32, dev))
    return table_out, refs_out, new_page, moved, counts


def hils_timing_enable(on: bool = True) -> None:
    """Bracket every library kernel launch of this thread with HIP events."""
    _check(LIB.hils_timing_enable(int(bool(on))))


def hils_timing_read(max_kernels: int = 64) -> dict:
    """Per kernel name: {"launches": n, "total_ms": t} for the launches recorded
    since timing was enabled (or last read); clears the records."""
    names = ctypes.create_string_buffer(4096)
    ms = (ctypes.c_float * max_kernels)()
    cnt = (ctypes.c_int * max_kernels)()
    nk = ctypes.c_int(0)
    _check(LIB.hils_timing_read(names, 4096, ms, cnt, max_kernels, ctypes.byref(nk)))
    keys = [k for k in names.value.decode().split("\n") if k]
    return {k: {"launches": cnt[i], "total_ms": ms[i]} for i, k in enumerate(keys[: nk.value])}
