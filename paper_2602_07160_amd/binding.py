"""Python binding of libfem.so (argument marshalling only).

Each function has the name of the C entry point it calls (``include/fem.h``)
and takes torch tensors for the device buffers: torch provides device memory
and the stream, every step of the read runs in the library's HIP kernels.
There is no fallback: if libfem.so is missing or a call fails, an exception
is raised.
"""

from __future__ import annotations

import contextlib
import ctypes
import os

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfem.so")

FEM_DTYPE = {torch.float32: 0, torch.bfloat16: 1}

EXPORTS = ("fem_softmax_fwd", "fem_softmax_fwd_ex", "fem_softmax_fwd_train", "fem_softmax_bwd",
           "fem_softmax_bwd_workspace_bytes", "fem_softmax_gated_fwd", "fem_softmax_decode",
           "fem_softmax_decode_workspace_bytes", "fem_softmax_decode_noalloc", "fem_linear_fwd", "fem_linear_workspace_bytes",
           "fem_gla_fwd", "fem_gla_workspace_bytes", "fem_cache_append", "fem_cache_gather",
           "fem_paged_workspace_bytes", "fem_paged_fwd", "fem_status_str")

FEM_FLAG_ENCODER = 1
FEM_FLAG_OUT_BF16 = 2

# fem_kv_type of a pool's element type
FEM_KV = {torch.bfloat16: 0, torch.float8_e4m3fn: 1, torch.int8: 2}


class _Cache(ctypes.Structure):  # fem_paged_cache
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p)] + [
                    (n, ctypes.c_int) for n in ("pages", "page", "heads", "d_qk", "d_v", "type")]


class _Batch(ctypes.Structure):  # fem_paged_batch
    _fields_ = [("q_start", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("table", ctypes.c_void_p)] + [
                    (n, ctypes.c_int) for n in ("n_seq", "table_len", "n_tok", "max_q")]

_lib = None


class FemError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


def load() -> ctypes.CDLL:
    """Load libfem.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2602_07160_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
        lib.fem_softmax_fwd.argtypes = [vp, vp, vp, f, f, i, i, i, i, i, vp]
        lib.fem_softmax_fwd.restype = i
        lib.fem_softmax_fwd_ex.argtypes = [vp, vp, vp, f, vp, i, i, i, i, i, i, i, vp]
        lib.fem_softmax_fwd_ex.restype = i
        lib.fem_softmax_decode.argtypes = [vp, vp, vp, vp, f, f, i, i, i, i, i, i, vp, sz, vp]
        lib.fem_softmax_decode.restype = i
        lib.fem_softmax_decode_workspace_bytes.argtypes = [i, i, i, i, i]
        lib.fem_softmax_decode_workspace_bytes.restype = sz
        lib.fem_softmax_decode_noalloc.argtypes = [vp, vp, vp, vp, f, f, i, i, i, i, i, i, vp]
        lib.fem_softmax_decode_noalloc.restype = i
        lib.fem_softmax_gated_fwd.argtypes = [vp, vp, vp, f, f, f, f, i, i, i, i, i, vp]
        lib.fem_softmax_gated_fwd.restype = i
        lib.fem_linear_fwd.argtypes = [vp, vp, vp, f, f, i, i, i, i, i, i, i, vp, sz, vp]
        lib.fem_linear_fwd.restype = i
        lib.fem_linear_workspace_bytes.argtypes = [i, i, i, i, i, i]
        lib.fem_linear_workspace_bytes.restype = sz
        lib.fem_gla_fwd.argtypes = [vp, vp, vp, f, f, f, i, i, i, i, i, i, i, vp, sz, vp]
        lib.fem_gla_fwd.restype = i
        lib.fem_gla_workspace_bytes.argtypes = [i, i, i, i, i, i]
        lib.fem_gla_workspace_bytes.restype = sz
        lib.fem_softmax_fwd_train.argtypes = [vp, vp, vp, f, f, f, i, i, i, i, i, vp]
        lib.fem_softmax_fwd_train.restype = i
        lib.fem_softmax_bwd.argtypes = [vp, vp, vp, f, f, f, f, f, f, f, f, i, i, i, i, i, vp, sz,
                                        vp]
        lib.fem_softmax_bwd.restype = i
        lib.fem_softmax_bwd_workspace_bytes.argtypes = [i, i, i, i]
        lib.fem_softmax_bwd_workspace_bytes.restype = sz
        cp, bp, ll = ctypes.POINTER(_Cache), ctypes.POINTER(_Batch), ctypes.c_longlong
        lib.fem_cache_append.argtypes = [cp, bp, vp, ll, vp, ll, vp]
        lib.fem_cache_append.restype = i
        lib.fem_cache_gather.argtypes = [cp, bp, vp, vp, i, vp]
        lib.fem_cache_gather.restype = i
        lib.fem_paged_workspace_bytes.argtypes = [cp, bp, i]
        lib.fem_paged_workspace_bytes.restype = sz
        lib.fem_paged_fwd.argtypes = [cp, bp, vp, ll, f, vp, i, i, vp, sz, vp]
        lib.fem_paged_fwd.restype = i
        lib.fem_status_str.argtypes = [i]
        lib.fem_status_str.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def fem_status_str(status: int) -> str:
    return load().fem_status_str(int(status)).decode()


def _check(rc: int):
    if rc != 0:
        raise FemError(rc, fem_status_str(rc))


def _dev_tensor(x: torch.Tensor, name: str, dtype=None) -> torch.Tensor:
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    return x


def _workspace(nbytes: int, device, ws, stream):
    """(tensor, pointer, size) of the workspace for a call that needs
    ``nbytes``: the caller's uint8 GPU tensor ``ws`` if given, else a new one
    from torch's allocator (its blocks are 512-byte aligned), allocated on the
    stream the call runs on so that torch does not hand the memory out again
    before the call's kernels have run.  (None, None, 0) when nothing is
    needed."""
    if ws is not None:
        _dev_tensor(ws, "ws", torch.uint8)
        return ws, ws.data_ptr(), ws.numel()
    if nbytes == 0:
        return None, None, 0
    s = torch.cuda.current_stream(device) if stream is None else stream
    if not isinstance(s, torch.cuda.Stream):
        s = torch.cuda.ExternalStream(int(s), device=device)
    with torch.cuda.stream(s):
        t = torch.empty(nbytes, device=device, dtype=torch.uint8)
    return t, t.data_ptr(), nbytes


# The current stream's handle without building a torch.cuda.Stream (1.9 us of a
# ~10 us call), where this torch has the accessor that its own generated code uses.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_HERE = contextlib.nullcontext()


def _stream_handle(device, stream) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(device.index)
    s = torch.cuda.current_stream(device) if stream is None else stream
    return s.cuda_stream if isinstance(s, torch.cuda.Stream) else int(s)


def _on(device):
    """Context in which ``device`` is current (nothing to do where it already is:
    entering and leaving torch.cuda.device costs 1.4 us)."""
    return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def fem_softmax_fwd(q, k, v, beta, out=None, stream=None) -> torch.Tensor:
    """Causal softmax-prior FEM read.  q, k, v: [B, H, T, d] bf16 or fp32;
    beta: [H, d] fp32.  Returns out [B, H, T, d] fp32 (enqueued on ``stream``,
    default torch's current stream)."""
    lib = load()
    if q.dtype not in FEM_DTYPE:
        raise ValueError(f"unsupported dtype {q.dtype}")
    for name, x in (("q", q), ("k", k), ("v", v)):
        _dev_tensor(x, name, q.dtype)
        if x.dim() != 4 or x.shape != q.shape:
            raise ValueError(f"{name} must be [B, H, T, d] like q")
    B, H, T, d = q.shape
    _dev_tensor(beta, "beta", torch.float32)
    if tuple(beta.shape) != (H, d):
        raise ValueError("beta must be [H, d]")
    if out is None:
        out = torch.empty((B, H, T, d), device=q.device, dtype=torch.float32)
    _dev_tensor(out, "out", torch.float32)
    if tuple(out.shape) != (B, H, T, d):
        raise ValueError("out must be [B, H, T, d]")
    with _on(q.device):
        rc = lib.fem_softmax_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
                                 out.data_ptr(), B, H, T, d, FEM_DTYPE[q.dtype],
                                 _stream_handle(q.device, stream))
    _check(rc)
    return out


def fem_softmax_fwd_ex(q, k, v, beta, out=None, causal: bool = True, out_dtype=torch.float32,
                       stream=None) -> torch.Tensor:
    """Variants of the softmax-prior read: causal or encoder (all keys),
    d_v = d_qk or d_qk / 2, fp32 or bf16 output.  q, k: [B, H, T, d_qk] bf16;
    v: [B, H, T, d_v] bf16; beta: [H, d_v] fp32.  Returns [B, H, T, d_v]."""
    lib = load()
    for name, x in (("q", q), ("k", k), ("v", v)):
        _dev_tensor(x, name, torch.bfloat16)
        if x.dim() != 4:
            raise ValueError(f"{name} must be [B, H, T, width]")
    if k.shape != q.shape or v.shape[:3] != q.shape[:3]:
        raise ValueError("q, k must be [B, H, T, d_qk] and v [B, H, T, d_v]")
    B, H, T, dqk = q.shape
    dv = v.shape[3]
    _dev_tensor(beta, "beta", torch.float32)
    if tuple(beta.shape) != (H, dv):
        raise ValueError("beta must be [H, d_v]")
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be float32 or bfloat16")
    if out is None:
        out = torch.empty((B, H, T, dv), device=q.device, dtype=out_dtype)
    _dev_tensor(out, "out", out_dtype)
    if tuple(out.shape) != (B, H, T, dv):
        raise ValueError("out must be [B, H, T, d_v]")
    flags = (0 if causal else FEM_FLAG_ENCODER) | \
        (FEM_FLAG_OUT_BF16 if out_dtype == torch.bfloat16 else 0)
    with _on(q.device):
        rc = lib.fem_softmax_fwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
                                    out.data_ptr(), B, H, T, dqk, dv, flags, FEM_DTYPE[q.dtype],
                                    _stream_handle(q.device, stream))
    _check(rc)
    return out


def _decode_args(q, k_cache, v_cache, beta, lens, out):
    _dev_tensor(q, "q", torch.bfloat16)
    _dev_tensor(k_cache, "k_cache", torch.bfloat16)
    _dev_tensor(v_cache, "v_cache", torch.bfloat16)
    if q.dim() != 3 or k_cache.dim() != 4 or v_cache.dim() != 4:
        raise ValueError("q must be [B, H, d_qk], caches [B, H, L, width]")
    B, H, dqk = q.shape
    L = k_cache.shape[2]
    if tuple(k_cache.shape) != (B, H, L, dqk) or v_cache.shape[:3] != k_cache.shape[:3]:
        raise ValueError("k_cache must be [B, H, L, d_qk] and v_cache [B, H, L, d_v]")
    dv = v_cache.shape[3]
    _dev_tensor(beta, "beta", torch.float32)
    if tuple(beta.shape) != (H, dv):
        raise ValueError("beta must be [H, d_v]")
    if lens is not None:
        _dev_tensor(lens, "lens", torch.int32)
        if tuple(lens.shape) != (B,):
            raise ValueError("lens must be [B]")
    if out is None:
        out = torch.empty((B, H, dv), device=q.device, dtype=torch.float32)
    _dev_tensor(out, "out", torch.float32)
    if tuple(out.shape) != (B, H, dv):
        raise ValueError("out must be [B, H, d_v]")
    return B, H, L, dqk, dv, out


def fem_softmax_decode_noalloc(q, k_cache, v_cache, beta, lens=None, out=None,
                               stream=None) -> torch.Tensor:
    """fem_softmax_decode without a workspace: the library keeps the partial
    results in a fixed 8 MiB array per device (for callers that cannot
    allocate; overlapping calls on one device race).  Same arguments and
    result as fem_softmax_decode."""
    lib = load()
    B, H, L, dqk, dv, out = _decode_args(q, k_cache, v_cache, beta, lens, out)
    with _on(q.device):
        rc = lib.fem_softmax_decode_noalloc(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                            None if lens is None else lens.data_ptr(),
                                            beta.data_ptr(), out.data_ptr(), B, H, L, dqk, dv,
                                            FEM_DTYPE[q.dtype], _stream_handle(q.device, stream))
    _check(rc)
    return out


def fem_softmax_decode(q, k_cache, v_cache, beta, lens=None, out=None, ws=None,
                       stream=None) -> torch.Tensor:
    """One decoding step: q [B, H, d_qk] reads the first lens[b] rows of the
    caches k_cache [B, H, L, d_qk], v_cache [B, H, L, d_v] (bf16).  lens: [B]
    int32 GPU tensor or None (all L).  ws: optional uint8 GPU workspace of at
    least fem_softmax_decode_workspace_bytes(...) bytes.  Returns [B, H, d_v]
    fp32."""
    lib = load()
    B, H, L, dqk, dv, out = _decode_args(q, k_cache, v_cache, beta, lens, out)
    need = 0 if ws is not None else lib.fem_softmax_decode_workspace_bytes(B, H, L, dqk, dv)
    with _on(q.device):
        wst, wsp, wsn = _workspace(need, q.device, ws, stream)
        rc = lib.fem_softmax_decode(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                    None if lens is None else lens.data_ptr(), beta.data_ptr(),
                                    out.data_ptr(), B, H, L, dqk, dv, FEM_DTYPE[q.dtype],
                                    wsp, wsn, _stream_handle(q.device, stream))
    _check(rc)
    return out


def fem_softmax_gated_fwd(q, k, v, beta_max, lam, gate=None, out=None, stream=None) -> torch.Tensor:
    """Two-level gated read g * ((1 - lam) * mu + lam * F(beta_max)) with the
    causal softmax prior.  q, k, v: [B, H, T, d] bf16; beta_max: [H, d] fp32;
    lam, gate: [B, H, T, d] fp32 (gate None means g = 1).  Returns
    [B, H, T, d] fp32."""
    lib = load()
    for name, x in (("q", q), ("k", k), ("v", v)):
        _dev_tensor(x, name, torch.bfloat16)
        if x.dim() != 4 or x.shape != q.shape:
            raise ValueError(f"{name} must be [B, H, T, d] like q")
    B, H, T, d = q.shape
    _dev_tensor(beta_max, "beta_max", torch.float32)
    if tuple(beta_max.shape) != (H, d):
        raise ValueError("beta_max must be [H, d]")
    for name, x in (("lam", lam), ("gate", gate)):
        if x is None and name == "gate":
            continue
        _dev_tensor(x, name, torch.float32)
        if tuple(x.shape) != (B, H, T, d):
            raise ValueError(f"{name} must be [B, H, T, d]")
    if out is None:
        out = torch.empty((B, H, T, d), device=q.device, dtype=torch.float32)
    _dev_tensor(out, "out", torch.float32)
    if tuple(out.shape) != (B, H, T, d):
        raise ValueError("out must be [B, H, T, d]")
    with _on(q.device):
        rc = lib.fem_softmax_gated_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                       beta_max.data_ptr(), lam.data_ptr(),
                                       None if gate is None else gate.data_ptr(),
                                       out.data_ptr(), B, H, T, d, FEM_DTYPE[q.dtype],
                                       _stream_handle(q.device, stream))
    _check(rc)
    return out


def fem_linear_fwd(q, k, v, beta, out=None, chunk: int = 64, ws=None,
                   stream=None) -> torch.Tensor:
    """Causal linear-prior (phi = elu + 1) FEM read.  q, k: [B, H, T, d_k];
    v: [B, H, T, d_v] bf16; beta: [H, d_v] fp32; ws: optional uint8 GPU
    workspace of at least fem_linear_workspace_bytes(...) bytes.  Returns
    [B, H, T, d_v] fp32."""
    lib = load()
    if q.dtype not in FEM_DTYPE:
        raise ValueError(f"unsupported dtype {q.dtype}")
    _dev_tensor(q, "q", q.dtype)
    _dev_tensor(k, "k", q.dtype)
    _dev_tensor(v, "v", q.dtype)
    if q.dim() != 4 or k.shape != q.shape or v.dim() != 4 or v.shape[:3] != q.shape[:3]:
        raise ValueError("q, k must be [B, H, T, d_k] and v [B, H, T, d_v]")
    B, H, T, dk = q.shape
    dv = v.shape[3]
    _dev_tensor(beta, "beta", torch.float32)
    if tuple(beta.shape) != (H, dv):
        raise ValueError("beta must be [H, d_v]")
    if out is None:
        out = torch.empty((B, H, T, dv), device=q.device, dtype=torch.float32)
    _dev_tensor(out, "out", torch.float32)
    if tuple(out.shape) != (B, H, T, dv):
        raise ValueError("out must be [B, H, T, d_v]")
    need = 0 if ws is not None else lib.fem_linear_workspace_bytes(B, H, T, dk, dv, int(chunk))
    with _on(q.device):
        wst, wsp, wsn = _workspace(need, q.device, ws, stream)
        rc = lib.fem_linear_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
                                out.data_ptr(), B, H, T, dk, dv, int(chunk),
                                FEM_DTYPE[q.dtype], wsp, wsn, _stream_handle(q.device, stream))
    _check(rc)
    return out


def fem_gla_fwd(q, k, v, g, beta, out=None, chunk: int = 64, ws=None,
                stream=None) -> torch.Tensor:
    """Causal GLA-prior FEM read.  q, k: [B, H, T, d_k] bf16; v: [B, H, T, d_v]
    bf16; g: [B, H, T, d_k] fp32 log-decays; beta: [H, d_v] fp32.  Returns
    [B, H, T, d_v] fp32."""
    lib = load()
    _dev_tensor(q, "q", torch.bfloat16)
    _dev_tensor(k, "k", torch.bfloat16)
    _dev_tensor(v, "v", torch.bfloat16)
    _dev_tensor(g, "g", torch.float32)
    if q.dim() != 4 or k.shape != q.shape or g.shape != q.shape or v.dim() != 4 or \
            v.shape[:3] != q.shape[:3]:
        raise ValueError("q, k, g must be [B, H, T, d_k] and v [B, H, T, d_v]")
    B, H, T, dk = q.shape
    dv = v.shape[3]
    _dev_tensor(beta, "beta", torch.float32)
    if tuple(beta.shape) != (H, dv):
        raise ValueError("beta must be [H, d_v]")
    if out is None:
        out = torch.empty((B, H, T, dv), device=q.device, dtype=torch.float32)
    _dev_tensor(out, "out", torch.float32)
    if tuple(out.shape) != (B, H, T, dv):
        raise ValueError("out must be [B, H, T, d_v]")
    need = 0 if ws is not None else lib.fem_gla_workspace_bytes(B, H, T, dk, dv, int(chunk))
    with _on(q.device):
        wst, wsp, wsn = _workspace(need, q.device, ws, stream)
        rc = lib.fem_gla_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(),
                             beta.data_ptr(), out.data_ptr(), B, H, T, dk, dv, int(chunk),
                             FEM_DTYPE[q.dtype], wsp, wsn, _stream_handle(q.device, stream))
    _check(rc)
    return out


def fem_softmax_fwd_train(q, k, v, beta, out=None, lse=None, stream=None):
    """fem_softmax_fwd (bf16) that also returns the prior's log-normaliser
    lse [B, H, T] fp32.  Returns (out, lse)."""
    lib = load()
    for name, x in (("q", q), ("k", k), ("v", v)):
        _dev_tensor(x, name, torch.bfloat16)
        if x.dim() != 4 or x.shape != q.shape:
            raise ValueError(f"{name} must be [B, H, T, d] like q")
    B, H, T, d = q.shape
    _dev_tensor(beta, "beta", torch.float32)
    if tuple(beta.shape) != (H, d):
        raise ValueError("beta must be [H, d]")
    out = torch.empty((B, H, T, d), device=q.device, dtype=torch.float32) if out is None else out
    lse = torch.empty((B, H, T), device=q.device, dtype=torch.float32) if lse is None else lse
    _dev_tensor(out, "out", torch.float32)
    _dev_tensor(lse, "lse", torch.float32)
    if tuple(out.shape) != (B, H, T, d) or tuple(lse.shape) != (B, H, T):
        raise ValueError("out must be [B, H, T, d] and lse [B, H, T]")
    with _on(q.device):
        rc = lib.fem_softmax_fwd_train(q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
                                       out.data_ptr(), lse.data_ptr(), B, H, T, d,
                                       FEM_DTYPE[q.dtype], _stream_handle(q.device, stream))
    _check(rc)
    return out, lse


def fem_softmax_bwd(q, k, v, beta, out, lse, dout, ws=None, stream=None):
    """Gradients of sum(dout * out) w.r.t. q, k, v (fp32, shaped like them) and
    beta ([H, d], summed over batch and time).  ws: optional uint8 GPU
    workspace of at least fem_softmax_bwd_workspace_bytes(...) bytes.  Returns
    (dq, dk, dv, dbeta)."""
    lib = load()
    for name, x in (("q", q), ("k", k), ("v", v)):
        _dev_tensor(x, name, torch.bfloat16)
        if x.dim() != 4 or x.shape != q.shape:
            raise ValueError(f"{name} must be [B, H, T, d] like q")
    B, H, T, d = q.shape
    _dev_tensor(beta, "beta", torch.float32)
    for name, x, shp in (("out", out, (B, H, T, d)), ("lse", lse, (B, H, T)),
                         ("dout", dout, (B, H, T, d))):
        _dev_tensor(x, name, torch.float32)
        if tuple(x.shape) != shp:
            raise ValueError(f"{name} must be {list(shp)}")
    if tuple(beta.shape) != (H, d):
        raise ValueError("beta must be [H, d]")
    dq = torch.empty((B, H, T, d), device=q.device, dtype=torch.float32)
    dk = torch.empty_like(dq)
    dv = torch.empty_like(dq)
    db = torch.empty((H, d), device=q.device, dtype=torch.float32)
    need = 0 if ws is not None else lib.fem_softmax_bwd_workspace_bytes(B, H, T, d)
    with _on(q.device):
        wst, wsp, wsn = _workspace(need, q.device, ws, stream)
        rc = lib.fem_softmax_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
                                 out.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(),
                                 dk.data_ptr(), dv.data_ptr(), db.data_ptr(), B, H, T, d,
                                 FEM_DTYPE[q.dtype], wsp, wsn, _stream_handle(q.device, stream))
    _check(rc)
    return dq, dk, dv, db


class PagedCache:
    """A paged key/value cache over the caller's pools: k [pages, heads, page,
    d_qk] and v [pages, heads, page, d_v], both bfloat16, or both
    torch.float8_e4m3fn or torch.int8 codes with their scale bytes k_scale, v_scale
    [.., width / 32] (uint8).  The pools stay the caller's; the object holds
    them and describes them to the library.  ``PagedCache.empty`` allocates them."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if not isinstance(k, torch.Tensor) or k.dtype not in FEM_KV:
            raise ValueError("the pools must be bfloat16, float8_e4m3fn or int8 tensors")
        for name, x in (("k", k), ("v", v)):
            _dev_tensor(x, name, k.dtype)
            if x.dim() != 4 or x.shape[:3] != k.shape[:3]:
                raise ValueError("k must be [pages, heads, page, d_qk] and v [pages, heads, page, d_v]")
        if k.dtype == torch.bfloat16:
            if k_scale is not None or v_scale is not None:
                raise ValueError("a bfloat16 cache has no scales")
        else:
            for name, x, pool in (("k_scale", k_scale, k), ("v_scale", v_scale, v)):
                _dev_tensor(x, name, torch.uint8)
                if tuple(x.shape) != (*pool.shape[:3], pool.shape[3] // 32):
                    raise ValueError(f"{name} must be [pages, heads, page, width / 32]")
        if any(x is not None and x.device != k.device for x in (v, k_scale, v_scale)):
            raise ValueError("the pools must be on one device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.index = k.device, k.get_device()
        pages, self.heads, page, self.d_qk = k.shape
        self.d_v = v.shape[3]
        self.c = _Cache(k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
                        None if v_scale is None else v_scale.data_ptr(), pages, page, self.heads,
                        self.d_qk, self.d_v, FEM_KV[k.dtype])
        self.ref = ctypes.byref(self.c)

    @classmethod
    def empty(cls, pages, heads, d_qk, d_v=None, page=64, dtype=torch.bfloat16, device="cuda"):
        """A cache with pools of its own (uninitialised)."""
        def pool(w, dt):
            return torch.empty((pages, heads, page, w), device=device, dtype=dt)

        d_v = d_qk if d_v is None else d_v
        scales = (None, None) if dtype == torch.bfloat16 else (pool(d_qk // 32, torch.uint8),
                                                               pool(d_v // 32, torch.uint8))
        return cls(pool(d_qk, dtype), pool(d_v, dtype), *scales)


class PagedBatch:
    """The sequences of a call: q_start [B + 1], lens [B] and table [B, table_len],
    int32 GPU tensors (read on the GPU at each call, so they may change in place
    between calls), the packed tensors' rows n_tok and the most new tokens of a
    sequence max_q (default n_tok).  See fem_paged_batch in fem.h."""

    def __init__(self, q_start, lens, table, n_tok=None, max_q=None):
        _dev_tensor(lens, "lens", torch.int32)
        _dev_tensor(table, "table", torch.int32)
        if lens.dim() != 1 or table.dim() != 2 or table.shape[0] != lens.shape[0]:
            raise ValueError("lens must be [B] and table [B, table_len]")
        if q_start is not None:
            _dev_tensor(q_start, "q_start", torch.int32)
            if tuple(q_start.shape) != (lens.shape[0] + 1,):
                raise ValueError("q_start must be [B + 1]")
        if any(x is not None and x.device != lens.device for x in (q_start, table)):
            raise ValueError("q_start, lens and table must be on one device")
        self.q_start, self.lens, self.table = q_start, lens, table
        self.device, self.index = lens.device, lens.get_device()
        self.n_seq = lens.shape[0]
        self.n_tok = 0 if n_tok is None else int(n_tok)
        self.c = _Batch(None if q_start is None else q_start.data_ptr(), lens.data_ptr(),
                        table.data_ptr(), lens.shape[0], table.shape[1], self.n_tok,
                        self.n_tok if max_q is None else min(int(max_q), self.n_tok))
        self.ref = ctypes.byref(self.c)


def _paged(cache, batch):
    if type(cache) is not PagedCache or type(batch) is not PagedBatch:
        raise ValueError("cache must be a PagedCache and batch a PagedBatch")
    if cache.index != batch.index:
        raise ValueError("cache and batch must be on one device")


def _packed(x, name, n_tok, heads, width, index):
    """Row stride of a packed [n_tok, heads, width] bf16 tensor whose tokens may
    lie apart (a slice of one projection's output)."""
    if not isinstance(x, torch.Tensor) or x.get_device() != index:
        raise ValueError(f"{name} must be a GPU tensor on the cache's device")
    if x.dtype != torch.bfloat16:
        raise ValueError(f"{name} must be bfloat16, got {x.dtype}")
    shape = x.shape
    if len(shape) != 3 or shape[0] != n_tok or shape[2] != width or \
            (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [n_tok, heads, width] of the batch and the cache")
    s0, s1, s2 = x.stride()
    if s2 != 1 or (s1 != width and shape[1] > 1):
        raise ValueError(f"a token's heads must be contiguous in {name}")
    return s0 if n_tok > 1 else shape[1] * width


def fem_cache_append(cache, batch, k, v, stream=None) -> None:
    """Store the batch's new keys k [n_tok, heads, d_qk] and values v [n_tok,
    heads, d_v] (bf16; tokens may be strided) in the cache, quantised if its pools
    are."""
    lib = load()
    _paged(cache, batch)
    kld = _packed(k, "k", batch.n_tok, cache.heads, cache.d_qk, cache.index)
    vld = _packed(v, "v", batch.n_tok, cache.heads, cache.d_v, cache.index)
    with _on(cache.device):
        rc = lib.fem_cache_append(cache.ref, batch.ref, k.data_ptr(), kld, v.data_ptr(), vld,
                                  _stream_handle(cache.device, stream))
    _check(rc)


def _gathered(x, name, B, H, L, w, cache, stream):
    """The caller's buffer of a read-back, or a new one of zeros made on its stream."""
    if x is None:
        s = torch.cuda.current_stream(cache.device) if stream is None else stream
        if not isinstance(s, torch.cuda.Stream):
            s = torch.cuda.ExternalStream(int(s), device=cache.device)
        with torch.cuda.stream(s):
            return torch.zeros((B, H, L, w), device=cache.device, dtype=torch.bfloat16)
    _dev_tensor(x, name, torch.bfloat16)
    if x.shape != (B, H, L, w) or x.get_device() != cache.index:
        raise ValueError(f"{name} must be [B, heads, L, width] on the cache's device")
    return x


def fem_cache_gather(cache, batch, k=None, v=None, L=None, stream=None):
    """The sequences' cached rows as k [B, heads, L, d_qk] and v [B, heads, L, d_v]
    bf16, the dense reads' layout; rows at or past a sequence's length are left as
    they were.  Buffers that are not given are allocated with zeros (L: by default
    the table's length in tokens).  Returns (k, v)."""
    lib = load()
    _paged(cache, batch)
    B, H = batch.n_seq, cache.heads
    if L is None:
        given = k if k is not None else v
        if given is None:
            L = batch.c.table_len * cache.c.page
        elif not isinstance(given, torch.Tensor) or given.dim() != 4:
            raise ValueError("k and v must be [B, heads, L, width]")
        else:
            L = given.shape[2]
    k = _gathered(k, "k", B, H, L, cache.d_qk, cache, stream)
    v = _gathered(v, "v", B, H, L, cache.d_v, cache, stream)
    with _on(cache.device):
        rc = lib.fem_cache_gather(cache.ref, batch.ref, k.data_ptr(), v.data_ptr(), L,
                                  _stream_handle(cache.device, stream))
    _check(rc)
    return k, v


def fem_paged_workspace_bytes(cache, batch, H) -> int:
    """Exact workspace size (bytes) of fem_paged_fwd with H query heads."""
    _paged(cache, batch)
    return int(load().fem_paged_workspace_bytes(cache.ref, batch.ref, int(H)))


def fem_paged_fwd(cache, batch, q, beta, causal: bool = True, out=None, out_dtype=torch.float32,
                  ws=None, stream=None) -> torch.Tensor:
    """The read of the batch's new tokens q [n_tok, H, d_qk] (bf16; tokens may be
    strided) over the cache: every token the keys up to its own position, or with
    causal=False all of its sequence's.  beta: [heads, d_v] fp32.  H / heads query
    heads share a cached head.  ws: optional uint8 GPU workspace of at least
    fem_paged_workspace_bytes(...) bytes.  Returns [n_tok, H, d_v], fp32 or bf16
    (out's type, or out_dtype)."""
    lib = load()
    _paged(cache, batch)
    qld = _packed(q, "q", batch.n_tok, None, cache.d_qk, cache.index)
    H = q.shape[1]
    _dev_tensor(beta, "beta", torch.float32)
    if beta.shape != (cache.heads, cache.d_v) or beta.get_device() != cache.index:
        raise ValueError("beta must be [heads, d_v] on the cache's device")
    if out is not None:
        out_dtype = out.dtype
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be float32 or bfloat16")
    if out is None:
        out = torch.empty((batch.n_tok, H, cache.d_v), device=cache.device, dtype=out_dtype)
    _dev_tensor(out, "out", out_dtype)
    if out.shape != (batch.n_tok, H, cache.d_v) or out.get_device() != cache.index:
        raise ValueError("out must be [n_tok, H, d_v] on the cache's device")
    flags = (0 if causal else FEM_FLAG_ENCODER) | \
        (FEM_FLAG_OUT_BF16 if out_dtype == torch.bfloat16 else 0)
    need = 0 if ws is not None else lib.fem_paged_workspace_bytes(cache.ref, batch.ref, H)
    with _on(cache.device):
        wst, wsp, wsn = _workspace(need, cache.device, ws, stream)
        rc = lib.fem_paged_fwd(cache.ref, batch.ref, q.data_ptr(), qld, beta.data_ptr(),
                               out.data_ptr(), H, flags, wsp, wsn,
                               _stream_handle(cache.device, stream))
    _check(rc)
    return out


def workspace_bytes(entry: str, *sizes) -> int:
    """Exact workspace size (bytes) of the entry point ``entry`` ("linear",
    "gla", "decode" or "bwd") for the given size arguments, as in fem.h."""
    lib = load()
    fn = {"linear": lib.fem_linear_workspace_bytes, "gla": lib.fem_gla_workspace_bytes,
          "decode": lib.fem_softmax_decode_workspace_bytes,
          "bwd": lib.fem_softmax_bwd_workspace_bytes}[entry]
    return int(fn(*[int(x) for x in sizes]))
