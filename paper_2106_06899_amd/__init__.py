"""MI355X (gfx950) top-k attention -- Python binding of ``libtopk.so``.

Argument marshalling only: every step of the computation runs in the HIP kernels
of ``libtopk.so`` (built from ``csrc/`` by ``paper_2106_06899_amd.build``). There
is no CPU or PyTorch fallback; if the library is missing the calls raise.

* ``attn(q, k, v, topk, chunk, causal, scale)`` -> top-k attention (Eq. 4, softmax)
* ``ffn(x, w1, w2, topk, chunk)``               -> top-k feed-forward (Eq. 3 + Eq. 4, ReLU)
* ``qk_norm_rope(qkv, ...)``, ``rope(x, ...)``    -> heads for the attention calls: head norms and
  rotary positions; ``qk_norm_rope_append`` writes keys and values to a cache
* ``attn_prefix(q, prefix_k, prefix_v, k, v, lengths)`` -> attention of requests that share a prefix

Tensors live on the GPU (PyTorch provides device memory and the stream); the
work is enqueued on ``torch.cuda.current_stream()``. The workspace is a PyTorch
byte tensor registered with ``topk_set_workspace`` for the duration of the call,
so PyTorch's memory statistics include it.
"""
from __future__ import annotations

import ctypes
import math
import os

__all__ = ["attn", "attn_dense", "scan_ablation", "probe_mfma", "ffn", "attn_workspace_bytes", "ffn_workspace_bytes", "attn_path", "ffn_path",
           "mfma_layout", "lib", "TopkError", "LIB_PATH", "profile_begin", "profile_end", "STAGES",
           "attn_backward", "ffn_backward", "rope", "rope_frequencies", "rope_axes", "qk_norm_rope", "qk_norm_rope_append",
           "qk_norm_rope_backward", "attn_prefix", "attn_prefix_workspace_bytes", "set_backward_lists", "set_memory_budget", "last_fallback_rows"]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtopk.so")

TOPK_F32, TOPK_BF16 = 0, 1
MAX_SELECT_K = 2048  # largest k the select handles (k = Lk above it runs attn_dense)
TOPK_LISTS_AUTO, TOPK_LISTS_BUCKET, TOPK_LISTS_ATOMIC = 0, 1, 2
_STATUS = {0: "OK", -1: "TOPK_E_INVAL", -2: "TOPK_E_NULL", -3: "TOPK_E_ALIGN", -4: "TOPK_E_UNSUPPORTED",
           -5: "TOPK_E_NOMEM", -6: "TOPK_E_HIP"}

_lib = None


class _Rotation(ctypes.Structure):  # topk_rotation
    _fields_ = [("positions", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("pair_axis", ctypes.c_char_p),
                ("d_rot", ctypes.c_int64), ("axis_stride", ctypes.c_int64), ("batch_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("n_axes", ctypes.c_int), ("position_bytes", ctypes.c_int),
                ("adjacent", ctypes.c_int), ("inverse", ctypes.c_int)]


class _PrefixStrides(ctypes.Structure):  # topk_prefix_strides
    _fields_ = [(n, ctypes.c_int64) for n in ("prefix_k_head", "prefix_k_key", "prefix_v_head", "prefix_v_key", "k_batch",
                                              "k_head", "k_key", "v_batch", "v_head", "v_key")]


class TopkError(RuntimeError):
    """A non-OK status from libtopk; ``status`` holds the code."""

    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def lib() -> ctypes.CDLL:
    """Load ``libtopk.so`` (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2106_06899_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    i64, vp, i32, f32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    attn_args = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, i32, f32, i32, vp]
    ffn_args = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i32, vp]
    sigs = {
        "topk_attn": (attn_args, i32),
        "topk_attn_noalloc": (attn_args, i32),
        "topk_attn_dense": ([vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, f32, i32, vp], i32),
        "topk_noalloc_scratch_bytes": ([], ctypes.c_size_t),
        "topk_attn_debug": (attn_args + [vp, vp], i32),
        "topk_ffn": (ffn_args, i32),
        "topk_ffn_debug": (ffn_args + [vp, vp], i32),
        "topk_attn_with_cache": (attn_args + [vp, vp], i32),
        "topk_ffn_with_cache": (ffn_args + [vp, vp], i32),
        "topk_attn_workspace_bytes": ([i64] * 7 + [i32, i32], ctypes.c_size_t),
        "topk_ffn_workspace_bytes": ([i64] * 5 + [i32], ctypes.c_size_t),
        "topk_set_workspace": ([vp, ctypes.c_size_t], i32),
        "topk_last_error": ([], ctypes.c_char_p),
        "topk_last_fallback_rows": ([], i64),
        "topk_set_backward_lists": ([i32], i32),
        "topk_set_memory_budget": ([ctypes.c_size_t], i32),
        "topk_attn_backward": ([vp] * 9 + [i64] * 6 + [ctypes.c_float, i32, vp], i32),
        "topk_ffn_backward": ([vp] * 9 + [i64] * 4 + [i32, vp], i32),
        "topk_attn_backward_workspace_bytes": ([i64] * 6 + [i32], ctypes.c_size_t),
        "topk_ffn_backward_workspace_bytes": ([i64] * 4 + [i32], ctypes.c_size_t),
        "topk_attn_path": ([i64] * 7 + [i32, i32], i32),
        "topk_ffn_path": ([i64] * 5 + [i32], i32),
        "topk_rope": ([vp, vp] + [i64] * 7 + [ctypes.POINTER(_Rotation), i32, vp], i32),
        "topk_qk_norm_rope": ([vp] * 6 + [i64] * 7 + [i32, f32, ctypes.POINTER(_Rotation), i32, vp], i32),
        "topk_qk_norm_rope_append": ([vp] * 7 + [i64] * 14 + [i32, f32, ctypes.POINTER(_Rotation), i32, vp], i32),
        "topk_qk_norm_rope_backward": ([vp] * 9 + [i64] * 7 + [i32, f32, ctypes.POINTER(_Rotation), i32, vp], i32),
        "topk_qk_norm_rope_backward_workspace_bytes": ([i64] * 6 + [i32], ctypes.c_size_t),
        "topk_attn_prefix": ([vp] * 8 + [i64] * 7 + [ctypes.POINTER(_PrefixStrides), i32, f32, i32, vp], i32),
        "topk_attn_prefix_workspace_bytes": ([i64] * 7 + [i32], ctypes.c_size_t),
        "topk_selftest_mfma_layout": ([vp, vp, vp], i32),
        "topk_scan_ablation": ([vp, vp] + [i64] * 7 + [i32, vp], i32),
        "topk_probe_mfma": ([ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), vp], i32),
        "topk_profile_begin": ([], i32),
        "topk_profile_end": ([ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64), i32], i32),
    }
    for name, (args, res) in sigs.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    _lib = L
    return L


def _raise(rc: int):
    if rc != 0:
        raise TopkError(rc, lib().topk_last_error().decode())


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return TOPK_F32
    if t.dtype == torch.bfloat16:
        return TOPK_BF16
    raise TypeError(f"unsupported dtype {t.dtype}: use torch.float32 or torch.bfloat16")


def _check(t, name, ndim, dtype, device):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _stream_ptr(device):
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _stream_of(device):
    """The current stream of an indexed device, as an address (without a Stream object, which
    costs small calls two microseconds)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def _with_workspace(nbytes: int, device, fn):
    import torch
    ws = torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)
    L = lib()
    _raise(L.topk_set_workspace(ctypes.c_void_p(ws.data_ptr()), int(nbytes)))
    try:
        _raise(fn())
    finally:
        L.topk_set_workspace(None, 0)
    return ws  # caller keeps it until the call is enqueued (stream-ordered reuse is safe)


def attn_workspace_bytes(B, H, Lq, Lk, d, k, chunk=0, causal=False, dtype=TOPK_BF16) -> int:
    return int(lib().topk_attn_workspace_bytes(B, H, Lq, Lk, d, k, chunk, int(causal), dtype))


def ffn_workspace_bytes(N, d_model, d_ff, k, chunk=0, dtype=TOPK_BF16) -> int:
    return int(lib().topk_ffn_workspace_bytes(N, d_model, d_ff, k, chunk, dtype))


def attn_path(B, H, Lq, Lk, d, k, chunk=0, causal=False, dtype=TOPK_BF16) -> int:
    """1 = fused score+filter path, 2 = chunk-tile path, 3 = both, by rows, 4 = filtered chunk-tile path
    (negative: invalid arguments); short rows and few queries as topk_attn.h says."""
    return int(lib().topk_attn_path(B, H, Lq, Lk, d, k, chunk, int(causal), dtype))


def ffn_path(N, d_model, d_ff, k, chunk=0, dtype=TOPK_BF16) -> int:
    return int(lib().topk_ffn_path(N, d_model, d_ff, k, chunk, dtype))


def attn(q, k, v, topk: int, chunk: int = 0, causal: bool = False, scale: float | None = None,
         debug: bool = False, cache: bool = False):
    """Top-k attention over [B, H, L, d] tensors; returns out (and idx, scores if debug
    or cache).

    ``scale`` is the softmax temperature 1/lambda of Eq. 1 (default 1/sqrt(d)).
    ``debug`` also returns the selected indices (int32 [B, H, Lq, topk], -1 pads) and
    their raw fp32 scores (-inf pads), ordered by (score desc, index asc), and records
    the fallback row count (the call waits for the stream). ``cache`` returns the same
    two tensors, the backward pass's input-checkpointing cache, without waiting.
    """
    import torch
    device = q.device
    _check(q, "q", 4, q.dtype, device)
    _check(k, "k", 4, q.dtype, device)
    _check(v, "v", 4, q.dtype, device)
    B, H, Lq, d = q.shape
    Lk = k.shape[2]
    if tuple(k.shape) != (B, H, Lk, d) or tuple(v.shape) != (B, H, Lk, d):
        raise ValueError(f"shape mismatch q {tuple(q.shape)} k {tuple(k.shape)} v {tuple(v.shape)}")
    dt = _dtype_code(q)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if topk == Lk and topk > MAX_SELECT_K and not (debug or cache):
        return attn_dense(q, k, v, chunk, causal, scale)
    out = torch.empty_like(q)
    idx = torch.empty((B, H, Lq, topk), dtype=torch.int32, device=device) if debug or cache else None
    sc = torch.empty((B, H, Lq, topk), dtype=torch.float32, device=device) if debug or cache else None
    L = lib()
    nbytes = L.topk_attn_workspace_bytes(B, H, Lq, Lk, d, topk, chunk, int(causal), dt)
    if nbytes == 0:  # invalid arguments: let the call report why
        _raise(L.topk_attn(None, None, None, None, B, H, Lq, Lk, d, topk, chunk, int(causal), scale, dt, None))
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, Lq, Lk, d, topk, chunk, int(causal),
            float(scale), dt, _stream_ptr(device))
    if debug or cache:
        fn = L.topk_attn_debug if debug else L.topk_attn_with_cache
        _with_workspace(nbytes, device, lambda: fn(*args, idx.data_ptr(), sc.data_ptr()))
        return out, idx, sc
    _with_workspace(nbytes, device, lambda: L.topk_attn(*args))
    return out


def scan_ablation(q, k, topk: int, chunk: int = 0, score_only: bool = False):
    """Measurement hook: only the fused path's score kernel of an attention call
    (``score_only``: the score-core ablation without the filter); time it with
    profile_begin / profile_end (stage "score")."""
    B, H, Lq, d = q.shape
    Lk = k.shape[2]
    _raise(lib().topk_scan_ablation(q.data_ptr(), k.data_ptr(), B, H, Lq, Lk, d, topk, chunk, int(score_only),
                                    _stream_ptr(q.device)))


def probe_mfma():
    """(sustained bf16 MFMA TFLOP/s, shader clock MHz) of the current device."""
    t, c = ctypes.c_double(), ctypes.c_double()
    import torch
    _raise(lib().topk_probe_mfma(ctypes.byref(t), ctypes.byref(c), _stream_ptr(torch.device("cuda", torch.cuda.current_device()))))
    return t.value, c.value


def attn_dense(q, k, v, chunk: int = 0, causal: bool = False, scale: float | None = None):
    """Query chunking with the top-k disabled (the paper's comparison baseline): every
    valid key contributes through the softmax of Eq. 1 (k = Lk). bf16, d = 64 or 128;
    no workspace."""
    import torch
    device = q.device
    _check(q, "q", 4, q.dtype, device)
    _check(k, "k", 4, q.dtype, device)
    _check(v, "v", 4, q.dtype, device)
    B, H, Lq, d = q.shape
    Lk = k.shape[2]
    if tuple(k.shape) != (B, H, Lk, d) or tuple(v.shape) != (B, H, Lk, d):
        raise ValueError(f"shape mismatch q {tuple(q.shape)} k {tuple(k.shape)} v {tuple(v.shape)}")
    dt = _dtype_code(q)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    out = torch.empty_like(q)
    _raise(lib().topk_attn_dense(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, Lq, Lk, d, chunk,
                                 int(causal), float(scale), dt, _stream_ptr(device)))
    return out


def ffn(x, w1, w2, topk: int, chunk: int = 0, debug: bool = False, cache: bool = False):
    """Top-k feed-forward layer: x [N, d_model], w1/w2 [d_ff, d_model] (row j = key/value j).
    ``debug`` / ``cache`` as for ``attn``."""
    import torch
    device = x.device
    _check(x, "x", 2, x.dtype, device)
    _check(w1, "w1", 2, x.dtype, device)
    _check(w2, "w2", 2, x.dtype, device)
    N, dm = x.shape
    dff = w1.shape[0]
    if tuple(w1.shape) != (dff, dm) or tuple(w2.shape) != (dff, dm):
        raise ValueError(f"shape mismatch x {tuple(x.shape)} w1 {tuple(w1.shape)} w2 {tuple(w2.shape)}")
    dt = _dtype_code(x)
    out = torch.empty_like(x)
    idx = torch.empty((N, topk), dtype=torch.int32, device=device) if debug or cache else None
    sc = torch.empty((N, topk), dtype=torch.float32, device=device) if debug or cache else None
    L = lib()
    nbytes = L.topk_ffn_workspace_bytes(N, dm, dff, topk, chunk, dt)
    if nbytes == 0:
        _raise(L.topk_ffn(None, None, None, None, N, dm, dff, topk, chunk, dt, None))
    args = (x.data_ptr(), w1.data_ptr(), w2.data_ptr(), out.data_ptr(), N, dm, dff, topk, chunk, dt,
            _stream_ptr(device))
    if debug or cache:
        fn = L.topk_ffn_debug if debug else L.topk_ffn_with_cache
        _with_workspace(nbytes, device, lambda: fn(*args, idx.data_ptr(), sc.data_ptr()))
        return out, idx, sc
    _with_workspace(nbytes, device, lambda: L.topk_ffn(*args))
    return out


def attn_backward(q, k, v, idx, dots, d_out, scale: float | None = None):
    """Gradients (d_q, d_k, d_v) of top-k attention from the forward's cache: idx and
    dots are what ``attn(..., debug=True)`` returns (selected keys, their raw scores).
    Input checkpointing (Section 2.2): no Lq x Lk matrix is formed."""
    import torch
    device = q.device
    _check(q, "q", 4, q.dtype, device)
    _check(k, "k", 4, q.dtype, device)
    _check(v, "v", 4, q.dtype, device)
    _check(d_out, "d_out", 4, q.dtype, device)
    B, H, Lq, d = q.shape
    Lk = k.shape[2]
    topk = idx.shape[-1]
    if tuple(k.shape) != (B, H, Lk, d) or tuple(v.shape) != (B, H, Lk, d) or tuple(d_out.shape) != (B, H, Lq, d):
        raise ValueError("shape mismatch")
    if idx.dtype != torch.int32 or dots.dtype != torch.float32 or tuple(idx.shape) != (B, H, Lq, topk) \
            or tuple(dots.shape) != (B, H, Lq, topk) or not idx.is_contiguous() or not dots.is_contiguous():
        raise ValueError("idx (int32) and dots (float32) must be contiguous [B, H, Lq, k]")
    dt = _dtype_code(q)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    L = lib()
    nbytes = L.topk_attn_backward_workspace_bytes(B, H, Lq, Lk, d, topk, dt)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), idx.data_ptr(), dots.data_ptr(), d_out.data_ptr(),
            dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Lq, Lk, d, topk, float(scale), dt, _stream_ptr(device))
    if nbytes == 0:
        _raise(L.topk_attn_backward(*args))
    _with_workspace(nbytes, device, lambda: L.topk_attn_backward(*args))
    return dq, dk, dv


def ffn_backward(x, w1, w2, idx, dots, d_out):
    """Gradients (d_x, d_w1, d_w2) of the top-k feed-forward layer from the forward's
    cache (idx, dots as ``ffn(..., debug=True)`` returns them)."""
    import torch
    device = x.device
    for t, n in ((x, "x"), (w1, "w1"), (w2, "w2"), (d_out, "d_out")):
        _check(t, n, 2, x.dtype, device)
    N, dm = x.shape
    dff = w1.shape[0]
    topk = idx.shape[-1]
    if tuple(w1.shape) != (dff, dm) or tuple(w2.shape) != (dff, dm) or tuple(d_out.shape) != (N, dm):
        raise ValueError("shape mismatch")
    if idx.dtype != torch.int32 or dots.dtype != torch.float32 or tuple(idx.shape) != (N, topk) \
            or tuple(dots.shape) != (N, topk) or not idx.is_contiguous() or not dots.is_contiguous():
        raise ValueError("idx (int32) and dots (float32) must be contiguous [N, k]")
    dt = _dtype_code(x)
    dx, dw1, dw2 = torch.empty_like(x), torch.empty_like(w1), torch.empty_like(w2)
    L = lib()
    nbytes = L.topk_ffn_backward_workspace_bytes(N, dm, dff, topk, dt)
    args = (x.data_ptr(), w1.data_ptr(), w2.data_ptr(), idx.data_ptr(), dots.data_ptr(), d_out.data_ptr(),
            dx.data_ptr(), dw1.data_ptr(), dw2.data_ptr(), N, dm, dff, topk, dt, _stream_ptr(device))
    if nbytes == 0:
        _raise(L.topk_ffn_backward(*args))
    _with_workspace(nbytes, device, lambda: L.topk_ffn_backward(*args))
    return dx, dw1, dw2


def _rows(t, name, shape, dtype, device):
    """A tensor whose last dimension is contiguous; the others may have any strides."""
    if t.device == device and t.dtype == dtype and t.shape == shape and device.type == "cuda" and t.stride()[-1] == 1:
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.shape[-1] != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")


def _launch(device, fn, args, nbytes: int = 0):
    """fn(*args) with the tensors' device current and a workspace of nbytes; raises on a status."""
    import torch
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _launch(device, fn, args, nbytes)
    if nbytes:
        _with_workspace(nbytes, device, lambda: fn(*args))
        return
    rc = fn(*args)
    if rc:
        _raise(rc)


def rope_frequencies(sections, theta: float = 10000.0, restart: bool = False, device="cuda"):
    """Radians a position of each feature pair, for ``rope``: theta^(-p / n) for n pairs.
    ``sections`` is n, or the pairs of each axis; with ``restart`` every axis begins at 1."""
    import torch
    parts = [int(n) for n in ((sections,) if isinstance(sections, int) else sections)]
    if not parts or min(parts) < 0:
        raise ValueError(f"sections must be pair counts, got {sections}")
    runs = parts if restart else [sum(parts)]
    return torch.cat([float(theta) ** (-torch.arange(n, dtype=torch.float64, device="cpu") / max(n, 1)) for n in runs]).to(device)


def rope_axes(sections, interleaved: bool = False) -> tuple:
    """The axis of each pair, for ``rope``: ``sections[a]`` pairs turn by axis a, in order, or
    in turns (pair 0 by axis 0, pair 1 by axis 1, ...; axes that are used up are passed over)."""
    left = [int(n) for n in sections]
    if not interleaved:
        return tuple(a for a, n in enumerate(left) for _ in range(n))
    out = []
    for turn in range(max(left, default=0)):
        out += [a for a, n in enumerate(left) if turn < n]
    return tuple(out)


def _rotation(positions, freqs, axes, adjacent, inverse, B, L, d, device):
    """(topk_rotation, or None where nothing is rotated; what it points to)."""
    import torch
    if freqs is None or freqs.numel() == 0:
        if freqs is None and (positions is not None or axes is not None):
            raise ValueError("positions and axes need freqs")
        return None
    if positions is None:
        raise ValueError("freqs need positions")
    for t, n in ((positions, "positions"), (freqs, "freqs")):
        if not t.is_cuda or t.device != device:
            raise ValueError(f"{n} must be on {device}, got {t.device}")
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
        raise TypeError("freqs must be a contiguous float64 vector, one entry a pair")
    n = freqs.shape[0]
    if 2 * n > d:
        raise ValueError(f"{n} pairs do not fit into {d} features")
    if positions.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"positions must be int32 or int64, got {positions.dtype}")
    shape, st = tuple(positions.shape), tuple(positions.stride())
    if not 1 <= len(shape) <= 3:
        raise ValueError(f"positions must be [L], [B, L] or [axes, B, L], got {shape}")
    shape, st = (1,) * (3 - len(shape)) + shape, (0,) * (3 - len(st)) + st
    if shape[1] not in (1, B) or shape[2] not in (1, L):
        raise ValueError(f"positions of shape {tuple(positions.shape)} do not go with B = {B}, L = {L}")
    if axes is None:
        if shape[0] != 1:
            raise ValueError("positions on several axes need axes: the axis of each pair")
    elif len(axes) != n:
        raise ValueError(f"axes must name one axis for each of {n} pairs, got {len(axes)}")
    return _Rotation(positions.data_ptr(), freqs.data_ptr(), None if axes is None else bytes(axes), 2 * n,
                     st[0], st[1] if shape[1] > 1 else 0, st[2] if shape[2] > 1 else 0, shape[0],
                     positions.element_size(), int(adjacent), int(inverse))


def rope(x, positions, freqs, axes=None, adjacent: bool = False, inverse: bool = False):
    """Rotary positions: x [B, H, L, d] with each feature pair p turned by
    positions[axes[p]] * freqs[p] radians; features beyond the 2 * len(freqs) first pass.

    ``positions``: int32 or int64, [L], [B, L] or [axes, B, L] (size 1 broadcasts), any
    values; ``freqs``: float64, one entry a pair (``rope_frequencies``); ``axes``: the axis
    of each pair (``rope_axes``), needed with several. A pair is features p and
    p + len(freqs), or 2p and 2p + 1 with ``adjacent``. ``inverse`` turns back, which is
    also the gradient. x may have any strides but for the last dimension; the result is
    contiguous. bf16 or fp32, d even, at most 512."""
    import torch
    device = x.device
    if x.dim() != 4:
        raise ValueError(f"x must have 4 dimensions, got {tuple(x.shape)}")
    B, H, L, d = x.shape
    _rows(x, "x", x.shape, x.dtype, device)
    dt = _dtype_code(x)
    rot = _rotation(positions, freqs, axes, adjacent, inverse, B, L, d, device)
    out = torch.empty((B, H, L, d), dtype=x.dtype, device=device)
    sb, sh, sl, _ = x.stride()
    _launch(device, lib().topk_rope,
            (x.data_ptr(), out.data_ptr(), B, H, L, d, sb, sh, sl, rot, dt, _stream_of(device)))
    return out


def _qkv(qkv, heads, kv_heads, q_weight, k_weight, norm):
    """Checks of the packed projection; (B, L, d)."""
    if qkv.dim() != 3:
        raise ValueError(f"qkv must have 3 dimensions, got {tuple(qkv.shape)}")
    B, L, W = qkv.shape
    if heads < 1 or kv_heads < 1 or W % (heads + 2 * kv_heads):
        raise ValueError(f"{W} columns are not {heads} query and 2 x {kv_heads} key and value heads of one size")
    d = W // (heads + 2 * kv_heads)
    _rows(qkv, "qkv", qkv.shape, qkv.dtype, qkv.device)
    for w, n in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None:
            if not norm:
                raise ValueError(f"{n} scales a norm that is switched off")
            _check(w, n, 1, qkv.dtype, qkv.device)
            if w.shape[0] != d:
                raise ValueError(f"{n} must have {d} entries, got {w.shape[0]}")
    return B, L, d


def _ptr(t):
    return None if t is None else t.data_ptr()


def qk_norm_rope(qkv, heads: int, kv_heads: int, q_weight=None, k_weight=None, positions=None, freqs=None, axes=None,
                 adjacent: bool = False, eps: float = 1e-6, norm: bool = True):
    """(q [B, heads, L, d], k, v [B, kv_heads, L, d]) from the packed projection qkv
    [B, L, (heads + 2 kv_heads) d]: query and key heads divided by their root mean square
    (``norm``), scaled by q_weight / k_weight [d] and rotated as ``rope`` says (freqs None:
    not); values as they are. One pass; what ``attn_prefix`` takes, and with kv_heads ==
    heads ``attn`` and ``attn_dense``."""
    import torch
    B, L, d = _qkv(qkv, heads, kv_heads, q_weight, k_weight, norm)
    device = qkv.device
    dt = _dtype_code(qkv)
    rot = _rotation(positions, freqs, axes, adjacent, False, B, L, d, device)
    q, k = qkv.new_empty((B, heads, L, d)), qkv.new_empty((B, kv_heads, L, d))
    v = torch.empty_like(k)
    sb, sl, _ = qkv.stride()
    _launch(device, lib().topk_qk_norm_rope,
            (qkv.data_ptr(), _ptr(q_weight), _ptr(k_weight), q.data_ptr(), k.data_ptr(), v.data_ptr(), B, L, heads, kv_heads,
             d, sb, sl, int(norm), float(eps), rot, dt, _stream_of(device)))
    return q, k, v


def qk_norm_rope_append(qkv, heads: int, kv_heads: int, k_cache, v_cache, lengths, q_weight=None, k_weight=None,
                        positions=None, freqs=None, axes=None, adjacent: bool = False, eps: float = 1e-6,
                        norm: bool = True):
    """``qk_norm_rope`` for serving: returns q; keys and values of token l of request b are
    written to row ``lengths[b] + l`` of k_cache / v_cache [B, kv_heads, S, d] (any strides
    but for the last dimension). Rows at S and behind are dropped; no other row changes.
    ``lengths`` (int32 [B], on the GPU) is not advanced."""
    import torch
    B, L, d = _qkv(qkv, heads, kv_heads, q_weight, k_weight, norm)
    device = qkv.device
    dt = _dtype_code(qkv)
    S = k_cache.shape[2] if k_cache.dim() == 4 else 0
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _rows(t, n, (B, kv_heads, S, d), qkv.dtype, device)
        if 0 in t.stride() and any(st == 0 and size > 1 for st, size in zip(t.stride(), t.shape)):
            raise ValueError(f"{n} is written to and must not be expanded")
    if S and k_cache.data_ptr() == v_cache.data_ptr():
        raise ValueError("k_cache and v_cache are the same memory")
    _check(lengths, "lengths", 1, torch.int32, device)
    if lengths.shape[0] != B:
        raise ValueError(f"lengths must have {B} entries, got {lengths.shape[0]}")
    rot = _rotation(positions, freqs, axes, adjacent, False, B, L, d, device)
    q = torch.empty((B, heads, L, d), dtype=qkv.dtype, device=device)
    if S == 0:  # nothing can be stored; the library wants an address all the same
        k_cache = v_cache = q
    sb, sl, _ = qkv.stride()
    _launch(device, lib().topk_qk_norm_rope_append,
            (qkv.data_ptr(), _ptr(q_weight), _ptr(k_weight), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
             lengths.data_ptr(), B, L, heads, kv_heads, d, sb, sl, S, *k_cache.stride()[:3], *v_cache.stride()[:3],
             int(norm), float(eps), rot, dt, _stream_of(device)))
    return q


def qk_norm_rope_backward(qkv, heads: int, kv_heads: int, d_q, d_k, d_v, q_weight=None, k_weight=None, positions=None,
                          freqs=None, axes=None, adjacent: bool = False, eps: float = 1e-6, norm: bool = True,
                          weights: bool = True):
    """Gradients (d_qkv, d_q_weight, d_k_weight) of ``qk_norm_rope`` from its input and the
    gradients of q, k and v (contiguous). The weights' are None where there is no weight,
    or with ``weights`` false; they are summed in a fixed order."""
    import torch
    B, L, d = _qkv(qkv, heads, kv_heads, q_weight, k_weight, norm)
    device = qkv.device
    dt = _dtype_code(qkv)
    for t, n, h in ((d_q, "d_q", heads), (d_k, "d_k", kv_heads), (d_v, "d_v", kv_heads)):
        _check(t, n, 4, qkv.dtype, device)
        if tuple(t.shape) != (B, h, L, d):
            raise ValueError(f"{n} must have shape {(B, h, L, d)}, got {tuple(t.shape)}")
    rot = _rotation(positions, freqs, axes, adjacent, False, B, L, d, device)
    dqkv = torch.empty(qkv.shape, dtype=qkv.dtype, device=device)
    dwq, dwk = (torch.empty_like(w) if weights and w is not None else None for w in (q_weight, k_weight))
    Lb = lib()
    sb, sl, _ = qkv.stride()
    args = (qkv.data_ptr(), _ptr(q_weight), _ptr(k_weight), d_q.data_ptr(), d_k.data_ptr(), d_v.data_ptr(), dqkv.data_ptr(),
            _ptr(dwq), _ptr(dwk), B, L, heads, kv_heads, d, sb, sl, int(norm), float(eps), rot, dt, _stream_of(device))
    nbytes = 0
    if dwq is not None or dwk is not None:
        nbytes = Lb.topk_qk_norm_rope_backward_workspace_bytes(B, L, heads, kv_heads, d, rot.d_rot if rot else 0, dt)
    _launch(device, Lb.topk_qk_norm_rope_backward, args, nbytes)
    return dqkv, dwq, dwk


def attn_prefix_workspace_bytes(B, H, Hkv, Lq, P, S, d, dtype=TOPK_BF16) -> int:
    return int(lib().topk_attn_prefix_workspace_bytes(B, H, Hkv, Lq, P, S, d, dtype))


def attn_prefix(q, prefix_k, prefix_v, k=None, v=None, lengths=None, causal: bool = True, scale: float | None = None,
                lse: bool = False):
    """Attention over every valid key (Eq. 1) of B requests behind one shared prefix:
    q [B, H, Lq, d]; prefix_k, prefix_v [Hkv, P, d], one copy for all; k, v [B, Hkv, S, d],
    each request's own cache, of which the first ``lengths[b]`` rows count (int32 [B] on the
    GPU, taken into [0, S]; None: all). H / Hkv query heads share a key head. ``causal``: the
    queries are the last Lq positions of their request, so query i sees own keys
    j <= lengths[b] - Lq + i, and the whole prefix. A row that sees nothing is 0.

    Returns out [B, H, Lq, d]; with ``lse`` also the fp32 [B, H, Lq] logarithm of the sum of
    exp(scale * score), by which results over different keys can be joined. Keys and values
    may have any strides but for the last dimension (caches cut from larger ones), multiples
    of 8; None stands for no keys. bf16, d = 64 or 128. Forward only.

    The work is divided for S keys a request. Where caches have far more rows than any
    request holds, pass them cut (``k[:, :, :n]``, n at least the longest length): behind 65536
    shared keys 8 requests of up to 1000 take 105 us so, 354 with caches of 131072 rows."""
    import torch
    device = q.device
    _check(q, "q", 4, q.dtype, device)
    B, H, Lq, d = q.shape
    dt = _dtype_code(q)
    given = [t for t in (prefix_k, k) if t is not None]
    if not given:
        raise ValueError("attn_prefix needs a prefix or a cache")
    if (prefix_k is None) != (prefix_v is None) or (k is None) != (v is None):
        raise ValueError("keys and values go together")
    Hkv = given[0].shape[given[0].dim() - 3] if given[0].dim() >= 3 else 0
    P = prefix_k.shape[-2] if prefix_k is not None and prefix_k.dim() == 3 else 0
    S = k.shape[-2] if k is not None and k.dim() == 4 else 0
    st = _PrefixStrides()
    for t, n in ((prefix_k, "prefix_k"), (prefix_v, "prefix_v")):
        if t is not None:
            _rows(t, n, (Hkv, P, d), q.dtype, device)
    for t, n in ((k, "k"), (v, "v")):
        if t is not None:
            _rows(t, n, (B, Hkv, S, d), q.dtype, device)
    if P:
        st.prefix_k_head, st.prefix_k_key, st.prefix_v_head, st.prefix_v_key = prefix_k.stride()[:2] + prefix_v.stride()[:2]
    if S:
        st.k_batch, st.k_head, st.k_key, st.v_batch, st.v_head, st.v_key = k.stride()[:3] + v.stride()[:3]
    if lengths is not None:
        _check(lengths, "lengths", 1, torch.int32, device)
        if lengths.shape[0] != B:
            raise ValueError(f"lengths must have {B} entries, got {lengths.shape[0]}")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    out = torch.empty_like(q)
    sums = torch.empty((B, H, Lq), dtype=torch.float32, device=device) if lse else None
    L = lib()
    nbytes = L.topk_attn_prefix_workspace_bytes(B, H, Hkv, Lq, P, S, d, dt)
    args = (q.data_ptr(), _ptr(prefix_k), _ptr(prefix_v), _ptr(k), _ptr(v), _ptr(lengths), out.data_ptr(), _ptr(sums),
            B, H, Hkv, Lq, P, S, d, st, int(causal), float(scale), dt, _stream_of(device))
    _launch(device, L.topk_attn_prefix, args, nbytes)
    return (out, sums) if lse else out


STAGES = ("score", "select", "redo", "finalize", "backward")


def profile_begin():
    """Start per-stage HIP-event timing of this thread's calls (see topk_profile_begin)."""
    _raise(lib().topk_profile_begin())


def profile_end():
    """Stop timing; return {stage: (total_ms, launches)} over the calls since profile_begin."""
    ms = (ctypes.c_double * len(STAGES))()
    n = (ctypes.c_int64 * len(STAGES))()
    _raise(lib().topk_profile_end(ms, n, len(STAGES)))
    return {s: (ms[i], n[i]) for i, s in enumerate(STAGES)}


def set_memory_budget(nbytes: int) -> None:
    """Most workspace a forward call sizes for itself (process-wide; 0 = 8 GiB). A small
    budget runs the query chunks in more passes (one chunk per pass at the limit)."""
    _raise(lib().topk_set_memory_budget(int(nbytes)))


def set_backward_lists(mode: int) -> None:
    """How backward calls group the selected pairs by key (process-wide):
    TOPK_LISTS_AUTO, TOPK_LISTS_BUCKET (stable bucket sort) or TOPK_LISTS_ATOMIC."""
    _raise(lib().topk_set_backward_lists(int(mode)))


def last_fallback_rows() -> int:
    """Rows the last debug call on this thread selected through a fallback path (-1: none / failed)."""
    return int(lib().topk_last_fallback_rows())


def mfma_layout(device="cuda"):
    """(rows, cols) int32 [64, 16]: output row / column held by lane l, register v of
    the bf16 32x32x16 MFMA the fused scan uses (test hook)."""
    import torch
    rows = torch.full((64, 16), -1, dtype=torch.int32, device=device)
    cols = torch.full((64, 16), -1, dtype=torch.int32, device=device)
    _raise(lib().topk_selftest_mfma_layout(ctypes.c_void_p(rows.data_ptr()), ctypes.c_void_p(cols.data_ptr()),
                                           _stream_ptr(torch.device(device))))
    return rows, cols
