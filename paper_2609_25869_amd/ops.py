"""Rotary positions and window attention on torch tensors.

Python binding of libbsa_ops.so (include/bsa_ops.h); the package exports these
functions.  Tensors are CUDA tensors [B, N, H, d] with d contiguous and 16-byte
aligned rows.  Work runs on the tensors' device, on its current stream unless
one is given; outputs and workspaces that are not passed in are allocated for
that stream.  Nothing here takes part in autograd: backward passes are calls of
their own (rope with inverse=True, window_backward).
"""
from __future__ import annotations

import contextlib
import ctypes
import math
from typing import Optional, Sequence, Tuple

from . import _ops_ffi
from ._ffi import BSA_OK, BsaError, DTYPE_BF16, DTYPE_F16, DTYPE_F32
from ._ops_ffi import RopeShapes, WindowGrads, WindowShapes

_lib = _ops_ffi.load()

ALL = -1  # window sides: every key


def _check(status: int):
    if status != BSA_OK:
        raise BsaError(status, _lib.bsa_ops_last_error().decode(errors="replace"))


def _torch():
    import torch
    return torch


def _dtype_code(dtype):
    torch = _torch()
    code = {torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16, torch.float32: DTYPE_F32}.get(dtype)
    if code is None:
        raise TypeError("tensors must be bfloat16, float16 or float32, not %s" % dtype)
    return code


def _want(name, t, like=None, shape=None):
    """t as a [B, N, H, d] tensor of like's device and type."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("%s must be [B, N, H, d] with d contiguous" % name)
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError("%s must be %s on %s" % (name, like.dtype, like.device))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    return t


def _want_ints(name, t, device, shape):
    torch = _torch()
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.device != device:
        raise TypeError("%s must be an int32 tensor on %s" % (name, device))
    if tuple(t.shape) != tuple(shape) or (t.numel() > 1 and t.stride(-1) != 1):
        raise ValueError("%s must have shape %s, its last dimension contiguous" % (name, tuple(shape)))
    return t.data_ptr()


def _set(dst, t):
    s = t.stride()
    dst[0], dst[1], dst[2] = s[0], s[2], s[1]


@contextlib.contextmanager
def _on(device, stream):
    """Makes `device` current, and yields the handle of `stream` (None: the
    device's current stream); allocations inside belong to that stream."""
    torch = _torch()
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream(device).cuda_stream
            return
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):
            yield handle


# ----------------------------------------------------------------------------
# Rotary positions

def rope_frequencies(pairs: Sequence[int], theta: float = 10000.0, shared: bool = False, device="cuda"):
    """float64 [sum(pairs)] angles per position, for `pairs` turned pairs on each
    axis: theta^(-i / n) over the n pairs of each axis, or with shared=True over
    all pairs in a row (text and image positions that share one ladder)."""
    torch = _torch()
    n_all, f = sum(pairs), []
    for n in pairs:
        start = len(f)
        f += [theta ** (-((start + i) / n_all if shared else i / n)) for i in range(n)]
    return torch.tensor(f, dtype=torch.float64, device=device)


def rope(q, k=None, v=None, *, freq, pairs: Sequence[int], interleaved: bool = True, positions=None,
         grid: Optional[Sequence[int]] = None, origin: Sequence[int] = (0, 0, 0), lengths=None, rows=None, out_q=None,
         out_k=None, out_v=None, inverse: bool = False, stream=None) -> Tuple:
    """Rotary positions of Q and K on up to three axes (bsa_rope).

    q is [B, N, H, d], k and v [B, N, Hkv, d].  The first sum(pairs) pairs of a
    head are turned, pairs[a] of them by the position on axis a (time, height,
    width) times `freq` (rope_frequencies).  Positions are an int32 tensor
    [axes, B, N] (or [axes, 1, N], the same for the batch), or the points of a
    `grid` (T, H, W) from `origin` on; tokens past the grid stay as they are.
    `lengths` int32 [B]: tokens of each sequence, output rows behind them are
    left as they were.  `rows` int32 [B]: rows of out_k and out_v that the
    sequences' first tokens go to (new tokens of a cache [B, capacity, Hkv, d]);
    v is copied there unturned.  inverse=True turns back: the backward pass on
    gradients.  out_q may be q, and out_k k.  Returns the outputs of the tensors
    given, allocated where they are not passed in."""
    torch = _torch()
    _want("q", q)
    B, N, H, d = q.shape
    s = RopeShapes()
    s.dtype = _dtype_code(q.dtype)
    dev = q.device
    if v is not None and k is None:
        raise ValueError("v needs k")
    Hkv = 0
    if k is not None:
        _want("k", k, q)
        Hkv = k.shape[2]
        if tuple(k.shape) != (B, N, Hkv, d):
            raise ValueError("k must have shape %s, not %s" % ((B, N, Hkv, d), tuple(k.shape)))
        if v is not None:
            _want("v", v, q, k.shape)
    pairs = tuple(int(x) for x in pairs)
    if not 1 <= len(pairs) <= 3:
        raise ValueError("pairs must name one to three axes")
    if (not isinstance(freq, torch.Tensor) or freq.dtype != torch.float64 or freq.device != dev or
            tuple(freq.shape) != (sum(pairs),) or not freq.is_contiguous()):
        raise TypeError("freq must be a contiguous float64 tensor of sum(pairs) elements on %s" % dev)
    if (positions is None) == (grid is None):
        raise ValueError("give either positions or grid")
    if rows is not None and k is None:
        raise ValueError("rows needs k")
    pos_ptr = None
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dim() != 3:
            raise TypeError("positions must be an int32 tensor [axes, B, N]")
        if positions.shape[0] < len(pairs) or positions.shape[1] not in (1, B):
            raise ValueError("positions must be [axes, B, N] or [axes, 1, N] with at least %d axes" % len(pairs))
        pos_ptr = _want_ints("positions", positions, dev, (positions.shape[0], positions.shape[1], N))
        s.pos_stride[0] = positions.stride(0)
        s.pos_stride[1] = positions.stride(1) if positions.shape[1] == B and B > 1 else 0
    else:
        if len(grid) != 3 or len(origin) != 3:
            raise ValueError("grid and origin must be (time, height, width)")
        for i in range(3):
            s.grid[i], s.origin[i] = int(grid[i]), int(origin[i])
    len_ptr = _want_ints("lengths", lengths, dev, (B,))
    row_ptr = _want_ints("rows", rows, dev, (B,))
    if rows is not None and (out_k is None or (v is not None and out_v is None)):
        raise ValueError("rows needs the caches as out_k (and out_v)")
    for i, n in enumerate(pairs):
        s.pairs[i] = n
    s.batch, s.heads, s.kv_heads, s.seq, s.head_dim = B, H, Hkv, N, d
    s.interleaved, s.inverse = 1 if interleaved else 0, 1 if inverse else 0
    with _on(dev, stream) as handle:
        # (rows behind a sequence's end are not written: zeros there, not stale memory)
        new = torch.zeros_like if lengths is not None else torch.empty_like
        fresh = lambda t: new(t, memory_format=torch.contiguous_format)
        out_q = fresh(q) if out_q is None else _want("out_q", out_q, q, q.shape)
        _set(s.q_stride, q)
        _set(s.q_out_stride, out_q)
        outs = [out_q]
        if k is not None:
            if out_k is None:
                out_k = fresh(k)
            _want("out_k", out_k, q)
            cap = out_k.shape[1]
            if tuple(out_k.shape) != (B, cap, Hkv, d) or (rows is None and cap < N):
                raise ValueError("out_k must be [%d, %s, %d, %d]" % (B, "tokens" if rows is not None else N, Hkv, d))
            s.kv_rows = cap
            _set(s.k_stride, k)
            _set(s.k_out_stride, out_k)
            outs.append(out_k)
            if v is not None:
                out_v = fresh(v) if out_v is None else out_v
                _want("out_v", out_v, q)
                if tuple(out_v.shape[::2]) != (B, Hkv) or out_v.shape[3] != d or out_v.shape[1] < (
                        cap if rows is not None else N):
                    raise ValueError("out_v must be shaped like out_k")
                s.kv_rows = min(cap, out_v.shape[1])
                _set(s.v_stride, v)
                _set(s.v_out_stride, out_v)
                outs.append(out_v)
        _check(_lib.bsa_rope(ctypes.byref(s), freq.data_ptr(), pos_ptr, len_ptr, row_ptr, q.data_ptr(),
                             None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                             out_q.data_ptr(), None if k is None else out_k.data_ptr(),
                             None if v is None else out_v.data_ptr(), handle))
    return tuple(outs)


# ----------------------------------------------------------------------------
# Window attention

def _window_shapes(q, k, v, left, right, sinks, scale):
    _want("q", q)
    _want("k", k, q)
    _want("v", v, q)
    B, Nq, H, d = q.shape
    Nkv, Hkv = k.shape[1], k.shape[2]
    if tuple(k.shape) != (B, Nkv, Hkv, d) or tuple(v.shape) != (B, Nkv, Hkv, d):
        raise ValueError("inconsistent q/k/v shapes")
    s = WindowShapes()
    s.batch, s.heads, s.kv_heads, s.seq_q, s.seq_kv, s.head_dim = B, H, Hkv, Nq, Nkv, d
    s.dtype = _dtype_code(q.dtype)
    big = (1 << 31) - 1
    s.left, s.right, s.sinks = min(int(left), big), min(int(right), big), min(int(sinks), big)
    if scale is not None and not (scale > 0 and math.isfinite(scale)):
        raise ValueError("scale must be positive and finite")
    s.scale = 0.0 if scale is None else scale
    _set(s.q_stride, q)
    _set(s.k_stride, k)
    _set(s.v_stride, v)
    return s


def _lse_of(lse, q):
    torch = _torch()
    B, Nq, H, _ = q.shape
    if (not isinstance(lse, torch.Tensor) or lse.dtype != torch.float32 or lse.device != q.device or
            tuple(lse.shape) != (B, H, Nq) or not lse.is_contiguous()):
        raise TypeError("lse must be a contiguous float32 tensor [B, H, Nq] on %s" % q.device)
    return lse


def _workspace(s, backward, workspace, device):
    """(pointer, bytes, tensor to keep alive until the call is made)"""
    torch = _torch()
    need = ctypes.c_size_t()
    _check(_lib.bsa_window_workspace(ctypes.byref(s), backward, ctypes.byref(need)))
    if need.value == 0:
        return None, 0, None
    if workspace is None:
        workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor on %s" % device)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def window_workspace(q, k, v, left: int, right: int = 0, sinks: int = 0, *, backward: bool = False) -> int:
    """Bytes of device workspace that window_forward or window_backward needs for
    these tensors, for callers that pass their own."""
    need = ctypes.c_size_t()
    s = _window_shapes(q, k, v, left, right, sinks, None)
    _set(s.o_stride, q)
    _check(_lib.bsa_window_workspace(ctypes.byref(s), 1 if backward else 0, ctypes.byref(need)))
    return need.value


def window_forward(q, k, v, left: int, right: int = 0, sinks: int = 0, *, scale: Optional[float] = None, q_len=None,
                   kv_len=None, o=None, lse=None, workspace=None, stream=None) -> Tuple:
    """Attention over a sliding window and a few first tokens (bsa_window_forward).

    q is [B, Nq, H, d], k and v [B, Nkv, Hkv, d] in bfloat16 or float16, d 64 or
    128, H a multiple of Hkv.  Query i of a sequence lies at p = i + kv_len - q_len
    and sees the keys p - left .. p + right (ALL or -1: no bound) and of the
    first `sinks` keys those up to p + right.  q_len and kv_len are int32 [B] on
    the device (default: Nq, Nkv).  Returns (o, lse), lse float32 [B, H, Nq]; a
    query that sees nothing gets o = 0 and lse = -inf.  Rows of a given o and
    lse from q_len on keep what they held; allocated ones hold zeros there."""
    torch = _torch()
    s = _window_shapes(q, k, v, left, right, sinks, scale)
    B, Nq, H, _ = q.shape
    dev = q.device
    ql, kl = _want_ints("q_len", q_len, dev, (B,)), _want_ints("kv_len", kv_len, dev, (B,))
    with _on(dev, stream) as handle:
        if o is None:
            o = (torch.empty if q_len is None else torch.zeros)(q.shape, dtype=q.dtype, device=dev)
        else:
            _want("o", o, q, q.shape)
        if lse is None:
            lse = (torch.empty if q_len is None else torch.zeros)((B, H, Nq), dtype=torch.float32, device=dev)
        else:
            _lse_of(lse, q)
        _set(s.o_stride, o)
        ws, n, keep = _workspace(s, 0, workspace, dev)
        _check(_lib.bsa_window_forward(ctypes.byref(s), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                       lse.data_ptr(), ql, kl, ws, n, handle))
    return o, lse


def window_backward(q, k, v, o, lse, do, left: int, right: int = 0, sinks: int = 0, *, scale: Optional[float] = None,
                    q_len=None, kv_len=None, dq=None, dk=None, dv=None, workspace=None, stream=None) -> Tuple:
    """Gradients (dq, dk, dv) of window_forward for the gradient `do` of o
    (bsa_window_backward), with the o and lse that it returned and its other
    arguments unchanged.  Rows of given dq from q_len on, and of dk and dv from
    kv_len on, keep what they held; allocated ones hold zeros there."""
    torch = _torch()
    s = _window_shapes(q, k, v, left, right, sinks, scale)
    B, Nq, H, _ = q.shape
    dev = q.device
    _want("o", o, q, q.shape)
    _want("do", do, q, q.shape)
    _lse_of(lse, q)
    ql, kl = _want_ints("q_len", q_len, dev, (B,)), _want_ints("kv_len", kv_len, dev, (B,))
    g = WindowGrads()
    with _on(dev, stream) as handle:
        def grad(name, t, x, ragged):
            if t is None:
                return (torch.empty if ragged is None else torch.zeros)(x.shape, dtype=x.dtype, device=dev)
            return _want(name, t, x, x.shape)
        dq, dk, dv = grad("dq", dq, q, q_len), grad("dk", dk, k, kv_len), grad("dv", dv, v, kv_len)
        _set(s.o_stride, o)
        _set(g.do_stride, do)
        _set(g.dq_stride, dq)
        _set(g.dk_stride, dk)
        _set(g.dv_stride, dv)
        ws, n, keep = _workspace(s, 1, workspace, dev)
        _check(_lib.bsa_window_backward(ctypes.byref(s), ctypes.byref(g), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                        o.data_ptr(), lse.data_ptr(), do.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                        dv.data_ptr(), ql, kl, ws, n, handle))
    return dq, dk, dv
