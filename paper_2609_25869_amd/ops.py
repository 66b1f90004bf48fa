"""Rotary positions and window attention on torch tensors.

Python binding of libbsa_ops.so (include/bsa_ops.h); the package exports these
functions.  Tensors are CUDA tensors [B, N, H, d] with d contiguous and 16-byte
aligned rows.  Work runs on the tensors' device, on its current stream unless
one is given; outputs and workspaces that are not passed in are allocated for
that stream.  Nothing here takes part in autograd: backward passes are calls of
their own (rope with inverse=True, window_backward), and a call on tensors that
require gradients while torch records them warns that its results have none.

A call of a few microseconds on the device is bound by what the host does for
it, so the checks take each tensor's properties once, the shape structures are
packed in one go, and the device is only changed where it differs.  (One token
of one stream over a cache, two launches of 10 us: 14 us a call, and 21 with a
structure filled field by field and a device context around every call.)
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import struct
import warnings
from typing import Optional, Sequence, Tuple

from . import _ops_ffi
from ._ffi import BSA_OK, BsaError, DTYPE_BF16, DTYPE_F16, DTYPE_F32

_lib = _ops_ffi.load()

try:
    import torch
    _CODES = {torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16, torch.float32: DTYPE_F32}
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
except ImportError:  # the package's host functions work without it
    torch = None

ALL = -1  # window sides: every key

_pack_rope = struct.Struct(_ops_ffi.ROPE_PACK).pack
_pack_window = struct.Struct(_ops_ffi.WINDOW_PACK).pack
_pack_grads = struct.Struct(_ops_ffi.GRADS_PACK).pack
_INT_MAX = (1 << 31) - 1


def _check(status: int):
    if status != BSA_OK:
        raise BsaError(status, _lib.bsa_ops_last_error().decode(errors="replace"))


def _first(name, t):
    """(device, type, type code) of the tensor that the others are held to."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    dtype = t.dtype
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError("tensors must be bfloat16, float16 or float32, not %s" % dtype)
    return t.device, dtype, code


def _rows(name, t, device, dtype, shape=None):
    """Strides of t, a [B, N, H, d] tensor of that device, type and (if given)
    shape, with d contiguous."""
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype is not dtype:
        raise TypeError("%s must be a %s tensor on %s" % (name, dtype, device))
    s = t.stride()
    if len(s) != 4 or (s[3] != 1 and t.shape[3] > 1):
        raise ValueError("%s must be [B, N, H, d] with d contiguous" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    return s


def _ints(name, t, device, n):
    """Address of t, int32 [n] on the device (None: NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or t.device != device:
        raise TypeError("%s must be an int32 tensor on %s" % (name, device))
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s must be contiguous and have shape (%d,)" % (name, n))
    return t.data_ptr()


@contextlib.contextmanager
def _on(device, stream):
    """Makes `device` and `stream` (None: the device's current one) current, so
    that allocations belong to them, and yields the stream's handle."""
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream().cuda_stream
            return
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):
            yield handle


def _run(device, stream, call):
    """call(handle) with `device` and `stream` current."""
    if stream is None and torch.cuda.current_device() == device.index:
        # (building a Stream object to read its handle takes 2.6 us)
        return call(_raw_stream(device.index) if _raw_stream else torch.cuda.current_stream().cuda_stream)
    with _on(device, stream) as handle:
        return call(handle)


def _not_recorded(name, backward):
    """Warns at the caller's line that a call's results carry no gradients."""
    if torch.is_grad_enabled():
        warnings.warn("%s takes no part in autograd: no gradient reaches its inputs through its results (%s gives it; "
                      "call this under torch.no_grad())" % (name, backward), stacklevel=3)


# ----------------------------------------------------------------------------
# Rotary positions

def rope_frequencies(pairs: Sequence[int], theta: float = 10000.0, shared: bool = False, device="cuda"):
    """float64 [sum(pairs)] angles per position, for `pairs` turned pairs on each
    axis: theta^(-i / n) over the n pairs of each axis, or with shared=True over
    all pairs in a row (text and image positions that share one ladder)."""
    n_all, f = sum(pairs), []
    for n in pairs:
        start = len(f)
        f += [theta ** (-((start + i) / n_all if shared else i / n)) for i in range(n)]
    return torch.tensor(f, dtype=torch.float64, device=device)


_NO_STRIDE = (0, 0, 0, 0)


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
    given, allocated where they are not passed in (zeros behind `lengths`).
    They carry no gradients: autograd does not record the call."""
    dev, dtype, code = _first("q", q)
    qs = _rows("q", q, dev, dtype)
    B, N, H, d = q_shape = q.shape
    Hkv, ks, vs = 0, _NO_STRIDE, _NO_STRIDE
    if k is not None:
        Hkv = k.shape[2] if k.dim() == 4 else 0
        kv_shape = (B, N, Hkv, d)
        ks = _rows("k", k, dev, dtype, kv_shape)
        if v is not None:
            vs = _rows("v", v, dev, dtype, kv_shape)
    elif v is not None or rows is not None:
        raise ValueError("v and rows need k")
    n_axes = len(pairs)
    if not 1 <= n_axes <= 3:
        raise ValueError("pairs must name one to three axes")
    p0, p1, p2 = (tuple(pairs) + (0, 0))[:3]
    if (not isinstance(freq, torch.Tensor) or freq.dtype is not torch.float64 or freq.device != dev or
            freq.shape != (p0 + p1 + p2,) or not freq.is_contiguous()):
        raise TypeError("freq must be a contiguous float64 tensor of sum(pairs) elements on %s" % dev)
    g0 = g1 = g2 = o0 = o1 = o2 = 0
    pos_ptr, ps0, ps1 = None, 0, 0
    if positions is not None:
        if grid is not None:
            raise ValueError("give either positions or grid")
        if not isinstance(positions, torch.Tensor) or positions.dtype is not torch.int32 or positions.device != dev:
            raise TypeError("positions must be an int32 tensor on %s" % dev)
        shape = positions.shape
        if len(shape) != 3 or shape[0] < n_axes or shape[1] not in (1, B) or shape[2] != N:
            raise ValueError("positions must be [axes, B, N] or [axes, 1, N] with at least %d axes" % n_axes)
        ps0, ps1, ps2 = positions.stride()
        if N > 1 and ps2 != 1:
            raise ValueError("positions must be contiguous along the tokens")
        if shape[1] == 1:
            ps1 = 0
        pos_ptr = positions.data_ptr()
    elif grid is None:
        raise ValueError("give either positions or grid")
    else:
        (g0, g1, g2), (o0, o1, o2) = grid, origin
    if q.requires_grad or (k is not None and k.requires_grad) or (v is not None and v.requires_grad):
        _not_recorded("rope", "rope with inverse=True")
    len_ptr, row_ptr = _ints("lengths", lengths, dev, B), _ints("rows", rows, dev, B)
    if rows is not None and (out_k is None or (v is not None and out_v is None)):
        raise ValueError("rows needs the caches as out_k (and out_v)")

    def call(handle):
        nonlocal out_q, out_k, out_v
        # (rows behind a sequence's end are not written: zeros there, not stale memory)
        new = torch.empty if lengths is None else torch.zeros
        if out_q is None:
            out_q = new(q_shape, dtype=dtype, device=dev)
        oqs, oks, ovs, cap = _rows("out_q", out_q, dev, dtype, q_shape), _NO_STRIDE, _NO_STRIDE, 0
        if k is not None:
            if out_k is None:
                out_k = new(kv_shape, dtype=dtype, device=dev)
            if v is not None and out_v is None:
                out_v = new(kv_shape, dtype=dtype, device=dev)
            cap = N if rows is None else out_k.shape[1] if out_k.dim() == 4 else 0
            out_shape = (B, cap, Hkv, d)
            oks = _rows("out_k", out_k, dev, dtype, out_shape)
            if v is not None:
                ovs = _rows("out_v", out_v, dev, dtype, out_shape)
        s = _pack_rope(B, H, Hkv, N, d, code, p0, p1, p2, 1 if interleaved else 0, 1 if inverse else 0, g0, g1, g2, o0,
                       o1, o2, cap, ps0, ps1, qs[0], qs[2], qs[1], ks[0], ks[2], ks[1], vs[0], vs[2], vs[1],
                       oqs[0], oqs[2], oqs[1], oks[0], oks[2], oks[1], ovs[0], ovs[2], ovs[1])
        _check(_lib.bsa_rope(s, freq.data_ptr(), pos_ptr, len_ptr, row_ptr, q.data_ptr(),
                             None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                             out_q.data_ptr(), None if k is None else out_k.data_ptr(),
                             None if v is None else out_v.data_ptr(), handle))

    _run(dev, stream, call)
    return (out_q,) if k is None else (out_q, out_k) if v is None else (out_q, out_k, out_v)


# ----------------------------------------------------------------------------
# Window attention

def _window_head(q, k, v, left, right, sinks, scale):
    """(device, type, q's shape, k's shape, packed fields but O's strides)"""
    dev, dtype, code = _first("q", q)
    qs = _rows("q", q, dev, dtype)
    B, Nq, H, d = q_shape = q.shape
    ks = _rows("k", k, dev, dtype)
    k_shape = k.shape
    _, Nkv, Hkv, _ = k_shape
    if k_shape[0] != B or k_shape[3] != d:
        raise ValueError("inconsistent q/k shapes")
    vs = _rows("v", v, dev, dtype, k_shape)
    if scale is None:
        scale = 0.0
    elif not (1e-37 < scale < 1e38):  # (0 in 32 bits asks for the default)
        raise ValueError("scale must be positive and finite in 32 bits")
    fields = (B, H, Hkv, Nq, Nkv, d, code, min(left, _INT_MAX), min(right, _INT_MAX), min(sinks, _INT_MAX), scale, 0,
              qs[0], qs[2], qs[1], ks[0], ks[2], ks[1], vs[0], vs[2], vs[1])
    return dev, dtype, q_shape, k_shape, fields


def _lse_of(lse, dev, shape):
    if (not isinstance(lse, torch.Tensor) or lse.dtype is not torch.float32 or lse.device != dev or
            lse.shape != shape or not lse.is_contiguous()):
        raise TypeError("lse must be a contiguous float32 tensor of shape %s on %s" % (shape, dev))
    return lse


@functools.lru_cache(maxsize=1024)
def _need(s: bytes, backward: int) -> int:
    """Bytes of workspace for packed shapes (a function of the sizes alone)."""
    need = ctypes.c_size_t()
    _check(_lib.bsa_window_workspace(s, backward, ctypes.byref(need)))
    return need.value


def _workspace(s, backward, workspace, device):
    """(address, bytes, the tensor)"""
    n = _need(s, backward)
    if n == 0:
        return None, 0, None
    if workspace is None:
        workspace = torch.empty(n, dtype=torch.uint8, device=device)
        return workspace.data_ptr(), n, workspace
    if not isinstance(workspace, torch.Tensor) or workspace.device != device or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor on %s" % device)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def window_workspace(q, k, v, left: int, right: int = 0, sinks: int = 0, *, backward: bool = False) -> int:
    """Bytes of device workspace that window_forward or window_backward needs for
    these tensors, for callers that pass their own."""
    return _need(_pack_window(*_window_head(q, k, v, left, right, sinks, None)[4], 0, 0, 0), 1 if backward else 0)


def window_forward(q, k, v, left: int, right: int = 0, sinks: int = 0, *, scale: Optional[float] = None, q_len=None,
                   kv_len=None, o=None, lse=None, workspace=None, stream=None) -> Tuple:
    """Attention over a sliding window and a few first tokens (bsa_window_forward).

    q is [B, Nq, H, d], k and v [B, Nkv, Hkv, d] in bfloat16 or float16, d 64 or
    128, H a multiple of Hkv.  Query i of a sequence lies at p = i + kv_len - q_len
    and sees the keys p - left .. p + right (ALL or -1: no bound) and of the
    first `sinks` keys those up to p + right.  q_len and kv_len are int32 [B] on
    the device (default: Nq, Nkv).  Returns (o, lse), lse float32 [B, H, Nq]; a
    query that sees nothing gets o = 0 and lse = -inf.  Rows of a given o and
    lse from q_len on keep what they held; allocated ones hold zeros there.
    o and lse carry no gradients: autograd does not record the call, and
    window_backward returns them."""
    dev, dtype, q_shape, _, fields = _window_head(q, k, v, left, right, sinks, scale)
    if q.requires_grad or k.requires_grad or v.requires_grad:
        _not_recorded("window_forward", "window_backward")
    B, Nq, H, _ = q_shape
    ql, kl = _ints("q_len", q_len, dev, B), _ints("kv_len", kv_len, dev, B)

    def call(handle):
        nonlocal o, lse
        new = torch.empty if q_len is None else torch.zeros
        if o is None:
            o = new(q_shape, dtype=dtype, device=dev)
        if lse is None:
            lse = new((B, H, Nq), dtype=torch.float32, device=dev)
        os, _ = _rows("o", o, dev, dtype, q_shape), _lse_of(lse, dev, (B, H, Nq))
        s = _pack_window(*fields, os[0], os[2], os[1])
        ws, n, _keep = _workspace(s, 0, workspace, dev)
        _check(_lib.bsa_window_forward(s, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), ql,
                                       kl, ws, n, handle))

    _run(dev, stream, call)
    return o, lse


def window_backward(q, k, v, o, lse, do, left: int, right: int = 0, sinks: int = 0, *, scale: Optional[float] = None,
                    q_len=None, kv_len=None, dq=None, dk=None, dv=None, workspace=None, stream=None) -> Tuple:
    """Gradients (dq, dk, dv) of window_forward for the gradient `do` of o
    (bsa_window_backward), with the o and lse that it returned and its other
    arguments unchanged.  Rows of given dq from q_len on, and of dk and dv from
    kv_len on, keep what they held; allocated ones hold zeros there.  The
    gradients carry none of their own."""
    dev, dtype, q_shape, k_shape, fields = _window_head(q, k, v, left, right, sinks, scale)
    B, Nq, H, _ = q_shape
    os, gs = _rows("o", o, dev, dtype, q_shape), _rows("do", do, dev, dtype, q_shape)
    _lse_of(lse, dev, (B, H, Nq))
    ql, kl = _ints("q_len", q_len, dev, B), _ints("kv_len", kv_len, dev, B)

    def call(handle):
        nonlocal dq, dk, dv
        if dq is None:
            dq = (torch.empty if q_len is None else torch.zeros)(q_shape, dtype=dtype, device=dev)
        new = torch.empty if kv_len is None else torch.zeros
        if dk is None:
            dk = new(k_shape, dtype=dtype, device=dev)
        if dv is None:
            dv = new(k_shape, dtype=dtype, device=dev)
        dqs = _rows("dq", dq, dev, dtype, q_shape)
        dks, dvs = _rows("dk", dk, dev, dtype, k_shape), _rows("dv", dv, dev, dtype, k_shape)
        s = _pack_window(*fields, os[0], os[2], os[1])
        g = _pack_grads(gs[0], gs[2], gs[1], dqs[0], dqs[2], dqs[1], dks[0], dks[2], dks[1], dvs[0], dvs[2], dvs[1])
        ws, n, _keep = _workspace(s, 1, workspace, dev)
        _check(_lib.bsa_window_backward(s, g, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                        do.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ql, kl, ws, n,
                                        handle))

    _run(dev, stream, call)
    return dq, dk, dv
