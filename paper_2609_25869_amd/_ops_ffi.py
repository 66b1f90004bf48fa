"""ctypes declarations of libbsa_ops.so (the C-ABI in include/bsa_ops.h).

Argument marshalling only.  Importing this module fails loudly when the
library has not been built.
"""
from __future__ import annotations

import ctypes
import os

from ._ffi import HERE, c_i32, c_i64, c_sz, c_vp

LIB_PATH = os.path.join(HERE, "libbsa_ops.so")

_Stride = c_i64 * 3


class RopeShapes(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("heads", c_i32), ("kv_heads", c_i32), ("seq", c_i32), ("head_dim", c_i32),
                ("dtype", c_i32), ("pairs", c_i32 * 3), ("interleaved", c_i32), ("inverse", c_i32),
                ("grid", c_i32 * 3), ("origin", c_i32 * 3), ("kv_rows", c_i32), ("pos_stride", c_i64 * 2),
                ("q_stride", _Stride), ("k_stride", _Stride), ("v_stride", _Stride),
                ("q_out_stride", _Stride), ("k_out_stride", _Stride), ("v_out_stride", _Stride)]


class WindowShapes(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("heads", c_i32), ("kv_heads", c_i32), ("seq_q", c_i32), ("seq_kv", c_i32),
                ("head_dim", c_i32), ("dtype", c_i32), ("left", c_i32), ("right", c_i32), ("sinks", c_i32),
                ("scale", ctypes.c_float), ("reserved", c_i32),
                ("q_stride", _Stride), ("k_stride", _Stride), ("v_stride", _Stride), ("o_stride", _Stride)]


class WindowGrads(ctypes.Structure):
    _fields_ = [("do_stride", _Stride), ("dq_stride", _Stride), ("dk_stride", _Stride), ("dv_stride", _Stride)]


# (name, restype, argtypes) of every exported entry point; the shape structures
# go by address: byref() of one of the above, or the same bytes
SIGNATURES = [
    ("bsa_ops_last_error", ctypes.c_char_p, []),
    ("bsa_rope", c_i32, [c_vp] * 12),
    ("bsa_window_workspace", c_i32, [c_vp, c_i32, ctypes.POINTER(c_sz)]),
    ("bsa_window_forward", c_i32, [c_vp] * 9 + [c_sz, c_vp]),
    ("bsa_window_backward", c_i32, [c_vp] * 14 + [c_sz, c_vp]),
]


# The same layouts for struct.pack (no field is padded).
ROPE_PACK = "=18i20q"
WINDOW_PACK = "=10ifi12q"
GRADS_PACK = "=12q"


def load() -> ctypes.CDLL:
    # torch's HIP runtime first: pointers and streams must come from one runtime
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    if not os.path.exists(LIB_PATH):
        raise ImportError("libbsa_ops.so is not built at %s; run `python paper_2609_25869_amd/build.py`" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    for name, res, args in SIGNATURES:
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib
