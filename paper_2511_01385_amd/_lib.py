"""ctypes view of ``librdfft.so``: the C ABI of include/rdfft.h, names unchanged.

Argument marshalling only.  Loading fails loudly when the library is missing; there
is no fallback implementation.
"""

from __future__ import annotations

import ctypes
import os
import struct

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librdfft.so")

RDFFT_F32 = 0
RDFFT_BF16 = 1
RDFFT_F16 = 2

RDFFT_ACT_NONE = 0
RDFFT_ACT_RELU = 1
RDFFT_ACT_GELU = 2
RDFFT_ACT_SILU = 3

RDFFT_OK = 0
RDFFT_EINVAL = -1
RDFFT_EUNSUPPORTED = -2
RDFFT_ELAUNCH = -3
RDFFT_EDEVICE = -4

# every entry point include/rdfft.h declares
EXPORTS = (
    "rdfft_forward",
    "rdfft_inverse",
    "rdfft_pairs_to_halfcomplex",
    "rdfft_halfcomplex_to_pairs",
    "rdfft_forward_halfcomplex",
    "rdfft_inverse_halfcomplex",
    "bca_forward",
    "bca_backward",
    "bca_backward_keep",
    "bca_forward_batched",
    "bca_backward_batched",
    "act8_quantize",
    "act8_dequantize",
    "layer_norm_forward",
    "layer_norm_backward_workspace",
    "layer_norm_backward",
    "linear_forward_workspace",
    "linear_forward",
    "linear_backward_workspace",
    "linear_backward",
    "fp8_quantize",
    "fp8_dequantize",
    "rms_norm_forward",
    "rms_norm_backward_workspace",
    "rms_norm_backward",
    "linear_fp8_forward_workspace",
    "linear_fp8_forward",
    "linear_fp8_backward_workspace",
    "linear_fp8_backward",
    "rdfft_init",
    "rdfft_table_bytes",
    "rdfft_status_string",
)


class BcaGrads(ctypes.Structure):
    """bca_grads_t"""

    _fields_ = [("dx", ctypes.c_void_p), ("dc", ctypes.c_void_p)]


# The argument structs of the operators around the adapter, every field of which is a pointer or an
# int64, as packers of their fields in order (a third of a ctypes.Structure's time).
_FIELDS = {
    "act8": "codes scales",
    "layer_norm_forward": "x ldx residual ldr weight bias y ldy mean rstd codes scales",
    "layer_norm_backward": "dy ldg x ldx residual ldr codes scales weight mean rstd dx ldd dweight dbias workspace "
                           "workspace_bytes",
    "linear_forward": "x ldx w ldw bias residual ldr y ldy codes scales workspace workspace_bytes",
    "linear_backward": "dy ldg codes scales x ldx w ldw add lda dx ldd dw lddw db workspace workspace_bytes",
    "fp8": "codes ld scales lds block_rows",
    "rms_norm_forward": "x ldx residual ldr weight y ldy summed lds rstd codes scales codes8 ld8 scales8 lds8 block_rows8",
    "rms_norm_backward": "dy ldg u ldu codes scales weight rstd add lda dx ldd dweight workspace workspace_bytes",
    "linear_fp8_forward": "x ldx x_scales ldxs x_block_rows w ldw w_scales ldws w_block_rows bias residual ldr y ldy codes "
                          "scales workspace workspace_bytes",
    "linear_fp8_backward": "dy ldg codes scales x ldx x_scales ldxs x_block_rows w ldw w_scales ldws w_block_rows add lda dx "
                           "ldd dw lddw db workspace workspace_bytes",
}
pack = {name: struct.Struct(f"{len(fields.split())}q").pack for name, fields in _FIELDS.items()}

_lib = None


def load() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run paper_2511_01385_amd.build.build() first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    for name in ("rdfft_forward", "rdfft_inverse", "rdfft_pairs_to_halfcomplex", "rdfft_halfcomplex_to_pairs",
                 "rdfft_forward_halfcomplex", "rdfft_inverse_halfcomplex"):
        f = getattr(lib, name)
        f.argtypes = [vp, i64, i64, i32, vp]
        f.restype = i32
    for name in ("bca_forward", "bca_backward", "bca_backward_keep"):
        f = getattr(lib, name)
        f.argtypes = [vp, vp, vp, ctypes.POINTER(BcaGrads), i64, i64, i64, i64, i32, vp]
        f.restype = i32
    pp = ctypes.POINTER(ctypes.c_void_p)
    lib.bca_forward_batched.argtypes = [i32, pp, pp, pp, i64, i64, i64, i64, i32, vp]
    lib.bca_forward_batched.restype = i32
    lib.bca_backward_batched.argtypes = [i32, pp, pp, pp, ctypes.POINTER(BcaGrads), i64, i64, i64, i64, i32, vp]
    lib.bca_backward_batched.restype = i32
    f32 = ctypes.c_float
    # (the structs come as bytes, see pack)
    lib.act8_quantize.argtypes = [vp, i64, vp, i64, i64, i32, vp]
    lib.act8_dequantize.argtypes = [vp, vp, i64, i64, i64, i32, vp]
    lib.layer_norm_forward.argtypes = [vp, i64, i64, f32, i32, vp]
    lib.layer_norm_backward.argtypes = [vp, i64, i64, i32, vp]
    lib.linear_forward.argtypes = [vp, i64, i64, i64, i32, i32, vp]
    lib.linear_backward.argtypes = [vp, i64, i64, i64, i32, i32, vp]
    lib.fp8_quantize.argtypes = [vp, i64, vp, vp, i64, i64, i32, vp]
    lib.fp8_dequantize.argtypes = [vp, vp, i64, i64, i64, i32, vp]
    lib.rms_norm_forward.argtypes = [vp, i64, i64, f32, i32, vp]
    lib.rms_norm_backward.argtypes = [vp, i64, i64, i32, vp]
    lib.linear_fp8_forward.argtypes = [vp, i64, i64, i64, i32, i32, vp]
    lib.linear_fp8_backward.argtypes = [vp, i64, i64, i64, i32, i32, vp]
    for name in ("act8_quantize", "act8_dequantize", "layer_norm_forward", "layer_norm_backward", "linear_forward",
                 "linear_backward", "fp8_quantize", "fp8_dequantize", "rms_norm_forward", "rms_norm_backward",
                 "linear_fp8_forward", "linear_fp8_backward"):
        getattr(lib, name).restype = i32
    lib.layer_norm_backward_workspace.argtypes = [i64, i64]
    lib.linear_forward_workspace.argtypes = [i64, i64, i64, i32]
    lib.linear_backward_workspace.argtypes = [i64, i64, i64, i32, i32, i32, i32, i32]
    lib.rms_norm_backward_workspace.argtypes = [i64, i64]
    lib.linear_fp8_forward_workspace.argtypes = [i64, i64, i64, i32]
    lib.linear_fp8_backward_workspace.argtypes = [i64, i64, i64, i32, i32, i32, i32]
    for name in ("layer_norm_backward_workspace", "linear_forward_workspace", "linear_backward_workspace",
                 "rms_norm_backward_workspace", "linear_fp8_forward_workspace", "linear_fp8_backward_workspace"):
        getattr(lib, name).restype = i64
    lib.rdfft_init.argtypes = []
    lib.rdfft_init.restype = i32
    lib.rdfft_table_bytes.argtypes = []
    lib.rdfft_table_bytes.restype = i64
    lib.rdfft_status_string.argtypes = [i32]
    lib.rdfft_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


_binding = None


def binding():
    """The native module that takes torch tensors (csrc/binding.cpp); it calls the same library."""
    global _binding
    if _binding is None:
        load()
        import torch  # noqa: F401  (whose libraries the module needs)

        try:
            from . import _binding as module
        except ImportError as e:
            raise ImportError(f"the _binding module is not built ({e}); run paper_2511_01385_amd.build.build() first") from e
        _binding = module
    return _binding


def status_string(status: int) -> str:
    return load().rdfft_status_string(status).decode()
