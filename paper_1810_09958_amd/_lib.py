"""Loader for the in-tree ``libisam.so`` and ctypes signatures of the C ABI (include/isam.h)."""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
ISAM_F32, ISAM_BF16 = 0, 1

# name -> (restype, argtypes), mirroring include/isam.h
i64, vp, sz, ci, cf = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
row = (vp, i64, i64)  # rows of a [T][batch] tensor: pointer and two strides
SIGNATURES = {
    "isam_gemm": (ci, [ci, ci, i64, i64, i64, ci, vp, i64, vp, i64, ci, ci, vp, i64, vp, sz, vp]),
    "isam_gemm_workspace_size": (sz, [ci, ci, i64, i64, i64, ci, ci]),
    "isam_dwsep_conv": (ci, [i64] * 10 + [ci, vp, vp, vp, ci, vp, vp, sz, vp]),
    "isam_dwsep_conv_workspace_size": (sz, [i64] * 10 + [ci, ci]),
    "isam_gru_forward": (ci, [i64, i64, i64, i64, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
    "isam_gru_forward_workspace_size": (sz, [i64, i64, i64, i64, ci]),
    "isam_gru_forward_noalloc": (ci, [i64, i64, i64, i64, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
    "isam_conv1d": (ci, [i64, i64, i64, i64, i64, ci, vp, vp, ci, ci, vp, vp]),
    "isam_linear_gru": (ci, [i64, i64, i64, ci, ci, vp, i64, i64, vp, vp, vp, i64, i64, vp, i64, i64, vp, vp, vp, sz, vp]),
    "isam_linear_gru_workspace_size": (sz, [i64, i64, i64, ci]),
    "isam_linear_gru_backward": (ci, [i64, i64, i64, ci, ci, vp, i64, i64, vp, vp, i64, i64, vp, vp, i64, i64, vp, vp, i64,
                                      i64, vp, vp, vp, sz, vp]),
    "isam_linear_gru_backward_workspace_size": (sz, [i64, i64, i64, ci]),
    "isam_norm_residual": (ci, [i64, i64, i64, ci, vp, i64, vp, i64, vp, vp, vp, cf, cf, vp, i64, vp, i64, vp]),
    "isam_norm_residual_backward": (ci, [i64, i64, i64, ci, vp, i64, vp, i64, vp, vp, vp, cf, cf, vp, i64, vp, i64, vp, i64,
                                         vp, i64, vp, vp, vp, vp, sz, vp]),
    "isam_norm_residual_backward_workspace_size": (sz, [i64, i64, i64, ci]),
    "isam_gated_ffn": (ci, [i64, i64, i64, ci, ci, vp, i64, vp, i64, vp, vp, i64, vp, sz, vp]),
    "isam_gated_ffn_workspace_size": (sz, [i64, i64, i64, ci, ci]),
    "isam_gated_ffn_backward": (ci, [i64, i64, i64, ci, ci, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]),
    "isam_gated_ffn_backward_workspace_size": (sz, [i64, i64, i64, ci, ci]),
    "isam_selective_scan": (ci, [i64] * 4 + [ci, *row, *row, vp, *row, *row, vp, *row, vp, vp, *row, *row, vp, vp, vp, sz, vp]),
    "isam_selective_scan_workspace_size": (sz, [i64] * 4 + [ci]),
    "isam_selective_scan_backward": (ci, [i64] * 4 + [ci, *row, *row, vp, *row, *row, vp, *row, vp, *row, vp, *row, vp, *row, *row, vp,
                                          *row, *row, vp, *row, vp, vp, vp, sz, vp]),
    "isam_selective_scan_backward_workspace_size": (sz, [i64] * 4 + [ci]),
    "isam_causal_conv": (ci, [i64] * 4 + [ci, ci, *row, vp, vp, vp, *row, *row, vp, vp]),
    "isam_causal_conv_backward": (ci, [i64] * 4 + [ci, ci, *row, vp, vp, vp, *row, *row, vp, *row, vp, vp, vp, vp, sz, vp]),
    "isam_causal_conv_backward_workspace_size": (sz, [i64] * 4 + [ci]),
    "isam_beam_step": (ci, [i64] * 4 + [ci, *row, vp, vp, i64, vp, vp, vp, vp, vp, sz, vp]),
    "isam_beam_step_workspace_size": (sz, [i64] * 4 + [ci]),
    "isam_beam_reorder": (ci, [i64] * 5 + [vp, vp, vp, vp]),
    "isam_linear": (ci, [i64] * 3 + [ci, ci, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, sz, vp]),
    "isam_linear_workspace_size": (sz, [i64] * 3 + [ci, ci]),
    "isam_linear_backward": (ci, [i64] * 3 + [ci, ci, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]),
    "isam_linear_backward_workspace_size": (sz, [i64] * 3 + [ci, ci]),
    "isam_status_string": (ctypes.c_char_p, [ci]),
    "isam_last_error": (ctypes.c_char_p, []),
    "isam_version": (ci, []),
}


class IsamError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(msg)
        self.status = status


def lib_path() -> str:
    """The in-tree libisam.so, or the file ISAM_LIB names (e.g. the sanitizer build)."""
    return os.environ.get("ISAM_LIB") or os.path.join(HERE, "libisam.so")


_lib = None


def lib():
    """Load libisam.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with `python -m paper_1810_09958_amd.build`")
        L = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib
