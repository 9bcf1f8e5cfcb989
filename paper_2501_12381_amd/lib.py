"""ctypes binding of libgspn.so: the C ABI declared in include/gspn.h.

Functions here have the C names and take plain integers for pointers and the
stream; `paper_2501_12381_amd.ops` wraps them for torch tensors.  Loading fails
loudly if the library has not been built: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libgspn.so")

GSPN_F32, GSPN_BF16 = 0, 1
GSPN_DIR_T2B, GSPN_DIR_B2T, GSPN_DIR_L2R, GSPN_DIR_R2L = 1, 2, 4, 8
GSPN_ALGO_AUTO, GSPN_ALGO_RESIDENT, GSPN_ALGO_STREAM, GSPN_ALGO_RESIDENT_GENERIC = 0, 1, 2, 3
GSPN_ALGO_TWO_PASS = 4
GSPN_FLAG_W_LOGITS, GSPN_FLAG_EDGE_RENORM, GSPN_FLAG_LAM_PER_DIR = 1, 2, 4
GSPN_FLAG_U_PER_DIR, GSPN_FLAG_Y_PER_DIR, GSPN_FLAG_SAVE_STATE = 8, 16, 32
GSPN_MAX_LINE = 4096
GSPN_LINATTN_DECAY_PER_TOKEN = 1
GSPN_ACT_NONE, GSPN_ACT_SILU, GSPN_ACT_GELU = 0, 1, 2
STATUS = {0: "GSPN_OK", 1: "GSPN_ERR_NULL", 2: "GSPN_ERR_SHAPE", 3: "GSPN_ERR_MASK",
          4: "GSPN_ERR_DTYPE", 5: "GSPN_ERR_ALIGN", 6: "GSPN_ERR_ALIAS",
          7: "GSPN_ERR_UNSUPPORTED", 8: "GSPN_ERR_WORKSPACE", 9: "GSPN_ERR_HIP"}

# every symbol include/gspn.h declares
EXPORTS = ("gspn_scan_fwd_workspace_bytes", "gspn_scan_fwd", "gspn_scan_fwd_noalloc",
           "gspn_scan_bwd_workspace_bytes", "gspn_scan_bwd", "gspn_linattn_fwd_workspace_bytes",
           "gspn_linattn_fwd", "gspn_linattn_bwd_workspace_bytes", "gspn_linattn_bwd", "gspn_linattn_step",
           "gspn_group_norm_fwd_workspace_bytes", "gspn_group_norm_fwd", "gspn_group_norm_bwd_workspace_bytes",
           "gspn_group_norm_bwd", "gspn_copy_calibration", "gspn_strerror", "gspn_version")
GSPN_NOALLOC_SCRATCH_BYTES = 64 << 20

_lib = None

_p, _i64, _u32, _i, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint32, ctypes.c_int,
                           ctypes.c_size_t)
_f = ctypes.c_float


class GSPNError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({gspn_strerror(status)})")


def load() -> ctypes.CDLL:
    """Load libgspn.so (once).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2501_12381_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    ws_args = [_i64, _i64, _i64, _i64, _u32, _i, _i64, _i64, _u32, _i]
    lib.gspn_scan_fwd_workspace_bytes.argtypes = ws_args
    lib.gspn_scan_fwd_workspace_bytes.restype = _sz
    lib.gspn_scan_bwd_workspace_bytes.argtypes = ws_args
    lib.gspn_scan_bwd_workspace_bytes.restype = _sz
    lib.gspn_scan_fwd.argtypes = [_p, _p, _p, _p, _p, _i64, _i64, _i64, _i64, _u32, _i, _i64, _i64, _u32,
                                  _i, _p, _sz, _p]
    lib.gspn_scan_fwd.restype = _i
    lib.gspn_scan_fwd_noalloc.argtypes = [_p, _p, _p, _p, _p, _i64, _i64, _i64, _i64, _u32, _i, _i64, _i64,
                                          _u32, _p]
    lib.gspn_scan_fwd_noalloc.restype = _i
    lib.gspn_scan_bwd.argtypes = [_p, _p, _p, _p, _p, _p, _p, _p, _p, _i64, _i64, _i64, _i64, _u32,
                                  _i, _i64, _i64, _u32, _i, _p, _sz, _p]
    lib.gspn_scan_bwd.restype = _i
    for fn in (lib.gspn_linattn_fwd_workspace_bytes, lib.gspn_linattn_bwd_workspace_bytes):
        fn.argtypes = [_i64] * 7 + [_i, _i, _u32]
        fn.restype = _sz
    lib.gspn_linattn_fwd.argtypes = [_p] * 8 + [_i64] * 7 + [_p, _i, _u32, _f, _p, _sz, _p]
    lib.gspn_linattn_bwd.argtypes = [_p] * 13 + [_i64] * 7 + [_p, _i, _u32, _f, _p, _p, _sz, _p]
    lib.gspn_linattn_step.argtypes = [_p] * 7 + [_i64] * 6 + [_p, _i, _u32, _f, _p]
    for fn in (lib.gspn_group_norm_fwd_workspace_bytes, lib.gspn_group_norm_bwd_workspace_bytes):
        fn.argtypes = [_i64] * 4 + [_i]
        fn.restype = _sz
    lib.gspn_group_norm_fwd.argtypes = [_p] * 6 + [_i64] * 4 + [_f, _i, _i, _p, _sz, _p]
    lib.gspn_group_norm_bwd.argtypes = [_p] * 9 + [_i64] * 4 + [_i, _i, _p, _sz, _p]
    for fn in (lib.gspn_linattn_fwd, lib.gspn_linattn_bwd, lib.gspn_linattn_step, lib.gspn_group_norm_fwd,
               lib.gspn_group_norm_bwd):
        fn.restype = _i
    lib.gspn_copy_calibration.argtypes = [_p, _p, _sz, _p]
    lib.gspn_copy_calibration.restype = _i
    lib.gspn_strerror.argtypes = [_i]
    lib.gspn_strerror.restype = ctypes.c_char_p
    lib.gspn_version.argtypes = []
    lib.gspn_version.restype = _i
    _lib = lib
    return lib


def gspn_scan_fwd_workspace_bytes(B, C, H, W, mask, dtype, group_h=0, group_w=0, flags=0,
                                  algo=GSPN_ALGO_AUTO) -> int:
    return int(load().gspn_scan_fwd_workspace_bytes(B, C, H, W, mask, dtype, group_h, group_w, flags,
                                                    algo))


def gspn_scan_bwd_workspace_bytes(B, C, H, W, mask, dtype, group_h=0, group_w=0, flags=0,
                                  algo=GSPN_ALGO_AUTO) -> int:
    return int(load().gspn_scan_bwd_workspace_bytes(B, C, H, W, mask, dtype, group_h, group_w, flags,
                                                    algo))


def gspn_scan_fwd(x, w, lam, u, y, B, C, H, W, mask, dtype, group_h, group_w, flags, algo, workspace,
                  workspace_bytes, stream) -> int:
    return int(load().gspn_scan_fwd(x, w, lam, u, y, B, C, H, W, mask, dtype, group_h, group_w, flags,
                                    algo, workspace, workspace_bytes, stream))


def gspn_scan_fwd_noalloc(x, w, lam, u, y, B, C, H, W, mask, dtype, group_h, group_w, flags,
                          stream) -> int:
    return int(load().gspn_scan_fwd_noalloc(x, w, lam, u, y, B, C, H, W, mask, dtype, group_h, group_w,
                                            flags, stream))


def gspn_scan_bwd(dy, x, w, lam, u, dx, dw, dlam, du, B, C, H, W, mask, dtype, group_h, group_w, flags,
                  algo, workspace, workspace_bytes, stream) -> int:
    return int(load().gspn_scan_bwd(dy, x, w, lam, u, dx, dw, dlam, du, B, C, H, W, mask, dtype,
                                    group_h, group_w, flags, algo, workspace, workspace_bytes, stream))


def gspn_linattn_fwd_workspace_bytes(n_seq, B, T, H, Hk, Dk, Dv, packed, dtype, flags=0) -> int:
    return int(load().gspn_linattn_fwd_workspace_bytes(n_seq, B, T, H, Hk, Dk, Dv, packed, dtype, flags))


def gspn_linattn_bwd_workspace_bytes(n_seq, B, T, H, Hk, Dk, Dv, packed, dtype, flags=0) -> int:
    return int(load().gspn_linattn_bwd_workspace_bytes(n_seq, B, T, H, Hk, Dk, Dv, packed, dtype, flags))


def gspn_linattn_fwd(q, k, v, log_decay, initial_state, cu_seqlens, o, final_state, n_seq, B, T, H, Hk, Dk, Dv,
                     strides, dtype, flags, scale, workspace, workspace_bytes, stream) -> int:
    return int(load().gspn_linattn_fwd(q, k, v, log_decay, initial_state, cu_seqlens, o, final_state, n_seq, B, T,
                                       H, Hk, Dk, Dv, strides, dtype, flags, scale, workspace, workspace_bytes,
                                       stream))


def gspn_linattn_bwd(dout, q, k, v, log_decay, initial_state, dfinal_state, cu_seqlens, dq, dk, dv, dlog_decay,
                     dinitial_state, n_seq, B, T, H, Hk, Dk, Dv, strides, dtype, flags, scale, forward_workspace,
                     workspace, workspace_bytes, stream) -> int:
    return int(load().gspn_linattn_bwd(dout, q, k, v, log_decay, initial_state, dfinal_state, cu_seqlens, dq, dk,
                                       dv, dlog_decay, dinitial_state, n_seq, B, T, H, Hk, Dk, Dv, strides, dtype,
                                       flags, scale, forward_workspace, workspace, workspace_bytes, stream))


def gspn_linattn_step(q, k, v, log_decay, state, slots, o, n_slots, B, H, Hk, Dk, Dv, strides, dtype, flags, scale,
                      stream) -> int:
    return int(load().gspn_linattn_step(q, k, v, log_decay, state, slots, o, n_slots, B, H, Hk, Dk, Dv, strides,
                                        dtype, flags, scale, stream))


def gspn_group_norm_fwd_workspace_bytes(B, L, C, G, dtype) -> int:
    return int(load().gspn_group_norm_fwd_workspace_bytes(B, L, C, G, dtype))


def gspn_group_norm_bwd_workspace_bytes(B, L, C, G, dtype) -> int:
    return int(load().gspn_group_norm_bwd_workspace_bytes(B, L, C, G, dtype))


def gspn_group_norm_fwd(x, weight, bias, y, mean, rstd, B, L, C, G, eps, act, dtype, workspace, workspace_bytes,
                        stream) -> int:
    return int(load().gspn_group_norm_fwd(x, weight, bias, y, mean, rstd, B, L, C, G, eps, act, dtype, workspace,
                                          workspace_bytes, stream))


def gspn_group_norm_bwd(dy, x, weight, bias, mean, rstd, dx, dweight, dbias, B, L, C, G, act, dtype, workspace,
                        workspace_bytes, stream) -> int:
    return int(load().gspn_group_norm_bwd(dy, x, weight, bias, mean, rstd, dx, dweight, dbias, B, L, C, G, act,
                                          dtype, workspace, workspace_bytes, stream))


def gspn_copy_calibration(src, dst, nbytes, stream) -> int:
    return int(load().gspn_copy_calibration(src, dst, nbytes, stream))


def gspn_strerror(status: int) -> str:
    return load().gspn_strerror(status).decode()


def gspn_version() -> int:
    return int(load().gspn_version())
