"""ctypes binding of libeqlinear.so: the C ABI of include/eqlinear.h, eqlinear_block.h, eqlinear_encoder.h and
eqlinear_recurrent.h, same names.

Argument marshalling only.  Every function takes device addresses as Python
ints (or None for NULL) and returns the library's status code; ``check``
turns a non-zero status into an ``EqlError``.  Loading fails loudly when the
library has not been built: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libeqlinear.so")

EQL_F32 = 0
EQL_F16 = 1
EQL_BF16 = 2

EQL_OK = 0
EQL_ERR_INVALID_ARG = 1
EQL_ERR_UNSUPPORTED = 2
EQL_ERR_ALIGNMENT = 3
EQL_ERR_WORKSPACE = 4
EQL_ERR_NO_DEVICE = 5
EQL_ERR_LAUNCH = 6
EQL_ERR_SCRATCH = 7

# Bytes of the static device scratch of eqlinear_backward_weight_noalloc
# (EQLINEAR_STATIC_SCRATCH_BYTES in include/eqlinear.h).
STATIC_SCRATCH_BYTES = 64 << 20

EQL_ACT_NONE = 0
EQL_ACT_RELU = 1
EQL_ACT_SILU = 2
EQL_ACT_GELU = 3

EQL_NORM_LAYER = 0
EQL_NORM_RMS = 1

_vp, _i, _i64, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_f = ctypes.c_float


class RotaryShape(ctypes.Structure):
    """eqlinear_rotary_shape of include/eqlinear_encoder.h."""
    _fields_ = [("B", _i64), ("L", _i64), ("heads", _i), ("dh", _i), ("T", _i), ("axes", _i), ("sections", _i * 4),
                ("float_positions", _i), ("interleaved", _i), ("inverse", _i), ("dtype", _i), ("x_stride", _i64 * 3),
                ("y_stride", _i64 * 3), ("pos_stride", _i64 * 2)]


class WindowShape(ctypes.Structure):
    """eqlinear_window_shape of include/eqlinear_encoder.h."""
    _fields_ = [("B", _i64), ("Lq", _i64), ("Lk", _i64), ("left", _i64), ("right", _i64), ("sinks", _i64),
                ("heads", _i), ("kv_heads", _i), ("head_dim", _i), ("dtype", _i), ("scale", _f), ("reserved", _i)] + [
                    (n + "_stride", _i64 * 3) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")]


class ScanShape(ctypes.Structure):
    """eqlinear_scan_shape of include/eqlinear_recurrent.h."""
    _fields_ = [("B", _i64), ("L", _i64), ("C", _i), ("T", _i), ("N", _i), ("groups", _i), ("softplus", _i), ("dtype", _i),
                ("x_stride", _i64 * 2), ("delta_stride", _i64 * 2), ("z_stride", _i64 * 2), ("b_stride", _i64 * 3),
                ("c_stride", _i64 * 3)]


class ConvShape(ctypes.Structure):
    """eqlinear_conv_shape of include/eqlinear_recurrent.h."""
    _fields_ = [("B", _i64), ("L", _i64), ("C", _i), ("T", _i), ("W", _i), ("act", _i), ("dtype", _i), ("reserved", _i),
                ("x_stride", _i64 * 2)]


class ResidualShape(ctypes.Structure):
    """eqlinear_residual_shape of include/eqlinear_recurrent.h."""
    _fields_ = [("B", _i64), ("L", _i64), ("C", _i), ("T", _i), ("kind", _i), ("dtype", _i), ("eps", _f), ("reserved", _i)]


# Every function the headers declare, with (restype, argtypes).
_RS, _WS = ctypes.POINTER(RotaryShape), ctypes.POINTER(WindowShape)
_SS, _CS, _NS = ctypes.POINTER(ScanShape), ctypes.POINTER(ConvShape), ctypes.POINTER(ResidualShape)
SIGNATURES = {
    "eqlinear_abi_version": (_i, []),
    "eqlinear_status_string": (ctypes.c_char_p, [_i]),
    "eqlinear_weight_spectrum_bytes": (_sz, [_i, _i, _i, _i]),
    "eqlinear_weight_spectrum": (_i, [_vp, _vp, _i, _i, _i, _i, _vp]),
    "eqlinear_forward": (_i, [_vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp]),
    "eqlinear_backward_input": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp]),
    "eqlinear_backward_weight_workspace_bytes": (_sz, [_i64, _i, _i, _i, _i]),
    "eqlinear_backward_weight": (_i, [_vp, _vp, _vp, _vp, _vp, _sz, _i64, _i, _i, _i, _i, _vp]),
    "eqlinear_backward_weight_noalloc": (_i, [_vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp]),
    "eqlinear_backward_workspace_bytes": (_sz, [_i64, _i, _i, _i, _i]),
    "eqlinear_backward_is_fused": (_i, [_i64, _i, _i, _i, _i]),
    "eqlinear_backward": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _i64, _i, _i, _i, _i, _vp]),
    "eqlinear_dihedral_expand": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "eqlinear_dihedral_fold": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "eqlinear_gconv_gather": (_i, [_vp, _vp, _i64, _i, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_gconv_scatter": (_i, [_vp, _vp, _i64, _i, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_gconv_pack_weight": (_i, [_vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_gconv_pack_weight_adjoint": (_i, [_vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_gconv_unpack_weight": (_i, [_vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_gconv_forward": (_i, [_vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_group_norm": (_i, [_vp, _vp, _vp, _vp, _i64, _i, _i, ctypes.c_float, _i, _vp]),
    "eqlinear_attention": (_i, [_vp, _vp, _i64, _i, _i, _i, ctypes.c_float, _i, _vp]),
    "eqlinear_rotary": (_i, [_RS, _vp, _vp, _vp, _vp, _vp]),
    "eqlinear_window_attention_workspace_bytes": (_sz, [_WS]),
    "eqlinear_window_attention": (_i, [_WS] + [_vp] * 8 + [_sz, _vp]),
    "eqlinear_window_attention_backward_workspace_bytes": (_sz, [_WS]),
    "eqlinear_window_attention_backward": (_i, [_WS] + [_vp] * 12 + [_sz, _vp]),
    "eqlinear_group_norm_act_workspace_bytes": (_sz, [_i64, _i64, _i, _i, _i, _i]),
    "eqlinear_group_norm_act": (_i, [_vp] * 6 + [_sz, _i64, _i64, _i, _i, _i, _f, _i, _i, _vp]),
    "eqlinear_group_norm_act_backward_workspace_bytes": (_sz, [_i64, _i64, _i, _i, _i, _i]),
    "eqlinear_group_norm_act_backward": (_i, [_vp] * 9 + [_sz, _i64, _i64, _i, _i, _i, _i, _i, _vp]),
    "eqlinear_selective_scan_workspace_bytes": (_sz, [_SS]),
    "eqlinear_selective_scan_states_bytes": (_sz, [_SS]),
    "eqlinear_selective_scan": (_i, [_SS] + [_vp] * 14 + [_sz, _vp]),
    "eqlinear_selective_scan_backward_workspace_bytes": (_sz, [_SS]),
    "eqlinear_selective_scan_backward": (_i, [_SS] + [_vp] * 22 + [_sz, _vp]),
    "eqlinear_causal_conv": (_i, [_CS] + [_vp] * 8),
    "eqlinear_causal_conv_backward_workspace_bytes": (_sz, [_CS]),
    "eqlinear_causal_conv_backward": (_i, [_CS] + [_vp] * 12 + [_sz, _vp]),
    "eqlinear_residual_norm": (_i, [_NS] + [_vp] * 11),
    "eqlinear_residual_norm_backward_workspace_bytes": (_sz, [_NS]),
    "eqlinear_residual_norm_backward": (_i, [_NS] + [_vp] * 18 + [_sz, _vp]),
}


class EqlError(RuntimeError):
    def __init__(self, status: int, where: str = ""):
        self.status = status
        super().__init__("%s: status %d (%s)" % (where or "eqlinear", status, status_string(status)))


_lib = None


def lib(path: str | None = None):
    """Load libeqlinear.so (cached).  Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError("libeqlinear.so is not built (%s); run __graft_entry__.build() or "
                           "python -m paper_2607_21271_amd.build" % p)
    handle = ctypes.CDLL(p)
    for name, (res, args) in SIGNATURES.items():
        f = getattr(handle, name)
        f.restype = res
        f.argtypes = args
    if path is None:
        _lib = handle
    return handle


def status_string(status: int) -> str:
    return lib().eqlinear_status_string(status).decode()


def check(status: int, where: str = "") -> None:
    if status != EQL_OK:
        raise EqlError(status, where)


def eqlinear_abi_version() -> int:
    return lib().eqlinear_abi_version()


def eqlinear_status_string(status: int) -> str:
    return status_string(status)


def eqlinear_weight_spectrum_bytes(T, Cin, Cout, dtype) -> int:
    return lib().eqlinear_weight_spectrum_bytes(T, Cin, Cout, dtype)


def eqlinear_weight_spectrum(w, wspec, T, Cin, Cout, dtype, stream) -> int:
    return lib().eqlinear_weight_spectrum(w, wspec, T, Cin, Cout, dtype, stream)


def eqlinear_forward(x, wspec, bias, y, N, T, Cin, Cout, dtype, stream) -> int:
    return lib().eqlinear_forward(x, wspec, bias, y, N, T, Cin, Cout, dtype, stream)


def eqlinear_backward_input(dy, wspec, dx, N, T, Cin, Cout, dtype, stream) -> int:
    return lib().eqlinear_backward_input(dy, wspec, dx, N, T, Cin, Cout, dtype, stream)


def eqlinear_backward_weight_workspace_bytes(N, T, Cin, Cout, dtype) -> int:
    return lib().eqlinear_backward_weight_workspace_bytes(N, T, Cin, Cout, dtype)


def eqlinear_backward_weight(x, dy, dw, dbias, workspace, workspace_bytes, N, T, Cin, Cout, dtype,
                             stream) -> int:
    return lib().eqlinear_backward_weight(x, dy, dw, dbias, workspace, workspace_bytes, N, T, Cin,
                                          Cout, dtype, stream)


def eqlinear_backward_weight_noalloc(x, dy, dw, dbias, N, T, Cin, Cout, dtype, stream) -> int:
    return lib().eqlinear_backward_weight_noalloc(x, dy, dw, dbias, N, T, Cin, Cout, dtype, stream)


def eqlinear_backward_workspace_bytes(N, T, Cin, Cout, dtype) -> int:
    return lib().eqlinear_backward_workspace_bytes(N, T, Cin, Cout, dtype)


def eqlinear_backward_is_fused(N, T, Cin, Cout, dtype) -> int:
    return lib().eqlinear_backward_is_fused(N, T, Cin, Cout, dtype)


def eqlinear_backward(x, dy, wspec, dx, dw, dbias, workspace, workspace_bytes, N, T, Cin, Cout, dtype,
                      stream) -> int:
    return lib().eqlinear_backward(x, dy, wspec, dx, dw, dbias, workspace, workspace_bytes, N, T, Cin,
                                   Cout, dtype, stream)


def eqlinear_dihedral_expand(w, bias, w_ct, bias_ct, T, Cin, Cout, dtype, stream) -> int:
    return lib().eqlinear_dihedral_expand(w, bias, w_ct, bias_ct, T, Cin, Cout, dtype, stream)


def eqlinear_dihedral_fold(dw_ct, dbias_ct, dw, dbias, T, Cin, Cout, dtype, stream) -> int:
    return lib().eqlinear_dihedral_fold(dw_ct, dbias_ct, dw, dbias, T, Cin, Cout, dtype, stream)


def eqlinear_gconv_gather(f, xcol, B, H, W, T, Cin, k, dtype, stream) -> int:
    return lib().eqlinear_gconv_gather(f, xcol, B, H, W, T, Cin, k, dtype, stream)


def eqlinear_gconv_scatter(dxcol, df, B, H, W, T, Cin, k, dtype, stream) -> int:
    return lib().eqlinear_gconv_scatter(dxcol, df, B, H, W, T, Cin, k, dtype, stream)


def eqlinear_gconv_pack_weight(psi, w_ct, T, Cin, Cout, k, dtype, stream) -> int:
    return lib().eqlinear_gconv_pack_weight(psi, w_ct, T, Cin, Cout, k, dtype, stream)


def eqlinear_gconv_pack_weight_adjoint(psi, w_adj, T, Cin, Cout, k, dtype, stream) -> int:
    return lib().eqlinear_gconv_pack_weight_adjoint(psi, w_adj, T, Cin, Cout, k, dtype, stream)


def eqlinear_gconv_unpack_weight(dw_ct, dpsi, T, Cin, Cout, k, dtype, stream) -> int:
    return lib().eqlinear_gconv_unpack_weight(dw_ct, dpsi, T, Cin, Cout, k, dtype, stream)


def eqlinear_gconv_forward(f, wspec, bias, y, B, H, W, T, Cin, Cout, k, dtype, stream) -> int:
    return lib().eqlinear_gconv_forward(f, wspec, bias, y, B, H, W, T, Cin, Cout, k, dtype, stream)


def eqlinear_group_norm(x, weight, bias, y, rows, T, C, eps, dtype, stream) -> int:
    return lib().eqlinear_group_norm(x, weight, bias, y, rows, T, C, eps, dtype, stream)


def eqlinear_attention(qkv, o, B, L, heads, head_dim, scale, dtype, stream) -> int:
    return lib().eqlinear_attention(qkv, o, B, L, heads, head_dim, scale, dtype, stream)


def eqlinear_rotary(shape, x, positions, freqs, y, stream) -> int:
    return lib().eqlinear_rotary(shape, x, positions, freqs, y, stream)


def eqlinear_window_attention_workspace_bytes(shape) -> int:
    return lib().eqlinear_window_attention_workspace_bytes(shape)


def eqlinear_window_attention(shape, q, k, v, lengths, starts, o, lse, workspace, workspace_bytes, stream) -> int:
    return lib().eqlinear_window_attention(shape, q, k, v, lengths, starts, o, lse, workspace, workspace_bytes, stream)


def eqlinear_window_attention_backward_workspace_bytes(shape) -> int:
    return lib().eqlinear_window_attention_backward_workspace_bytes(shape)


def eqlinear_window_attention_backward(shape, q, k, v, lengths, starts, o, lse, d_o, dq, dk, dv, workspace,
                                       workspace_bytes, stream) -> int:
    return lib().eqlinear_window_attention_backward(shape, q, k, v, lengths, starts, o, lse, d_o, dq, dk, dv,
                                                    workspace, workspace_bytes, stream)


def eqlinear_group_norm_act_workspace_bytes(B, S, T, C, groups, dtype) -> int:
    return lib().eqlinear_group_norm_act_workspace_bytes(B, S, T, C, groups, dtype)


def eqlinear_group_norm_act(x, weight, bias, y, stats, workspace, workspace_bytes, B, S, T, C, groups, eps, act,
                            dtype, stream) -> int:
    return lib().eqlinear_group_norm_act(x, weight, bias, y, stats, workspace, workspace_bytes, B, S, T, C, groups,
                                         eps, act, dtype, stream)


def eqlinear_group_norm_act_backward_workspace_bytes(B, S, T, C, groups, dtype) -> int:
    return lib().eqlinear_group_norm_act_backward_workspace_bytes(B, S, T, C, groups, dtype)


def eqlinear_group_norm_act_backward(x, weight, bias, stats, dy, dx, dw, db, workspace, workspace_bytes, B, S, T, C,
                                     groups, act, dtype, stream) -> int:
    return lib().eqlinear_group_norm_act_backward(x, weight, bias, stats, dy, dx, dw, db, workspace, workspace_bytes,
                                                  B, S, T, C, groups, act, dtype, stream)


def eqlinear_selective_scan_workspace_bytes(shape) -> int:
    return lib().eqlinear_selective_scan_workspace_bytes(shape)


def eqlinear_selective_scan_states_bytes(shape) -> int:
    return lib().eqlinear_selective_scan_states_bytes(shape)


def eqlinear_selective_scan(shape, x, delta, A, b, c, D, z, delta_bias, lengths, state_in, y, state_out, states, workspace,
                            workspace_bytes, stream) -> int:
    return lib().eqlinear_selective_scan(shape, x, delta, A, b, c, D, z, delta_bias, lengths, state_in, y, state_out,
                                         states, workspace, workspace_bytes, stream)


def eqlinear_selective_scan_backward_workspace_bytes(shape) -> int:
    return lib().eqlinear_selective_scan_backward_workspace_bytes(shape)


def eqlinear_selective_scan_backward(shape, x, delta, A, b, c, D, z, delta_bias, lengths, states, dy, d_state_out, dx,
                                     ddelta, dA, db, dc, dD, dz, ddelta_bias, d_state_in, workspace, workspace_bytes,
                                     stream) -> int:
    return lib().eqlinear_selective_scan_backward(shape, x, delta, A, b, c, D, z, delta_bias, lengths, states, dy,
                                                  d_state_out, dx, ddelta, dA, db, dc, dD, dz, ddelta_bias, d_state_in,
                                                  workspace, workspace_bytes, stream)


def eqlinear_causal_conv(shape, x, weight, bias, lengths, state_in, y, state_out, stream) -> int:
    return lib().eqlinear_causal_conv(shape, x, weight, bias, lengths, state_in, y, state_out, stream)


def eqlinear_causal_conv_backward_workspace_bytes(shape) -> int:
    return lib().eqlinear_causal_conv_backward_workspace_bytes(shape)


def eqlinear_causal_conv_backward(shape, x, weight, bias, lengths, state_in, dy, d_state_out, dx, dweight, dbias,
                                  d_state_in, workspace, workspace_bytes, stream) -> int:
    return lib().eqlinear_causal_conv_backward(shape, x, weight, bias, lengths, state_in, dy, d_state_out, dx, dweight,
                                               dbias, d_state_in, workspace, workspace_bytes, stream)


def eqlinear_residual_norm(shape, x, branch, weight, bias, scale, gate, post_weight, post_bias, r, h, stream) -> int:
    return lib().eqlinear_residual_norm(shape, x, branch, weight, bias, scale, gate, post_weight, post_bias, r, h, stream)


def eqlinear_residual_norm_backward_workspace_bytes(shape) -> int:
    return lib().eqlinear_residual_norm_backward_workspace_bytes(shape)


def eqlinear_residual_norm_backward(shape, x, branch, weight, scale, gate, post_weight, post_bias, dr, dh, dx, dbranch,
                                    dweight, dbias, dscale, dgate, dpost_weight, dpost_bias, workspace, workspace_bytes,
                                    stream) -> int:
    return lib().eqlinear_residual_norm_backward(shape, x, branch, weight, scale, gate, post_weight, post_bias, dr, dh, dx,
                                                 dbranch, dweight, dbias, dscale, dgate, dpost_weight, dpost_bias,
                                                 workspace, workspace_bytes, stream)
