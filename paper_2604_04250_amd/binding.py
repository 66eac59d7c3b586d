"""Thin binding of libcawn's C ABI (include/cawn.h): argument marshalling only.

Every step of the hot path runs in the HIP kernels of libcawn.so.  PyTorch tensors are used as
device-memory handles (``data_ptr()``) and for the current stream; nothing here computes.  The forward and
backward entry points are called through a small C module (csrc/cawn_call.c), the rest through ctypes.  If the
shared libraries have not been built the first call fails loudly -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcawn.so")

CAWN_OK, CAWN_EINVAL, CAWN_EUNSUPPORTED, CAWN_EWORKSPACE, CAWN_ELAUNCH, CAWN_ETIMEOUT = 0, -1, -2, -3, -4, -5

EXPORTS = ["cawn_state_bytes", "cawn_workspace_bytes", "cawn_ckpt_bytes", "cawn_tile_len",
           "cawn_status_string", "cawn_workspace_init", "cawn_workspace_status", "cawn_set_spin_limit",
           "cawn_theta_init", "cawn_syntax_conv", "cawn_phase_accumulate_fwd",
           "cawn_phase_accumulate_bwd", "cawn_phase_accumulate_bf16_bwd", "cawn_phase_accumulate_bf16_fwd", "cawn_phase_accumulate_hconv_fwd", "cawn_phase_accumulate_hconv_bwd", "cawn_phase_accumulate_ret_bwd", "cawn_phase_accumulate_ret_fwd",
           "cawn_phase_accumulate_valve_fwd",
           "cawn_phase_accumulate_valve_bwd", "cawn_stream_copy", "cawn_phase_accumulate_fwd_static",
           "cawn_delta_state_bytes", "cawn_delta_ckpt_bytes", "cawn_delta_workspace_bytes", "cawn_delta_rule_fwd",
           "cawn_delta_rule_bwd", "cawn_group_norm_workspace_bytes", "cawn_group_norm_fwd", "cawn_group_norm_bwd",
           "cawn_dropout_add_fwd", "cawn_dropout_add_bwd"]


class cawn_desc(C.Structure):
    _fields_ = [("B", C.c_int32), ("L", C.c_int32), ("H", C.c_int32), ("F", C.c_int32),
                ("conv_k", C.c_int32), ("amp_mode", C.c_int32), ("gate_mode", C.c_int32),
                ("gate_tau", C.c_float), ("conv_clamp", C.c_float), ("out_clamp", C.c_float),
                ("grad_clamp", C.c_float), ("accumulate_param_grads", C.c_int32),
                ("lane_consts_cached", C.c_int32), ("valve_eps", C.c_float),
                ("ret_mode", C.c_int32), ("hconv_k", C.c_int32),
                ("in_stride_b", C.c_int64), ("in_stride_t", C.c_int64),
                ("out_stride_b", C.c_int64), ("out_stride_t", C.c_int64)]

    @property
    def J(self) -> int:
        return self.H * self.F


def make_desc(B, L, H, F, conv_k=0, amp_mode=0, gate_tau=0.0, conv_clamp=50.0, out_clamp=100.0,
              grad_clamp=100.0, accumulate_param_grads=0, lane_consts_cached=0, in_stride_b=0,
              in_stride_t=0, out_stride_b=0, out_stride_t=0, gate_mode=0, valve_eps=0.001,
              ret_mode=0, hconv_k=0) -> cawn_desc:
    return cawn_desc(B, L, H, F, conv_k, amp_mode, gate_mode, gate_tau, conv_clamp, out_clamp, grad_clamp,
                     accumulate_param_grads, lane_consts_cached, valve_eps, ret_mode, hconv_k, in_stride_b, in_stride_t,
                     out_stride_b, out_stride_t)


class cawn_delta_desc(C.Structure):
    _fields_ = [("B", C.c_int32), ("L", C.c_int32), ("H", C.c_int32), ("Hk", C.c_int32), ("K", C.c_int32), ("V", C.c_int32),
                ("bf16", C.c_int32), ("qk_norm", C.c_int32), ("scale", C.c_float), ("norm_eps", C.c_float),
                ("qk_stride_b", C.c_int64), ("qk_stride_t", C.c_int64), ("v_stride_b", C.c_int64),
                ("v_stride_t", C.c_int64), ("o_stride_b", C.c_int64), ("o_stride_t", C.c_int64)]


class cawn_norm_desc(C.Structure):
    _fields_ = [("B", C.c_int32), ("T", C.c_int32), ("C", C.c_int32), ("groups", C.c_int32), ("bf16", C.c_int32),
                ("act", C.c_int32), ("eps", C.c_float), ("accumulate_param_grads", C.c_int32),
                ("x_stride_b", C.c_int64), ("x_stride_t", C.c_int64), ("y_stride_b", C.c_int64), ("y_stride_t", C.c_int64)]


class cawn_dropout_desc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("x_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("y_stride", C.c_int64), ("p", C.c_double), ("bf16", C.c_int32), ("reserved", C.c_int32)]


def make_delta_desc(B, L, H, K, V, Hk=0, scale=1.0, qk_norm=0, norm_eps=1e-6, bf16=0, qk_stride_b=0, qk_stride_t=0,
                    v_stride_b=0, v_stride_t=0, o_stride_b=0, o_stride_t=0) -> cawn_delta_desc:
    return cawn_delta_desc(B, L, H, Hk, K, V, bf16, qk_norm, scale, norm_eps, qk_stride_b, qk_stride_t, v_stride_b, v_stride_t,
                           o_stride_b, o_stride_t)


def make_norm_desc(B, T, C, groups, act=0, eps=1e-5, bf16=0, accumulate_param_grads=0, x_stride_b=0, x_stride_t=0, y_stride_b=0,
                   y_stride_t=0) -> cawn_norm_desc:
    return cawn_norm_desc(B, T, C, groups, bf16, act, eps, accumulate_param_grads, x_stride_b, x_stride_t, y_stride_b, y_stride_t)


def make_dropout_desc(rows, cols, p=0.1, bf16=0, x_stride=0, residual_stride=0, y_stride=0) -> cawn_dropout_desc:
    return cawn_dropout_desc(rows, cols, x_stride, residual_stride, y_stride, p, bf16, 0)


_lib = None
_call = None        # csrc/cawn_call.c
_call_op = None
_entry = {}         # entry point -> address, for _call


def lib() -> C.CDLL:
    """Load libcawn.so; raise if it was not built (python -m paper_2604_04250_amd.build)."""
    global _lib, _call, _call_op
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(hipcc --offload-arch=gfx950); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        for n in ("cawn_state_bytes", "cawn_workspace_bytes", "cawn_ckpt_bytes"):
            getattr(L, n).restype = C.c_size_t
            getattr(L, n).argtypes = [C.POINTER(cawn_desc)]
        L.cawn_tile_len.restype = C.c_int32
        L.cawn_status_string.restype = C.c_char_p
        L.cawn_status_string.argtypes = [C.c_int]
        L.cawn_workspace_init.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]
        L.cawn_workspace_status.argtypes = [C.c_void_p, C.c_void_p]
        L.cawn_set_spin_limit.argtypes = [C.c_uint32]
        L.cawn_set_spin_limit.restype = None
        L.cawn_theta_init.argtypes = [C.c_int32, C.c_int32, C.c_void_p]
        L.cawn_syntax_conv.argtypes = [C.POINTER(cawn_desc), C.c_int32] + [C.c_void_p] * 7
        # (the wrappers below pass these calls to _cawn_call; programs that call lib() themselves need the types)
        L.cawn_phase_accumulate_fwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 13 +
                                                [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_bwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 19 +
                                                [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_valve_fwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 14 +
                                                      [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_valve_bwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 21 +
                                                      [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_ret_fwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 15 +
                                                    [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_ret_bwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 22 +
                                                    [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_bf16_fwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 16 +
                                                     [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_bf16_bwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 24 +
                                                     [C.c_size_t, C.c_void_p])
        L.cawn_phase_accumulate_hconv_fwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 18 +
                                                      [C.c_size_t, C.c_int32, C.c_void_p])
        L.cawn_phase_accumulate_hconv_bwd.argtypes = ([C.POINTER(cawn_desc)] + [C.c_void_p] * 28 +
                                                      [C.c_size_t, C.c_int32, C.c_void_p])
        L.cawn_stream_copy.argtypes = [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
        for n, ty in (("cawn_delta_state_bytes", cawn_delta_desc), ("cawn_delta_ckpt_bytes", cawn_delta_desc),
                      ("cawn_delta_workspace_bytes", cawn_delta_desc), ("cawn_group_norm_workspace_bytes", cawn_norm_desc)):
            getattr(L, n).restype = C.c_size_t
            getattr(L, n).argtypes = [C.POINTER(ty)]
        for n, ty, pointers, sized in (("cawn_delta_rule_fwd", cawn_delta_desc, 11, True), ("cawn_delta_rule_bwd", cawn_delta_desc, 16, True),
                                       ("cawn_group_norm_fwd", cawn_norm_desc, 6, True), ("cawn_group_norm_bwd", cawn_norm_desc, 9, True),
                                       ("cawn_dropout_add_fwd", cawn_dropout_desc, 4, False), ("cawn_dropout_add_bwd", cawn_dropout_desc, 3, False)):
            getattr(L, n).argtypes = [C.POINTER(ty)] + [C.c_void_p] * pointers + [C.c_size_t] * sized + [C.c_void_p]
        L.cawn_phase_accumulate_fwd_static.argtypes = [C.POINTER(cawn_desc)] + [C.c_void_p] * 13
        try:
            from . import _cawn_call
        except ImportError as e:
            raise RuntimeError("the marshalling module _cawn_call is missing: build it with __graft_entry__.build(); "
                               "there is no fallback path") from e
        _cawn_call.setup(cawn_desc, getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device), _raw_stream())
        _cawn_call.setup_ops((cawn_delta_desc, cawn_norm_desc, cawn_dropout_desc))
        for n in EXPORTS:
            if n.startswith("cawn_phase_accumulate") or n in _OPS:
                _entry[n] = C.cast(getattr(L, n), C.c_void_p).value
        _call = _cawn_call.call
        _call_op = _cawn_call.call_op
        _lib = L
    return _lib


def _raw_stream():
    """device index -> handle of its current stream (torch's own accessor where this build of it has one)."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw if raw is not None else (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _enter(name, form, *args) -> int:
    if _call is None:
        lib()
    return _call(_entry[name], form, *args)


# operators with a descriptor of their own: 2 * the descriptor's place in setup_ops, + 1 where a workspace comes last
_OPS = {"cawn_delta_rule_fwd": 1, "cawn_delta_rule_bwd": 1, "cawn_group_norm_fwd": 3, "cawn_group_norm_bwd": 3,
        "cawn_dropout_add_fwd": 4, "cawn_dropout_add_bwd": 4}


def _enter_op(name, *args) -> int:
    if _call_op is None:
        lib()
    return _call_op(_entry[name], _OPS[name], *args)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda, "libcawn takes device pointers"
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def check(status: int) -> None:
    if status != CAWN_OK:
        raise RuntimeError(f"libcawn: {cawn_status_string(status)} ({status})")


def cawn_state_bytes(d: cawn_desc) -> int:
    return int(lib().cawn_state_bytes(C.byref(d)))


def cawn_workspace_bytes(d: cawn_desc) -> int:
    return int(lib().cawn_workspace_bytes(C.byref(d)))


def cawn_ckpt_bytes(d: cawn_desc) -> int:
    return int(lib().cawn_ckpt_bytes(C.byref(d)))


def cawn_tile_len() -> int:
    return int(lib().cawn_tile_len())


def cawn_status_string(status: int) -> str:
    return lib().cawn_status_string(int(status)).decode()


def cawn_workspace_init(workspace: torch.Tensor, stream=None) -> int:
    return lib().cawn_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream))


def cawn_workspace_status(workspace: torch.Tensor, stream=None) -> int:
    return lib().cawn_workspace_status(_ptr(workspace), _stream(stream))


def cawn_set_spin_limit(polls: int) -> None:
    lib().cawn_set_spin_limit(int(polls))


def cawn_theta_init(H: int, F: int):
    """Host helper: the paper's rotation-angle initialisation as a float32 numpy array [H*F]."""
    import numpy as np
    out = np.empty(H * F, dtype=np.float32)
    check(lib().cawn_theta_init(H, F, out.ctypes.data_as(C.c_void_p)))
    return out


def cawn_syntax_conv(d, Cch, x, w, bias, conv_state_in, y, conv_state_out, stream=None) -> int:
    return lib().cawn_syntax_conv(C.byref(d), int(Cch), _ptr(x), _ptr(w), _ptr(bias),
                                  _ptr(conv_state_in), _ptr(y), _ptr(conv_state_out), _stream(stream))


def cawn_phase_accumulate_fwd(d, mag, ang, gamma, theta, conv_w, conv_b, state_in, z_re, z_im,
                              state_out, ckpt, gate_mask, workspace, stream=None) -> int:
    return _enter("cawn_phase_accumulate_fwd", 1,
                  d, mag, ang, gamma, theta, conv_w, conv_b, state_in, z_re, z_im, state_out, ckpt, gate_mask,
                  workspace, stream)


def cawn_phase_accumulate_bwd(d, mag, ang, gamma, theta, conv_w, conv_b, state_in, ckpt, dz_re,
                              dz_im, dstate_out, dmag, dang, dgamma, dtheta, dconv_w, dconv_b,
                              dstate_in, workspace, stream=None) -> int:
    return _enter("cawn_phase_accumulate_bwd", 1,
                  d, mag, ang, gamma, theta, conv_w, conv_b, state_in, ckpt, dz_re, dz_im, dstate_out, dmag, dang,
                  dgamma, dtheta, dconv_w, dconv_b, dstate_in, workspace, stream)


def cawn_phase_accumulate_valve_fwd(d, mag, ang, valve, gamma, theta, conv_w, conv_b, state_in, z_re,
                                    z_im, state_out, ckpt, gate_mask, workspace, stream=None) -> int:
    return _enter("cawn_phase_accumulate_valve_fwd", 1,
                  d, mag, ang, valve, gamma, theta, conv_w, conv_b, state_in, z_re, z_im, state_out, ckpt, gate_mask,
                  workspace, stream)


def cawn_phase_accumulate_valve_bwd(d, mag, ang, valve, gamma, theta, conv_w, conv_b, state_in, ckpt,
                                    dz_re, dz_im, dstate_out, dmag, dang, dvalve, dgamma, dtheta,
                                    dconv_w, dconv_b, dstate_in, workspace, stream=None) -> int:
    return _enter("cawn_phase_accumulate_valve_bwd", 1,
                  d, mag, ang, valve, gamma, theta, conv_w, conv_b, state_in, ckpt, dz_re, dz_im, dstate_out, dmag,
                  dang, dvalve, dgamma, dtheta, dconv_w, dconv_b, dstate_in, workspace, stream)


def cawn_phase_accumulate_ret_fwd(d, mag, ang, valve, ret, ret_bias, theta, conv_w, conv_b, state_in, z_re,
                                  z_im, state_out, ckpt, gate_mask, workspace, stream=None) -> int:
    return _enter("cawn_phase_accumulate_ret_fwd", 1,
                  d, mag, ang, valve, ret, ret_bias, theta, conv_w, conv_b, state_in, z_re, z_im, state_out, ckpt,
                  gate_mask, workspace, stream)


def cawn_phase_accumulate_ret_bwd(d, mag, ang, valve, ret, ret_bias, theta, conv_w, conv_b, state_in, ckpt,
                                  dz_re, dz_im, dstate_out, dmag, dang, dvalve, dret, dtheta, dconv_w,
                                  dconv_b, dstate_in, workspace, stream=None) -> int:
    return _enter("cawn_phase_accumulate_ret_bwd", 1,
                  d, mag, ang, valve, ret, ret_bias, theta, conv_w, conv_b, state_in, ckpt, dz_re, dz_im, dstate_out,
                  dmag, dang, dvalve, dret, dtheta, dconv_w, dconv_b, dstate_in, workspace, stream)


def cawn_phase_accumulate_bf16_fwd(d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, state_in,
                                   z_re, z_im, state_out, ckpt, gate_mask, workspace, stream=None) -> int:
    """mag, ang, z_re, z_im: torch.bfloat16 tensors."""
    return _enter("cawn_phase_accumulate_bf16_fwd", 1,
                  d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, state_in, z_re, z_im, state_out,
                  ckpt, gate_mask, workspace, stream)


def cawn_phase_accumulate_hconv_fwd(d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, hconv_w,
                                    hconv_b, state_in, zc_re, zc_im, state_out, ckpt, gate_mask, workspace,
                                    activations_bf16=0, stream=None) -> int:
    """mag, ang, zc_re, zc_im: fp32 tensors, or torch.bfloat16 with activations_bf16=1."""
    return _enter("cawn_phase_accumulate_hconv_fwd", 2,
                  d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, hconv_w, hconv_b, state_in, zc_re,
                  zc_im, state_out, ckpt, gate_mask, workspace, activations_bf16, stream)


def cawn_phase_accumulate_hconv_bwd(d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, hconv_w, hconv_b,
                                    state_in, ckpt, dc_re, dc_im, dstate_out, dmag, dang, dvalve, dret, dgamma, dtheta,
                                    dconv_w, dconv_b, dhconv_w, dhconv_b, dstate_in, workspace, activations_bf16=0,
                                    stream=None) -> int:
    """dc_re, dc_im: gradients of the convolved output; dhconv_w [2,H,3], dhconv_b [2,H] beside the usual gradients.
    mag, ang, dc_re, dc_im, dmag, dang: fp32 tensors, or torch.bfloat16 with activations_bf16=1."""
    return _enter("cawn_phase_accumulate_hconv_bwd", 2,
                  d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, hconv_w, hconv_b, state_in, ckpt,
                  dc_re, dc_im, dstate_out, dmag, dang, dvalve, dret, dgamma, dtheta, dconv_w, dconv_b, dhconv_w,
                  dhconv_b, dstate_in, workspace, activations_bf16, stream)


def cawn_phase_accumulate_bf16_bwd(d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, state_in, ckpt,
                                   dz_re, dz_im, dstate_out, dmag, dang, dvalve, dret, dgamma, dtheta, dconv_w,
                                   dconv_b, dstate_in, workspace, stream=None) -> int:
    """mag, ang, dz_re, dz_im, dmag, dang: torch.bfloat16 tensors."""
    return _enter("cawn_phase_accumulate_bf16_bwd", 1,
                  d, mag, ang, valve, ret, ret_bias, gamma, theta, conv_w, conv_b, state_in, ckpt, dz_re, dz_im,
                  dstate_out, dmag, dang, dvalve, dret, dgamma, dtheta, dconv_w, dconv_b, dstate_in, workspace, stream)


def cawn_phase_accumulate_fwd_static(d, mag, ang, gamma, theta, conv_w, conv_b, state_in, z_re, z_im,
                                     state_out, ckpt, gate_mask, stream=None) -> int:
    """cawn_phase_accumulate_fwd on the library's static scratch array: allocates nothing."""
    return _enter("cawn_phase_accumulate_fwd_static", 0,
                  d, mag, ang, gamma, theta, conv_w, conv_b, state_in, z_re, z_im, state_out, ckpt, gate_mask, stream)


def cawn_stream_copy(in0, in1, out0, out1, stream=None) -> int:
    """Plain copy of two fp32 streams (the bandwidth ceiling the scan kernels are read against)."""
    return lib().cawn_stream_copy(_ptr(in0), _ptr(in1), _ptr(out0), _ptr(out1), in0.numel(), _stream(stream))


def cawn_delta_state_bytes(d: cawn_delta_desc) -> int:
    return int(lib().cawn_delta_state_bytes(C.byref(d)))


def cawn_delta_ckpt_bytes(d: cawn_delta_desc) -> int:
    return int(lib().cawn_delta_ckpt_bytes(C.byref(d)))


def cawn_delta_workspace_bytes(d: cawn_delta_desc) -> int:
    return int(lib().cawn_delta_workspace_bytes(C.byref(d)))


def cawn_delta_rule_fwd(d, q, k, v, decay, beta, lengths, state_in, o, state_out, ckpt, workspace, stream=None) -> int:
    """q, k, v, o: fp32 tensors, or torch.bfloat16 with d.bf16 = 1; decay, beta, states fp32; lengths torch.int32."""
    return _enter_op("cawn_delta_rule_fwd", d, q, k, v, decay, beta, lengths, state_in, o, state_out, ckpt, workspace, stream)


def cawn_delta_rule_bwd(d, q, k, v, decay, beta, lengths, ckpt, do, dstate_out, dq, dk, dv, ddecay, dbeta, dstate_in, workspace,
                        stream=None) -> int:
    """do and dq, dk, dv: the type of q, k, v, o."""
    return _enter_op("cawn_delta_rule_bwd", d, q, k, v, decay, beta, lengths, ckpt, do, dstate_out, dq, dk, dv, ddecay, dbeta,
                     dstate_in, workspace, stream)


def cawn_group_norm_workspace_bytes(d: cawn_norm_desc) -> int:
    return int(lib().cawn_group_norm_workspace_bytes(C.byref(d)))


def cawn_group_norm_fwd(d, x, weight, bias, y, stats, workspace, stream=None) -> int:
    """x, y: fp32 tensors, or torch.bfloat16 with d.bf16 = 1; the rest fp32."""
    return _enter_op("cawn_group_norm_fwd", d, x, weight, bias, y, stats, workspace, stream)


def cawn_group_norm_bwd(d, x, weight, bias, stats, dy, dx, dweight, dbias, workspace, stream=None) -> int:
    return _enter_op("cawn_group_norm_bwd", d, x, weight, bias, stats, dy, dx, dweight, dbias, workspace, stream)


def cawn_dropout_add_fwd(d, x, residual, rng, y, stream=None) -> int:
    """rng: torch.int64 tensor {seed, offset} on the device."""
    return _enter_op("cawn_dropout_add_fwd", d, x, residual, rng, y, stream)


def cawn_dropout_add_bwd(d, dy, rng, dx, stream=None) -> int:
    return _enter_op("cawn_dropout_add_bwd", d, dy, rng, dx, stream)


def alloc_workspace(d: cawn_desc, device="cuda:0") -> torch.Tensor:
    """Allocate (torch caching allocator, 256-byte aligned) and initialise a workspace for `d`."""
    n = cawn_workspace_bytes(d)
    ws = torch.empty((n + 3) // 4, dtype=torch.int32, device=device)
    check(cawn_workspace_init(ws))
    return ws
