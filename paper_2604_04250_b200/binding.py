"""ctypes binding of ``libcawn.so`` -- argument marshalling only.

Function names and argument order follow ``include/cawn.h``.  Tensors are torch CUDA tensors
(used purely as device memory) or ``None``; complex64 tensors are passed as they are
(interleaved re, im).  Every step of the path runs in the library's CUDA kernels: there is no
CPU or eager fallback, and a missing library is an error.
"""
from __future__ import annotations

import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcawn.so")

CAWN_OK = 0
CAWN_ERR_INVALID_ARG = -1
CAWN_ERR_NULL_POINTER = -2
CAWN_ERR_MISALIGNED = -3
CAWN_ERR_UNSUPPORTED = -4
CAWN_ERR_WORKSPACE_TOO_SMALL = -5
CAWN_ERR_CUDA = -6
CAWN_ERR_STATIC_TOO_LARGE = -7
CAWN_STATIC_SCRATCH_BYTES = 4 << 20
CAWN_ERR_CARRY_TIMEOUT = 1
CAWN_STATUS_NONFINITE = 2

CAWN_FLAG_PRELUDE_CLAMP_SILU = 1
CAWN_FLAG_RETENTION_DYNAMIC = 2
CAWN_FLAG_INPUT_INDEPENDENT = 4
CAWN_FLAG_INPUT_BF16 = 8
CAWN_FLAG_OUTPUT_BF16 = 16

CAWN_OP_FWD, CAWN_OP_BWD_SAVED, CAWN_OP_BWD_PUSHES, CAWN_OP_STATE, CAWN_OP_FWD_HOST, CAWN_OP_MIXING_BWD = range(6)
CAWN_SAVED_STATES, CAWN_SAVED_PUSHES = 0, 1
CAWN_DELTA_FWD, CAWN_DELTA_BWD = 0, 1
CAWN_NORM_ACT_NONE, CAWN_NORM_ACT_SILU, CAWN_NORM_ACT_GATE = range(3)
CAWN_CONV_ACT_NONE, CAWN_CONV_ACT_SILU = range(2)
CAWN_SCAN_FWD, CAWN_SCAN_BWD, CAWN_SCAN_BWD_RECOMPUTE, CAWN_SCAN_CHECKPOINTS = range(4)
CAWN_NORM_OUT_SAME, CAWN_NORM_OUT_E4M3 = range(2)

EXPORTS = (
    "cawn_status_string", "cawn_workspace_bytes", "cawn_workspace_init",
    "cawn_phase_accumulate_fwd", "cawn_phase_accumulate_bwd", "cawn_state_carry",
    "cawn_poll_status", "cawn_phase_accumulate_fwd_host", "cawn_phase_accumulate_fwd_static",
    "cawn_phase_accumulate_bwd_dynamic", "cawn_mixing_bwd", "cawn_phase_accumulate_fwd_ear",
    "cawn_workspace_set_wait_hook", "cawn_mixing_bwd_dynamic",
    "cawn_delta_rule_workspace_bytes", "cawn_delta_rule_fwd", "cawn_delta_rule_step", "cawn_delta_rule_bwd",
    "cawn_group_norm_fwd", "cawn_group_norm_workspace_bytes", "cawn_group_norm_bwd", "cawn_dropout",
    "cawn_short_conv_fwd", "cawn_short_conv_workspace_bytes", "cawn_short_conv_bwd",
    "cawn_selective_scan_workspace_bytes", "cawn_selective_scan_fwd", "cawn_selective_scan_step", "cawn_selective_scan_bwd",
    "cawn_residual_norm_fwd", "cawn_residual_norm_workspace_bytes", "cawn_residual_norm_bwd",
)


class cawn_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32),
        ("L", ctypes.c_int64),
        ("H", ctypes.c_int32),
        ("F", ctypes.c_int32),
        ("gate_eps", ctypes.c_float),
        ("gate_tau", ctypes.c_float),
        ("clamp_abs", ctypes.c_float),
        ("grad_clamp_abs", ctypes.c_float),
        ("conv_k", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
    ]


class cawn_delta_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32),
        ("L", ctypes.c_int64),
        ("Hk", ctypes.c_int32),
        ("Hv", ctypes.c_int32),
        ("Dk", ctypes.c_int32),
        ("Dv", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("flags", ctypes.c_uint32),
        ("q_stride", ctypes.c_int64),
        ("k_stride", ctypes.c_int64),
        ("v_stride", ctypes.c_int64),
        ("o_stride", ctypes.c_int64),
    ]


class cawn_norm_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("G", ctypes.c_int32),
        ("N", ctypes.c_int64),
        ("M", ctypes.c_int32),
        ("act", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("rms", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
        ("x_stride", ctypes.c_int64),
        ("gate_stride", ctypes.c_int64),
    ]


class cawn_dropout_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("p", ctypes.c_float),
        ("n", ctypes.c_int64),
        ("seed", ctypes.c_uint64),
        ("offset", ctypes.c_uint64),
        ("flags", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
    ]


class cawn_conv_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32),
        ("L", ctypes.c_int64),
        ("C", ctypes.c_int32),
        ("K", ctypes.c_int32),
        ("act", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32 * 2),
        ("x_stride", ctypes.c_int64),
        ("rows", ctypes.c_int64),
    ]


class cawn_scan_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32),
        ("L", ctypes.c_int64),
        ("D", ctypes.c_int32),
        ("N", ctypes.c_int32),
        ("G", ctypes.c_int32),
        ("softplus", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
        ("x_stride", ctypes.c_int64),
        ("dt_stride", ctypes.c_int64),
        ("z_stride", ctypes.c_int64),
        ("b_stride", ctypes.c_int64),
        ("c_stride", ctypes.c_int64),
        ("rows", ctypes.c_int64),
    ]


class cawn_residual_norm_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("M", ctypes.c_int32),
        ("N", ctypes.c_int64),
        ("eps", ctypes.c_float),
        ("out", ctypes.c_int32),
        ("scale_block", ctypes.c_int32),
        ("stream_float", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
        ("x_stride", ctypes.c_int64),
    ]


class CawnError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, status_string(status), status))


_lib = None


def lib():
    """Load ``libcawn.so`` (built in-tree by ``paper_2604_04250_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libcawn.so is missing: run `python -m paper_2604_04250_b200.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, fp, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t
        pp = ctypes.POINTER(cawn_params)
        L.cawn_status_string.restype = ctypes.c_char_p
        L.cawn_status_string.argtypes = [ctypes.c_int]
        L.cawn_workspace_bytes.argtypes = [pp, ctypes.c_int, ctypes.POINTER(sz)]
        L.cawn_workspace_init.argtypes = [vp, sz, vp]
        L.cawn_phase_accumulate_fwd.argtypes = [pp, vp, fp, fp, fp, fp, fp, fp, vp, vp, vp, vp, vp, sz, vp]
        L.cawn_phase_accumulate_bwd.argtypes = [pp, vp, ctypes.c_int, fp, fp, vp, vp, vp, vp, fp, fp, vp, vp, sz, vp]
        L.cawn_phase_accumulate_bwd_dynamic.argtypes = [pp, vp, ctypes.c_int, fp, fp, fp, vp, vp, vp, vp, fp, fp, fp, vp, vp, sz, vp]
        L.cawn_mixing_bwd.argtypes = [pp, fp, fp, fp, fp, fp, vp, vp, vp, vp, fp, fp, fp, fp, fp, vp, vp, sz, vp]
        L.cawn_phase_accumulate_fwd_ear.argtypes = [pp, vp, fp, fp, fp, fp, fp, fp, vp, fp, fp, ctypes.c_int, fp, vp, vp, vp, sz, vp]
        L.cawn_mixing_bwd_dynamic.argtypes = [pp, fp, fp, fp, fp, fp, fp, vp, vp, vp, vp, fp, fp, fp, fp, fp, fp, vp, vp, sz, vp]
        L.cawn_state_carry.argtypes = [pp, vp, vp, ctypes.c_int64, fp, fp, vp, vp]
        L.cawn_poll_status.argtypes = [vp, vp]
        L.cawn_workspace_set_wait_hook.argtypes = [vp, ctypes.c_int, ctypes.c_uint, vp]
        L.cawn_phase_accumulate_fwd_host.argtypes = [pp, vp, fp, fp, vp, vp, vp, vp, vp, sz, vp]
        L.cawn_phase_accumulate_fwd_static.argtypes = [pp, vp, fp, fp, vp, vp, vp, vp, vp, vp]
        dp, np_, op = ctypes.POINTER(cawn_delta_params), ctypes.POINTER(cawn_norm_params), ctypes.POINTER(cawn_dropout_params)
        L.cawn_delta_rule_workspace_bytes.argtypes = [dp, ctypes.c_int, ctypes.POINTER(sz)]
        L.cawn_delta_rule_fwd.argtypes = [dp, vp, vp, vp, fp, fp, fp, vp, fp, vp, sz, vp]
        L.cawn_delta_rule_step.argtypes = [dp, vp, vp, vp, fp, fp, fp, vp, fp, vp]
        L.cawn_delta_rule_bwd.argtypes = [dp, vp, vp, vp, fp, fp, fp, vp, fp, vp, vp, vp, fp, fp, fp, vp, sz, vp]
        L.cawn_group_norm_fwd.argtypes = [np_, vp, fp, fp, vp, vp, vp]
        L.cawn_group_norm_workspace_bytes.argtypes = [np_, ctypes.POINTER(sz)]
        L.cawn_group_norm_bwd.argtypes = [np_, vp, fp, fp, vp, vp, vp, vp, fp, fp, vp, sz, vp]
        L.cawn_dropout.argtypes = [op, vp, vp, vp, vp, vp]
        cp, sp, rp = ctypes.POINTER(cawn_conv_params), ctypes.POINTER(cawn_scan_params), ctypes.POINTER(cawn_residual_norm_params)
        L.cawn_short_conv_fwd.argtypes = [cp, vp, fp, fp, fp, vp, vp, fp, vp]
        L.cawn_short_conv_workspace_bytes.argtypes = [cp, ctypes.POINTER(sz)]
        L.cawn_short_conv_bwd.argtypes = [cp, vp, fp, fp, fp, vp, vp, fp, vp, fp, fp, fp, vp, sz, vp]
        L.cawn_selective_scan_workspace_bytes.argtypes = [sp, ctypes.c_int, ctypes.POINTER(sz)]
        L.cawn_selective_scan_fwd.argtypes = [sp, vp, vp, fp, vp, vp, fp, fp, vp, fp, vp, vp, fp, fp, vp, sz, vp]
        L.cawn_selective_scan_step.argtypes = [sp, vp, vp, fp, vp, vp, fp, fp, vp, fp, vp, fp, vp]
        L.cawn_selective_scan_bwd.argtypes = [sp, vp, vp, fp, vp, vp, fp, fp, vp, fp, vp, fp, vp, fp, vp, vp, fp, vp, vp, fp, fp, vp, fp, vp, sz, vp]
        L.cawn_residual_norm_fwd.argtypes = [rp, vp, vp, fp, vp, vp, fp, vp]
        L.cawn_residual_norm_workspace_bytes.argtypes = [rp, ctypes.POINTER(sz)]
        L.cawn_residual_norm_bwd.argtypes = [rp, vp, fp, vp, vp, vp, vp, fp, vp, sz, vp]
        for name in EXPORTS:
            if name != "cawn_status_string":
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def make_params(B, L, H, F, gate_eps=0.0, gate_tau=0.0, clamp_abs=0.0, grad_clamp_abs=0.0,
                conv_k=0, flags=0):
    return cawn_params(ctypes.sizeof(cawn_params), B, L, H, F, gate_eps, gate_tau, clamp_abs,
                       grad_clamp_abs, conv_k, flags)


def status_string(status):
    return lib().cawn_status_string(int(status)).decode()


def _dp(t):
    """Device (or host) pointer of a tensor / numpy array / None."""
    if t is None:
        return None
    try:
        return t.data_ptr()
    except AttributeError:
        return t.ctypes.data


_current_stream = None


def _stream(stream):
    """The given stream's handle, or that of torch's current stream on the current device.  The latter is asked
    for by every call: torch's own raw lookup takes 0.3 us, building a Stream object for its handle 3 us."""
    global _current_stream
    if stream is None:
        if _current_stream is None:
            import torch
            torch.cuda.current_stream()         # initialises CUDA, with torch's own message where there is none
            raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            _current_stream = (lambda: raw(device())) if raw and device else lambda: torch.cuda.current_stream().cuda_stream
        return _current_stream()
    return getattr(stream, "cuda_stream", stream)


def _check(rc, where):
    if rc != CAWN_OK:
        raise CawnError(rc, where)


def cawn_workspace_bytes(params, op):
    n = ctypes.c_size_t(0)
    _check(lib().cawn_workspace_bytes(ctypes.byref(params), op, ctypes.byref(n)), "cawn_workspace_bytes")
    return n.value


def cawn_workspace_init(workspace, stream=None):
    _check(lib().cawn_workspace_init(_dp(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream)), "cawn_workspace_init")


def new_workspace(params, op, device="cuda"):
    """Allocate (with torch, as plain device memory) and initialise a workspace for `op`."""
    import torch
    n = cawn_workspace_bytes(params, op)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)
    cawn_workspace_init(ws)
    return ws


def cawn_phase_accumulate_fwd(params, input, gamma, theta, y, workspace, conv_w=None, conv_bias=None,
                              gamma_logit=None, freq_bias=None, state_in=None, state_out=None,
                              gate_mask=None, stream=None):
    _check(lib().cawn_phase_accumulate_fwd(
        ctypes.byref(params), _dp(input), _dp(gamma), _dp(theta), _dp(conv_w), _dp(conv_bias),
        _dp(gamma_logit), _dp(freq_bias), _dp(state_in), _dp(y), _dp(state_out), _dp(gate_mask),
        _dp(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
        "cawn_phase_accumulate_fwd")


def cawn_phase_accumulate_fwd_ear(params, input, gamma, theta, ear_w, ear_k, z_conv, workspace, ear_bias=None,
                                  conv_w=None, conv_bias=None, gamma_logit=None, freq_bias=None, state_in=None,
                                  state_out=None, gate_mask=None, stream=None):
    _check(lib().cawn_phase_accumulate_fwd_ear(
        ctypes.byref(params), _dp(input), _dp(gamma), _dp(theta), _dp(conv_w), _dp(conv_bias), _dp(gamma_logit),
        _dp(freq_bias), _dp(state_in),
        _dp(ear_w), _dp(ear_bias), int(ear_k), _dp(z_conv), _dp(state_out), _dp(gate_mask),
        _dp(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
        "cawn_phase_accumulate_fwd_ear")


def cawn_phase_accumulate_bwd(params, saved, saved_kind, gamma, theta, grad_y, grad_p, workspace,
                              state_in=None, grad_state_out=None, grad_gamma=None, grad_theta=None,
                              grad_state_in=None, stream=None):
    _check(lib().cawn_phase_accumulate_bwd(
        ctypes.byref(params), _dp(saved), saved_kind, _dp(gamma), _dp(theta), _dp(state_in),
        _dp(grad_y), _dp(grad_state_out), _dp(grad_p), _dp(grad_gamma), _dp(grad_theta),
        _dp(grad_state_in), _dp(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)), "cawn_phase_accumulate_bwd")


def cawn_mixing_bwd_dynamic(params, h, conv_w, gamma_logit, freq_bias, theta, grad_y, grad_h, workspace, conv_bias=None,
                            saved_states=None, state_in=None, grad_state_out=None, grad_conv_w=None, grad_conv_bias=None,
                            grad_gamma_logit=None, grad_freq_bias=None, grad_theta=None, grad_state_in=None, stream=None):
    _check(lib().cawn_mixing_bwd_dynamic(
        ctypes.byref(params), _dp(h), _dp(conv_w), _dp(conv_bias), _dp(gamma_logit), _dp(freq_bias), _dp(theta),
        _dp(saved_states), _dp(state_in), _dp(grad_y), _dp(grad_state_out), _dp(grad_h), _dp(grad_conv_w),
        _dp(grad_conv_bias), _dp(grad_gamma_logit), _dp(grad_freq_bias), _dp(grad_theta), _dp(grad_state_in),
        _dp(workspace), workspace.numel() * workspace.element_size(), _stream(stream)), "cawn_mixing_bwd_dynamic")


def cawn_state_carry(params, state_prev, state_local, n_steps, gamma, theta, state_out, stream=None):
    _check(lib().cawn_state_carry(ctypes.byref(params), _dp(state_prev), _dp(state_local),
                                  int(n_steps), _dp(gamma), _dp(theta), _dp(state_out),
                                  _stream(stream)), "cawn_state_carry")


def cawn_workspace_set_wait_hook(workspace, withhold_tile, poll_bound, stream=None):
    _check(lib().cawn_workspace_set_wait_hook(_dp(workspace), int(withhold_tile), int(poll_bound), _stream(stream)),
           "cawn_workspace_set_wait_hook")


def cawn_poll_status(workspace, stream=None):
    return lib().cawn_poll_status(_dp(workspace), _stream(stream))


def cawn_phase_accumulate_fwd_host(params, p_host, gamma_host, theta_host, y_host, device_scratch,
                                   state_in_host=None, state_out_host=None, gate_mask_host=None,
                                   stream=None):
    _check(lib().cawn_phase_accumulate_fwd_host(
        ctypes.byref(params), _dp(p_host), _dp(gamma_host), _dp(theta_host), _dp(state_in_host),
        _dp(y_host), _dp(state_out_host), _dp(gate_mask_host), _dp(device_scratch),
        device_scratch.numel() * device_scratch.element_size(), _stream(stream)),
        "cawn_phase_accumulate_fwd_host")


def cawn_phase_accumulate_fwd_static(params, input, gamma, theta, y, state_in=None, state_out=None,
                                     gate_mask=None, device_status=None, stream=None):
    """Forward scan on the library's built-in scratch array: for callers that hold input and
    output buffers but cannot allocate a workspace.  One call at a time per device."""
    _check(lib().cawn_phase_accumulate_fwd_static(
        ctypes.byref(params), _dp(input), _dp(gamma), _dp(theta), _dp(state_in), _dp(y),
        _dp(state_out), _dp(gate_mask), _dp(device_status), _stream(stream)),
        "cawn_phase_accumulate_fwd_static")


def cawn_phase_accumulate_bwd_dynamic(params, saved, saved_kind, gamma_logit, freq_bias, theta, grad_y, grad_p,
                                      workspace, state_in=None, grad_state_out=None, grad_gamma_logit=None,
                                      grad_freq_bias=None, grad_theta=None, grad_state_in=None, stream=None):
    _check(lib().cawn_phase_accumulate_bwd_dynamic(
        ctypes.byref(params), _dp(saved), saved_kind, _dp(gamma_logit), _dp(freq_bias), _dp(theta),
        _dp(state_in), _dp(grad_y), _dp(grad_state_out), _dp(grad_p), _dp(grad_gamma_logit),
        _dp(grad_freq_bias), _dp(grad_theta), _dp(grad_state_in), _dp(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)), "cawn_phase_accumulate_bwd_dynamic")


def cawn_mixing_bwd(params, h, conv_w, gamma, theta, grad_y, grad_h, workspace, conv_bias=None, saved_states=None,
                    state_in=None, grad_state_out=None, grad_conv_w=None, grad_conv_bias=None, grad_gamma=None,
                    grad_theta=None, grad_state_in=None, stream=None):
    _check(lib().cawn_mixing_bwd(
        ctypes.byref(params), _dp(h), _dp(conv_w), _dp(conv_bias), _dp(gamma), _dp(theta), _dp(saved_states),
        _dp(state_in), _dp(grad_y), _dp(grad_state_out), _dp(grad_h), _dp(grad_conv_w), _dp(grad_conv_bias),
        _dp(grad_gamma), _dp(grad_theta), _dp(grad_state_in), _dp(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)), "cawn_mixing_bwd")


# ---- operators next to the phase accumulation in a layer

def make_delta_params(B, L, Hk, Hv, Dk, Dv, scale=None, flags=0, q_stride=0, k_stride=0, v_stride=0, o_stride=0):
    return cawn_delta_params(ctypes.sizeof(cawn_delta_params), B, L, Hk, Hv, Dk, Dv,
                             max(Dk, 1) ** -0.5 if scale is None else scale, flags, q_stride, k_stride, v_stride, o_stride)


def _dense(names, *arrays):
    """What the kernels take as dense arrays has to be laid out so."""
    try:
        for x in arrays:
            if x is not None and not x.is_contiguous():
                break
        else:
            return
    except AttributeError:              # not a tensor (a numpy array): its owner's business
        return
    name = next(n for n, y in zip(names.split(), arrays) if y is x)
    raise ValueError(f"{name}: strides {tuple(x.stride())} of shape {tuple(x.shape)}, it has to be dense")


def _yes():
    return True

def _check_rows(name, x, width, row):
    """x's elements, in order, have to be rows of `width` neighbours that start `row` apart (the shape may be any that
    has whole rows: [B, L, H, D], [B, L, H * D], [B * L, H * D])."""
    if row == width and getattr(x, "is_contiguous", _yes)() or not hasattr(x, "stride"):
        return
    shape, strides = x.shape, x.stride()
    expect, inside = 1, 1               # the step that is due, the elements of a row that the dimensions so far hold
    for i in range(len(shape) - 1, -1, -1):
        size = shape[i]
        if size == 1:
            continue
        over = inside * size
        if strides[i] != expect or (inside < width < over and (over % width != 0 or row != width)):
            raise ValueError(f"{name} {row}: strides {tuple(strides)} of shape {tuple(shape)}, which are not rows of {width} "
                             f"elements {row} apart")
        expect *= size
        if inside < width:
            inside = over
            if inside >= width:
                expect = row * (inside // width)


def _delta_rows(params, q, k, v, o):
    """The params of a call whose tensors are [B, L, ...], their layout checked: rows (all heads of a token) contiguous and
    *_stride apart, batches L strides apart.  One token has no step to the next, so torch gives that dimension any
    stride (that of a slice of a projection, seen as heads, is the slice's width); the step between batches is then
    the rows' stride."""
    B, L, p = params.B, params.L, params
    if L < 1:
        return params
    try:                                # the usual cases at once: whole tensors, with no stride given or none that counts
        if (q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and o.is_contiguous() and
                (B * L == 1 or not (p.q_stride or p.k_stride or p.v_stride or p.o_stride))):
            return params
    except AttributeError:
        pass
    qk, vo = p.Hk * p.Dk, p.Hv * p.Dv
    for name, x, width, row in (("q_stride", q, qk, p.q_stride), ("k_stride", k, qk, p.k_stride),
                                ("v_stride", v, vo, p.v_stride), ("o_stride", o, vo, p.o_stride)):
        if row == 0:
            row = width
        if L == 1 and B > 1:
            shape = getattr(x, "shape", ())
            if len(shape) > 2 and shape[0] == B and shape[1] == 1:
                batch = x.stride(0)
                if batch < width:       # a tensor expanded over the batch; 0 would say dense in the C call
                    raise ValueError(f"{name}: batches of one row of {width} elements lie {batch} apart")
                if batch != row:
                    if p is params:
                        p = cawn_delta_params.from_buffer_copy(params)
                    setattr(p, name, batch)
                    row = batch
        _check_rows(name, x, width, row)
    return p


def cawn_delta_rule_workspace_bytes(params, op):
    n = ctypes.c_size_t(0)
    _check(lib().cawn_delta_rule_workspace_bytes(ctypes.byref(params), op, ctypes.byref(n)),
           "cawn_delta_rule_workspace_bytes")
    return n.value


def _plain_workspace(n, device):
    import torch
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def new_delta_workspace(params, op, device="cuda"):
    """Allocate (with torch, as plain device memory) a workspace for CAWN_DELTA_FWD or CAWN_DELTA_BWD."""
    return _plain_workspace(cawn_delta_rule_workspace_bytes(params, op), device)


def cawn_delta_rule_fwd(params, q, k, v, g, beta, o, workspace, state_in=None, state_out=None, stream=None):
    _dense("g beta state_in state_out", g, beta, state_in, state_out)
    params = _delta_rows(params, q, k, v, o)
    _check(lib().cawn_delta_rule_fwd(
        ctypes.byref(params), _dp(q), _dp(k), _dp(v), _dp(g), _dp(beta), _dp(state_in), _dp(o), _dp(state_out),
        _dp(workspace), workspace.numel() * workspace.element_size(), _stream(stream)), "cawn_delta_rule_fwd")


def cawn_delta_rule_step(params, q, k, v, g, beta, o, state_in=None, state_out=None, stream=None):
    _dense("g beta state_in state_out", g, beta, state_in, state_out)
    params = _delta_rows(params, q, k, v, o)
    _check(lib().cawn_delta_rule_step(
        ctypes.byref(params), _dp(q), _dp(k), _dp(v), _dp(g), _dp(beta), _dp(state_in), _dp(o), _dp(state_out),
        _stream(stream)), "cawn_delta_rule_step")


def cawn_delta_rule_bwd(params, q, k, v, g, beta, grad_o, grad_q, grad_k, grad_v, grad_g, grad_beta, workspace,
                        state_in=None, grad_state_out=None, grad_state_in=None, stream=None):
    _dense("g beta state_in grad_state_out grad_q grad_k grad_v grad_g grad_beta grad_state_in",
           g, beta, state_in, grad_state_out, grad_q, grad_k, grad_v, grad_g, grad_beta, grad_state_in)
    params = _delta_rows(params, q, k, v, grad_o)
    _check(lib().cawn_delta_rule_bwd(
        ctypes.byref(params), _dp(q), _dp(k), _dp(v), _dp(g), _dp(beta), _dp(state_in), _dp(grad_o),
        _dp(grad_state_out), _dp(grad_q), _dp(grad_k), _dp(grad_v), _dp(grad_g), _dp(grad_beta), _dp(grad_state_in),
        _dp(workspace), workspace.numel() * workspace.element_size(), _stream(stream)), "cawn_delta_rule_bwd")


def make_norm_params(N, G, M, eps=1e-5, act=CAWN_NORM_ACT_NONE, rms=False, flags=0, x_stride=0, gate_stride=0):
    return cawn_norm_params(ctypes.sizeof(cawn_norm_params), G, N, M, act, eps, int(rms), flags, 0, x_stride, gate_stride)


def cawn_group_norm_workspace_bytes(params):
    n = ctypes.c_size_t(0)
    _check(lib().cawn_group_norm_workspace_bytes(ctypes.byref(params), ctypes.byref(n)), "cawn_group_norm_workspace_bytes")
    return n.value


def new_norm_workspace(params, device="cuda"):
    """Allocate (with torch, as plain device memory) a workspace for cawn_group_norm_bwd."""
    return _plain_workspace(cawn_group_norm_workspace_bytes(params), device)


def _norm_rows(params, x, gate):
    if params.N > 0:
        width = params.G * params.M
        _check_rows("x_stride", x, width, params.x_stride or width)
        if gate is not None:
            _check_rows("gate_stride", gate, width, params.gate_stride or width)


def cawn_group_norm_fwd(params, x, y, weight=None, bias=None, gate=None, stream=None):
    _dense("y weight bias", y, weight, bias)
    _norm_rows(params, x, gate)
    _check(lib().cawn_group_norm_fwd(ctypes.byref(params), _dp(x), _dp(weight), _dp(bias), _dp(gate), _dp(y),
                                     _stream(stream)), "cawn_group_norm_fwd")


def cawn_group_norm_bwd(params, x, grad_y, grad_x, workspace=None, weight=None, bias=None, gate=None, grad_gate=None,
                        grad_weight=None, grad_bias=None, stream=None):
    _dense("grad_y grad_x weight bias grad_gate grad_weight grad_bias", grad_y, grad_x, weight, bias, grad_gate, grad_weight, grad_bias)
    _norm_rows(params, x, gate)
    n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().cawn_group_norm_bwd(
        ctypes.byref(params), _dp(x), _dp(weight), _dp(bias), _dp(gate), _dp(grad_y), _dp(grad_x), _dp(grad_gate),
        _dp(grad_weight), _dp(grad_bias), _dp(workspace), n, _stream(stream)), "cawn_group_norm_bwd")


def make_dropout_params(n, p, seed, offset=0, flags=0):
    return cawn_dropout_params(ctypes.sizeof(cawn_dropout_params), p, n, seed, offset, flags, 0)


def cawn_dropout(params, x, y, residual=None, offset_device=None, stream=None):
    _dense("x y residual", x, y, residual)
    _check(lib().cawn_dropout(ctypes.byref(params), _dp(x), _dp(residual), _dp(y), _dp(offset_device), _stream(stream)),
           "cawn_dropout")


# ---- operators of a selective state space layer

# The params' fields as they lie (filling a Structure field by field takes twice as long, a fifth of what checking a call does).
_CONV, _SCAN, _RESIDUAL_NORM = struct.Struct("@IiqiiiIIIqq"), struct.Struct("@IiqiiiiIIqqqqqq"), struct.Struct("@IiqfiiiIIq")


def make_conv_params(B, L, C, K, act=CAWN_CONV_ACT_NONE, flags=0, x_stride=0, rows=0):
    try:
        return cawn_conv_params.from_buffer_copy(_CONV.pack(_CONV.size, B, L, C, K, act, flags, 0, 0, x_stride, rows))
    except struct.error:                # a value that does not fit
        return cawn_conv_params(_CONV.size, B, L, C, K, act, flags, (0, 0), x_stride, rows)


_types = None


def _torch_types():
    """torch's float32 and bfloat16, asked for once."""
    global _types
    import torch
    _types = torch.float32, torch.bfloat16
    return _types


def _array(late, name, x, n, kind):
    """Pointer of an array that has to be dense, of one type, and to hold n elements at least.  A layout is refused at once, a type or size
    after all layouts have been looked at: what is wrong goes into `late`."""
    if x is None:
        return None
    try:
        if x.dtype is kind and x.numel() >= n and x.is_contiguous():
            return x.data_ptr()
        if not x.is_contiguous():
            raise ValueError(f"{name}: strides {tuple(x.stride())} of shape {tuple(x.shape)}, it has to be dense")
    except AttributeError:              # not a tensor (a numpy array): its owner's business
        return _dp(x)
    late.append(f"{name}: {tuple(x.shape)} of {x.dtype}, but {n} elements of {kind} are needed")


def _rows(name, x, rows, width, stride, kind):
    """Pointer of an array that has to be so many rows of one type, `stride` (0: width) elements apart.  One row has no step to the next,
    so torch gives that dimension any stride."""
    if x is None:
        return None
    try:                                # the usual cases at once: whole arrays, and slices of a projection
        if x.dtype is kind and (x.is_contiguous() and x.numel() == rows * width if stride == 0 or stride == width
                                else x.stride() == (stride, 1) and x.shape == (rows, width)):
            return x.data_ptr()
        x.is_contiguous
    except AttributeError:
        return _dp(x)
    if rows > 0:
        if x.dtype is not kind:
            raise ValueError(f"{name}: {x.dtype}, but the flags say {kind}")
        _check_sequence_rows(name, x, rows, width, stride or width)
    return x.data_ptr()


def _refuse(late):
    raise ValueError(late[0])


def _row_count(params, offsets):
    """Rows that the arrays of a call have."""
    if offsets is None:
        return params.B * params.L
    _dense("offsets", offsets)
    if hasattr(offsets, "dtype") and (str(offsets.dtype) not in ("torch.int64", "int64") or tuple(offsets.shape) != (params.B + 1,)):
        raise ValueError(f"offsets: {params.B + 1} values of int64 are needed, got {tuple(offsets.shape)} of {offsets.dtype}")
    return params.rows


def _check_sequence_rows(name, x, rows, width, row):
    shape, steps = x.shape, x.stride()
    if len(shape) == 2 and shape[1] == width and shape[0] == rows and steps[1] == 1 and (steps[0] == row or rows == 1):
        return
    if rows > 1:
        _check_rows(name, x, width, row)
    elif width > 1 and shape[-1] > 1 and steps[-1] != 1:
        raise ValueError(f"{name}: strides {tuple(steps)} of shape {tuple(shape)}, a row has to be dense")
    if x.numel() != rows * width:
        raise ValueError(f"{name}: {tuple(shape)} is not {rows} rows of {width} elements")


def cawn_short_conv_workspace_bytes(params):
    n = ctypes.c_size_t(0)
    _check(lib().cawn_short_conv_workspace_bytes(ctypes.byref(params), ctypes.byref(n)), "cawn_short_conv_workspace_bytes")
    return n.value


def new_conv_workspace(params, device="cuda"):
    """Allocate (with torch, as plain device memory) a workspace for cawn_short_conv_bwd."""
    return _plain_workspace(cawn_short_conv_workspace_bytes(params), device)


def cawn_short_conv_fwd(params, x, weight, y, bias=None, state_in=None, state_out=None, offsets=None, stream=None):
    C, K, rows, types, late = params.C, params.K, _row_count(params, offsets), _types or _torch_types(), []
    f, kind, history = types[0], types[params.flags != 0], params.B * (K - 1) * C
    arrays = (_rows("x_stride", x, rows, C, params.x_stride, kind), _array(late, "weight", weight, C * K, f), _array(late, "bias", bias, C, f),
              _array(late, "state_in", state_in, history, f), _dp(offsets), _rows("y", y, rows, C, 0, kind), _array(late, "state_out", state_out, history, f))
    if late:
        _refuse(late)
    _check(lib().cawn_short_conv_fwd(ctypes.byref(params), *arrays, _stream(stream)), "cawn_short_conv_fwd")


def cawn_short_conv_bwd(params, x, weight, grad_y, grad_x, workspace=None, bias=None, state_in=None, offsets=None, grad_state_out=None,
                        grad_weight=None, grad_bias=None, grad_state_in=None, stream=None):
    C, K, rows, types, late = params.C, params.K, _row_count(params, offsets), _types or _torch_types(), []
    f, kind, history = types[0], types[params.flags != 0], params.B * (K - 1) * C
    arrays = (_rows("x_stride", x, rows, C, params.x_stride, kind), _array(late, "weight", weight, C * K, f), _array(late, "bias", bias, C, f),
              _array(late, "state_in", state_in, history, f), _dp(offsets), _rows("grad_y", grad_y, rows, C, 0, kind),
              _array(late, "grad_state_out", grad_state_out, history, f), _rows("grad_x", grad_x, rows, C, 0, kind),
              _array(late, "grad_weight", grad_weight, C * K, f), _array(late, "grad_bias", grad_bias, C, f),
              _array(late, "grad_state_in", grad_state_in, history, f))
    if late:
        _refuse(late)
    n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().cawn_short_conv_bwd(ctypes.byref(params), *arrays, _dp(workspace), n, _stream(stream)), "cawn_short_conv_bwd")


def make_scan_params(B, L, D, N, G=1, softplus=True, flags=0, x_stride=0, dt_stride=0, z_stride=0, b_stride=0, c_stride=0, rows=0):
    values = _SCAN.size, B, L, D, N, G, int(softplus), flags, 0, x_stride, dt_stride, z_stride, b_stride, c_stride, rows
    try:
        return cawn_scan_params.from_buffer_copy(_SCAN.pack(*values))
    except struct.error:
        return cawn_scan_params(*values)


def cawn_selective_scan_workspace_bytes(params, op):
    n = ctypes.c_size_t(0)
    _check(lib().cawn_selective_scan_workspace_bytes(ctypes.byref(params), op, ctypes.byref(n)), "cawn_selective_scan_workspace_bytes")
    return n.value


def new_scan_workspace(params, op, device="cuda"):
    """Allocate (with torch, as plain device memory) a workspace for CAWN_SCAN_FWD, CAWN_SCAN_BWD or CAWN_SCAN_BWD_RECOMPUTE, or the
    checkpoints (CAWN_SCAN_CHECKPOINTS) that a forward leaves for its backward."""
    return _plain_workspace(cawn_selective_scan_workspace_bytes(params, op), device)


def _scan_rows(params, offsets, x, dt, z, B, C, *more):
    """Pointers of the rows of a call, `more`, (name, tensor, width) each, being dense."""
    rows, D, bc, kind = _row_count(params, offsets), params.D, params.G * params.N, (_types or _torch_types())[params.flags != 0]
    return (_rows("x_stride", x, rows, D, params.x_stride, kind), _rows("dt_stride", dt, rows, D, params.dt_stride, kind),
            _rows("z_stride", z, rows, D, params.z_stride, kind), _rows("b_stride", B, rows, bc, params.b_stride, kind),
            _rows("c_stride", C, rows, bc, params.c_stride, kind), *[_rows(name, t, rows, width, 0, kind) for name, t, width in more])


def _scan_checkpoints(params, checkpoints):
    """They carry no size of their own into the call, so it is looked at here."""
    if checkpoints is not None and hasattr(checkpoints, "numel"):
        _dense("checkpoints", checkpoints)
        need = cawn_selective_scan_workspace_bytes(params, CAWN_SCAN_CHECKPOINTS)
        if checkpoints.numel() * checkpoints.element_size() < need:
            raise ValueError(f"checkpoints: {checkpoints.numel() * checkpoints.element_size()} bytes, {need} are needed")


def cawn_selective_scan_fwd(params, x, dt, A, B, C, y, workspace=None, skip=None, dt_bias=None, z=None, state_in=None, state_out=None,
                            offsets=None, checkpoints=None, stream=None):
    _scan_checkpoints(params, checkpoints)
    D, f, late = params.D, (_types or _torch_types())[0], []
    rates = D * params.N
    states = params.B * rates
    x, dt, z, B, C, y = _scan_rows(params, offsets, x, dt, z, B, C, ("y", y, D))
    arrays = (x, dt, _array(late, "A", A, rates, f), B, C, _array(late, "skip", skip, D, f), _array(late, "dt_bias", dt_bias, D, f), z,
              _array(late, "state_in", state_in, states, f), _dp(offsets), y, _array(late, "state_out", state_out, states, f))
    if late:
        _refuse(late)
    n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().cawn_selective_scan_fwd(ctypes.byref(params), *arrays, _dp(checkpoints), _dp(workspace), n, _stream(stream)), "cawn_selective_scan_fwd")


def cawn_selective_scan_step(params, x, dt, A, B, C, y, skip=None, dt_bias=None, z=None, state_in=None, state_out=None, stream=None):
    types, late, batch, D, N = _types or _torch_types(), [], params.B, params.D, params.N
    f, kind, rows, bc, states = types[0], types[params.flags != 0], batch * params.L, params.G * N, batch * D * N
    # as _scan_rows, without the calls in between: a single token's call is half as long as its checks
    arrays = (_rows("x_stride", x, rows, D, params.x_stride, kind), _rows("dt_stride", dt, rows, D, params.dt_stride, kind), _array(late, "A", A, D * N, f),
              _rows("b_stride", B, rows, bc, params.b_stride, kind), _rows("c_stride", C, rows, bc, params.c_stride, kind), _array(late, "skip", skip, D, f),
              _array(late, "dt_bias", dt_bias, D, f), _rows("z_stride", z, rows, D, params.z_stride, kind), _array(late, "state_in", state_in, states, f),
              _rows("y", y, rows, D, 0, kind), _array(late, "state_out", state_out, states, f))
    if late:
        _refuse(late)
    _check(lib().cawn_selective_scan_step(ctypes.byref(params), *arrays, _stream(stream)), "cawn_selective_scan_step")


def cawn_selective_scan_bwd(params, x, dt, A, B, C, grad_y, grad_x, grad_dt, grad_A, grad_B, grad_C, workspace, skip=None, dt_bias=None, z=None,
                            state_in=None, offsets=None, checkpoints=None, grad_state_out=None, grad_skip=None, grad_dt_bias=None, grad_z=None,
                            grad_state_in=None, stream=None):
    _scan_checkpoints(params, checkpoints)
    D, bc, f, late = params.D, params.G * params.N, (_types or _torch_types())[0], []
    rates = D * params.N
    states = params.B * rates
    x, dt, z, B, C, grad_y, grad_x, grad_dt, grad_B, grad_C, grad_z = _scan_rows(
        params, offsets, x, dt, z, B, C, ("grad_y", grad_y, D), ("grad_x", grad_x, D), ("grad_dt", grad_dt, D), ("grad_B", grad_B, bc), ("grad_C", grad_C, bc),
        ("grad_z", grad_z, D))
    arrays = (x, dt, _array(late, "A", A, rates, f), B, C, _array(late, "skip", skip, D, f), _array(late, "dt_bias", dt_bias, D, f), z,
              _array(late, "state_in", state_in, states, f), _dp(offsets), _dp(checkpoints), grad_y, _array(late, "grad_state_out", grad_state_out, states, f),
              grad_x, grad_dt, _array(late, "grad_A", grad_A, rates, f), grad_B, grad_C, _array(late, "grad_skip", grad_skip, D, f),
              _array(late, "grad_dt_bias", grad_dt_bias, D, f), grad_z, _array(late, "grad_state_in", grad_state_in, states, f))
    if late:
        _refuse(late)
    _check(lib().cawn_selective_scan_bwd(ctypes.byref(params), *arrays, _dp(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "cawn_selective_scan_bwd")


def make_residual_norm_params(N, M, eps=1e-5, out=CAWN_NORM_OUT_SAME, scale_block=0, stream_float=False, flags=0, x_stride=0):
    values = _RESIDUAL_NORM.size, M, N, eps, out, scale_block, int(stream_float), flags, 0, x_stride
    try:
        return cawn_residual_norm_params.from_buffer_copy(_RESIDUAL_NORM.pack(*values))
    except (struct.error, OverflowError):
        return cawn_residual_norm_params(*values)


def cawn_residual_norm_workspace_bytes(params):
    n = ctypes.c_size_t(0)
    _check(lib().cawn_residual_norm_workspace_bytes(ctypes.byref(params), ctypes.byref(n)), "cawn_residual_norm_workspace_bytes")
    return n.value


def new_residual_norm_workspace(params, device="cuda"):
    """Allocate (with torch, as plain device memory) a workspace for cawn_residual_norm_bwd."""
    return _plain_workspace(cawn_residual_norm_workspace_bytes(params), device)


def _norm_types(params):
    """float32, and the types of the rows and of the stream."""
    f, b = _types or _torch_types()
    return (f, b, f if params.stream_float else b) if params.flags else (f, f, f)


def _norm_rows_in(late, x, rows, M, stride, kind):
    """Pointer of the norm's input: at least so many rows, `stride` (0: M) elements apart."""
    n = rows * M
    try:
        if x.dtype is kind and x.numel() >= n and (stride == 0 or stride == M) and x.is_contiguous():
            return x.data_ptr()
        if n > 0:
            _check_rows("x_stride", x, M, stride or M)
            if x.dtype is not kind or x.numel() < n:
                late.append(f"x: {tuple(x.shape)} of {x.dtype}, but {n} elements of {kind} are needed")
    except AttributeError:
        pass
    return _dp(x)


def cawn_residual_norm_fwd(params, x, y, residual=None, weight=None, sum_out=None, scales=None, stream=None):
    f, kind, of_stream = _norm_types(params)
    rows, M, late = params.N, params.M, []
    n, out, cols = rows * M, kind, 1
    if params.out == CAWN_NORM_OUT_E4M3:
        out = getattr(y, "dtype", None)             # any type of one byte
        if hasattr(y, "element_size") and y.element_size() != 1:
            raise ValueError(f"y: {out}, but values of 8 bits are written")
        cols = -(-M // params.scale_block) if params.scale_block > 0 else 1
    arrays = (_norm_rows_in(late, x, rows, M, params.x_stride, kind), _array(late, "residual", residual, n, of_stream), _array(late, "weight", weight, M, f),
              _array(late, "sum_out", sum_out, n, of_stream), _array(late, "y", y, n, out), _array(late, "scales", scales, rows * cols, f))
    if late:
        _refuse(late)
    _check(lib().cawn_residual_norm_fwd(ctypes.byref(params), *arrays, _stream(stream)), "cawn_residual_norm_fwd")


def cawn_residual_norm_bwd(params, sum, grad_y, workspace=None, weight=None, grad_sum=None, grad_residual=None, grad_x=None, grad_weight=None,
                           stream=None):
    f, kind, of_stream = _norm_types(params)
    M, n, late = params.M, params.N * params.M, []
    arrays = (_array(late, "sum", sum, n, of_stream), _array(late, "weight", weight, M, f), _array(late, "grad_y", grad_y, n, kind),
              _array(late, "grad_sum", grad_sum, n, of_stream), _array(late, "grad_residual", grad_residual, n, of_stream),
              _array(late, "grad_x", grad_x, n, kind), _array(late, "grad_weight", grad_weight, M, f))
    if late:
        _refuse(late)
    n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().cawn_residual_norm_bwd(ctypes.byref(params), *arrays, _dp(workspace), n, _stream(stream)), "cawn_residual_norm_bwd")
