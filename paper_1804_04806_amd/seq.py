"""ctypes binding of the sequence operators: the same entry points as include/ucd_seq.h, argument
marshalling only.  Device buffers are torch tensors (their ``data_ptr()``), raw integer addresses or
None; the library is the one ``ucd.lib()`` loads.  Kernels are launched on the current device, which has to be the
buffers', and by default on its current stream.
"""
import ctypes
import struct

from . import ucd

FWD, BWD = 0, 1
ACT_NONE, ACT_SILU = 0, 1

EXPORTS = [
    "ucd_group_norm_workspace_size", "ucd_group_norm_fwd", "ucd_group_norm_bwd",
    "ucd_causal_conv_workspace_size", "ucd_causal_conv_fwd", "ucd_causal_conv_bwd", "ucd_causal_conv_step",
    "ucd_scan_workspace_size", "ucd_scan_saved_size", "ucd_scan_fwd", "ucd_scan_bwd", "ucd_scan_step",
]

_I32, _I64, _P = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class GroupNormDesc(ctypes.Structure):
    """ucd_group_norm_t"""
    _fields_ = [(n, _I32) for n in ("N", "S", "C", "G", "act", "dtype")] + [("eps", ctypes.c_float)] + \
        [(n, _I64) for n in ("x_n", "x_s", "y_n", "y_s")]


class CausalConvDesc(ctypes.Structure):
    """ucd_causal_conv_t"""
    _fields_ = [(n, _I32) for n in ("B", "L", "D", "K", "act", "dtype", "n_slots")] + \
        [(n, _I64) for n in ("x_b", "x_l", "y_b", "y_l")]


class ScanDesc(ctypes.Structure):
    """ucd_scan_t"""
    _fields_ = [(n, _I32) for n in ("B", "L", "D", "N", "G", "dtype", "softplus", "n_slots")] + \
        [(f"{n}_{k}", _I64) for n in ("u", "dt", "Bm", "Cm", "z", "y") for k in ("b", "l")]


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = ucd.lib()
        sz, i, f = ctypes.c_size_t, ctypes.c_int, ctypes.c_float
        gp, cp, sp = (ctypes.POINTER(t) for t in (GroupNormDesc, CausalConvDesc, ScanDesc))
        L.ucd_group_norm_workspace_size.restype = sz
        L.ucd_group_norm_workspace_size.argtypes = [gp, i]
        L.ucd_group_norm_fwd.argtypes = [gp, _P, _P, _P, _P, _P, _P, sz, _P]
        L.ucd_group_norm_bwd.argtypes = [gp, _P, _P, _P, _P, _P, _P, _P, _P, f, _P, sz, _P]
        L.ucd_causal_conv_workspace_size.restype = sz
        L.ucd_causal_conv_workspace_size.argtypes = [cp]
        L.ucd_causal_conv_fwd.argtypes = [cp] + [_P] * 9
        L.ucd_causal_conv_bwd.argtypes = [cp] + [_P] * 11 + [f, _P, sz, _P]
        L.ucd_causal_conv_step.argtypes = [cp] + [_P] * 7
        L.ucd_scan_workspace_size.restype = sz
        L.ucd_scan_workspace_size.argtypes = [sp, i]
        L.ucd_scan_saved_size.restype = sz
        L.ucd_scan_saved_size.argtypes = [sp]
        L.ucd_scan_fwd.argtypes = [sp, _P, _P, _P, _P, _P, sz, _P, sz, _P]
        L.ucd_scan_bwd.argtypes = [sp, _P, _P, _P, _P, sz, _P, f, _P, sz, _P]
        L.ucd_scan_step.argtypes = [sp, _P, _P, _P, _P]
        _lib = L
    return _lib


# A step of one sequence takes the GPU two or three microseconds, and these calls hardly more: addresses are read
# without more checks than for None and int, ucd_scan_in_t and ucd_scan_grad_t are packed as bytes, and the current stream is asked for by its raw handle.
_pack_in, _pack_grad = struct.Struct("10P").pack, struct.Struct("9P").pack


def _ptr(t):
    """Device address of a torch tensor, or an int passed through; 0 for None."""
    return 0 if t is None else t if t.__class__ is int else t.data_ptr()


def _raw_stream():
    """The current stream of the current device; from the second call on without a look at whether the GPU is in use at all."""
    global _raw_stream
    import torch
    torch.cuda.current_device()
    device, current = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

    def _raw_stream():
        return current(device())
    return _raw_stream()


def _stream(stream):
    return _raw_stream() if stream is None else ucd._stream(stream)


def _bytes(t, nbytes):
    return nbytes if nbytes is not None else 0 if t is None else t.numel() * t.element_size()


def _check(status, where):
    if status != ucd.OK:
        raise ucd.UcdError(status, where)


def group_norm(N, S, C, G, act=ACT_NONE, dtype=0, eps=1e-5, x_stride=(0, 0), y_stride=(0, 0)):
    """GroupNormDesc.  Strides (sample, position) in elements; 0 is the dense one.  dtype 0: fp32 activations, 1: bf16."""
    return GroupNormDesc(N, S, C, G, act, dtype, eps, *x_stride, *y_stride)


def causal_conv(B, L, D, K, act=ACT_NONE, dtype=0, n_slots=0, x_stride=(0, 0), y_stride=(0, 0)):
    """CausalConvDesc.  Strides (sequence, token) in elements; 0 is the dense one."""
    return CausalConvDesc(B, L, D, K, act, dtype, n_slots, *x_stride, *y_stride)


def scan(B, L, D, N, G=1, dtype=0, softplus=True, n_slots=0, u_stride=(0, 0), dt_stride=(0, 0), Bm_stride=(0, 0),
         Cm_stride=(0, 0), z_stride=(0, 0), y_stride=(0, 0)):
    """ScanDesc.  Strides (sequence, token) in elements; 0 is the dense one."""
    return ScanDesc(B, L, D, N, G, dtype, int(softplus), n_slots, *u_stride, *dt_stride, *Bm_stride, *Cm_stride, *z_stride,
                    *y_stride)


def ucd_group_norm_workspace_size(desc, direction):
    return lib().ucd_group_norm_workspace_size(desc, direction)


def ucd_group_norm_fwd(desc, x, gamma, beta_w, y, stats=None, ws=None, ws_bytes=None, stream=None):
    _check((_lib or lib()).ucd_group_norm_fwd(
        desc, _ptr(x), _ptr(gamma), _ptr(beta_w), _ptr(y), _ptr(stats), _ptr(ws), _bytes(ws, ws_bytes), _stream(stream)),
        "ucd_group_norm_fwd")


def ucd_group_norm_bwd(desc, x, gamma, beta_w, stats, dy, dx, dgamma, dbeta, beta=0.0, ws=None, ws_bytes=None, stream=None):
    _check((_lib or lib()).ucd_group_norm_bwd(
        desc, _ptr(x), _ptr(gamma), _ptr(beta_w), _ptr(stats), _ptr(dy), _ptr(dx), _ptr(dgamma), _ptr(dbeta), beta, _ptr(ws),
        _bytes(ws, ws_bytes), _stream(stream)), "ucd_group_norm_bwd")


def ucd_causal_conv_workspace_size(desc):
    return lib().ucd_causal_conv_workspace_size(desc)


def ucd_causal_conv_fwd(desc, x, w, bias, y, lengths=None, slots=None, state_in=None, state_out=None, stream=None):
    _check((_lib or lib()).ucd_causal_conv_fwd(
        desc, _ptr(x), _ptr(w), _ptr(bias), _ptr(lengths), _ptr(slots), _ptr(state_in), _ptr(state_out), _ptr(y),
        _stream(stream)), "ucd_causal_conv_fwd")


def ucd_causal_conv_bwd(desc, x, w, bias, dy, dx, dw, dbias, lengths=None, state_in=None, dstate_out=None, dstate_in=None,
                        beta=0.0, ws=None, ws_bytes=None, stream=None):
    _check((_lib or lib()).ucd_causal_conv_bwd(
        desc, _ptr(x), _ptr(w), _ptr(bias), _ptr(lengths), _ptr(state_in), _ptr(dy), _ptr(dstate_out), _ptr(dx), _ptr(dw),
        _ptr(dbias), _ptr(dstate_in), beta, _ptr(ws), _bytes(ws, ws_bytes), _stream(stream)), "ucd_causal_conv_bwd")


def ucd_causal_conv_step(desc, x, w, bias, state, y, slots=None, stream=None):
    _check((_lib or lib()).ucd_causal_conv_step(
        desc, _ptr(x), _ptr(w), _ptr(bias), _ptr(slots), _ptr(state), _ptr(y), _stream(stream)), "ucd_causal_conv_step")


def ucd_scan_workspace_size(desc, direction):
    return lib().ucd_scan_workspace_size(desc, direction)


def ucd_scan_saved_size(desc):
    return lib().ucd_scan_saved_size(desc)


def ucd_scan_fwd(desc, u, dt, A, Bm, Cm, y, skip=None, z=None, dt_bias=None, lengths=None, slots=None, state_in=None,
                 state_out=None, saved=None, saved_bytes=None, ws=None, ws_bytes=None, stream=None):
    given = _pack_in(_ptr(u), _ptr(dt), _ptr(A), _ptr(Bm), _ptr(Cm), _ptr(skip), _ptr(z), _ptr(dt_bias), _ptr(lengths),
                     _ptr(slots))
    _check((_lib or lib()).ucd_scan_fwd(
        desc, given, _ptr(state_in), _ptr(state_out), _ptr(y), _ptr(saved), _bytes(saved, saved_bytes), _ptr(ws),
        _bytes(ws, ws_bytes), _stream(stream)), "ucd_scan_fwd")


def ucd_scan_bwd(desc, u, dt, A, Bm, Cm, dy, saved, du, ddt, dA, dBm, dCm, skip=None, dskip=None, z=None, dz=None,
                 dt_bias=None, ddt_bias=None, lengths=None, dstate_out=None, dstate_in=None, beta=0.0, saved_bytes=None,
                 ws=None, ws_bytes=None, stream=None):
    given = _pack_in(_ptr(u), _ptr(dt), _ptr(A), _ptr(Bm), _ptr(Cm), _ptr(skip), _ptr(z), _ptr(dt_bias), _ptr(lengths), 0)
    grad = _pack_grad(_ptr(du), _ptr(ddt), _ptr(dA), _ptr(dBm), _ptr(dCm), _ptr(dskip), _ptr(dz), _ptr(ddt_bias),
                      _ptr(dstate_in))
    _check((_lib or lib()).ucd_scan_bwd(
        desc, given, _ptr(dy), _ptr(dstate_out), _ptr(saved), _bytes(saved, saved_bytes), grad, beta, _ptr(ws),
        _bytes(ws, ws_bytes), _stream(stream)), "ucd_scan_bwd")


def ucd_scan_step(desc, u, dt, A, Bm, Cm, state, y, skip=None, z=None, dt_bias=None, slots=None, stream=None):
    given = _pack_in(_ptr(u), _ptr(dt), _ptr(A), _ptr(Bm), _ptr(Cm), _ptr(skip), _ptr(z), _ptr(dt_bias), 0, _ptr(slots))
    _check((_lib or lib()).ucd_scan_step(desc, given, _ptr(state), _ptr(y), _stream(stream)), "ucd_scan_step")
