"""Python binding of libfpo (include/fpo.h): the GB300 pseudogradient update of
Forward-Pass-Only MLP training.

Argument marshalling only: every function here passes device pointers, sizes
and the current CUDA stream to the C entry point of the same name; every step
of the computation runs in libfpo's CUDA kernels.  PyTorch supplies device
memory and streams.  There is no CPU fallback: importing this package fails
loudly when ``libfpo.so`` has not been built (``python -m
paper_2608_14563_gb300.build`` or ``__graft_entry__.build()``).
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfpo.so")

F32, BF16 = 0, 1
OK = 0
MAX_GROUPED_LAYERS = 64
STAGE_EVENTS = 7
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
ES_AUTO, ES_RECOMPUTE, ES_STORED_LOGITS, ES_DIRECT = 0, 1, 2, 3
AUTO_T_CHUNK = 8192  # FPO_AUTO_T_CHUNK: tokens per error-matrix chunk when t_chunk is 0

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libfpo.so is not built ({LIB_PATH} missing); run "
                      "`python -m paper_2608_14563_gb300.build` first")
_lib = ctypes.CDLL(LIB_PATH)
ABI_VERSION = 2  # FPO_ABI_VERSION of include/fpo.h that the structures below mirror
_lib.fpo_abi_version.restype = ctypes.c_int32
if _lib.fpo_abi_version() != ABI_VERSION:
    raise ImportError(f"libfpo.so reports ABI version {_lib.fpo_abi_version()}, this binding "
                      f"needs {ABI_VERSION}; rebuild it (`python -m paper_2608_14563_gb300.build`)")

_vp, _i64, _i32, _f32, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float,
                              ctypes.c_size_t)
_f64 = ctypes.c_double


class ErrorSignalDesc(ctypes.Structure):
    """Mirror of fpo_error_signal_desc."""
    _fields_ = [("T", _i64), ("d", _i64), ("V", _i64), ("dtype", _i32), ("eps", _f32),
                ("min_rms", _f32), ("loss_scale", _f32), ("algo", _i32), ("t_chunk", _i64),
                ("stage_events", ctypes.POINTER(_vp)), ("stage_events_per_chunk", _i32)]


_lib.fpo_abi_version.restype = _i32
_lib.fpo_status_string.argtypes = [_i32]
_lib.fpo_status_string.restype = ctypes.c_char_p
_lib.fpo_set_wait_limit_ns.argtypes = [ctypes.c_uint64]
_lib.fpo_set_wait_limit_ns.restype = None
_lib.fpo_error_signal_stage_events.argtypes = [ctypes.POINTER(ErrorSignalDesc)]
_lib.fpo_error_signal_stage_events.restype = _i32
_lib.fpo_error_signal_workspace.argtypes = [ctypes.POINTER(ErrorSignalDesc)]
_lib.fpo_error_signal_workspace.restype = _sz
_lib.fpo_error_signal.argtypes = [ctypes.POINTER(ErrorSignalDesc), _vp, _vp, _vp, _vp, _vp, _vp,
                                  _vp, _vp, _sz, _vp]
_lib.fpo_error_signal.restype = _i32
_lib.fpo_layer_update_workspace.argtypes = []
_lib.fpo_layer_update_workspace.restype = _sz
_lib.fpo_layer_update.argtypes = [_i64, _i64, _i64, _i32, _vp, _vp, _f32, _vp, _vp, _vp, _vp,
                                  _sz, _vp]
_lib.fpo_layer_update.restype = _i32
_lib.fpo_layer_update_grouped.argtypes = [_i32, _i64, _i64, _i64, _i32, _vp,
                                          ctypes.POINTER(_vp), _f32, ctypes.POINTER(_vp),
                                          ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, _sz, _vp]
_lib.fpo_layer_update_grouped.restype = _i32
_lib.fpo_layer_update_grouped_signals.argtypes = [_i32, _i64, _i64, _i64, _i32,
                                                  ctypes.POINTER(_vp), ctypes.POINTER(_vp), _f32,
                                                  ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                                  ctypes.POINTER(_vp), _vp, _sz, _vp]
_lib.fpo_layer_update_grouped_signals.restype = _i32
_lib.fpo_rmsnorm_vjp.argtypes = [_i64, _i64, _i32, _vp, _vp, _vp, _f32, _f32, _vp, _vp]
_lib.fpo_rmsnorm_vjp.restype = _i32
_lib.fpo_layer_signals.argtypes = [_i32, _i64, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _f32, _f32,
                                   _vp, _vp]
_lib.fpo_layer_signals.restype = _i32

_lib.fpo_layernorm.argtypes = [_i64, _i64, _i32, _vp, _vp, _vp, _f32, _vp, _vp, _vp, _vp]
_lib.fpo_layernorm.restype = _i32
_lib.fpo_layernorm_vjp_workspace.argtypes = [_i64, _i64, _i32]
_lib.fpo_layernorm_vjp_workspace.restype = _sz
_lib.fpo_layernorm_vjp.argtypes = [_i64, _i64, _i32, _vp, _vp, _vp, _f32, _f32, _vp, _vp, _vp, _vp,
                                   _sz, _vp]
_lib.fpo_layernorm_vjp.restype = _i32


class OptimizerDesc(ctypes.Structure):
    """Mirror of fpo_optimizer_desc."""
    _fields_ = [("kind", _i32), ("clip", _i32), ("lr", _f32), ("momentum", _f32),
                ("beta1", _f32), ("beta2", _f32), ("adam_eps", _f32), ("weight_decay", _f32),
                ("clip_frac", _f32), ("step", _i64)]


OPT_SGD, OPT_SGD_MOMENTUM, OPT_ADAMW = 0, 1, 2
CLIP_NONE, CLIP_STEP, CLIP_GRADIENT = 0, 1, 2
_lib.fpo_layer_optimize_workspace.argtypes = [_i32, _i64, _i64]
_lib.fpo_layer_optimize_workspace.restype = _sz
_lib.fpo_layer_optimize_grouped.argtypes = [_i32, _i64, _i64, _i64, _i32, ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), ctypes.POINTER(OptimizerDesc),
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, _sz, _vp]
_lib.fpo_layer_optimize_grouped.restype = _i32


_lib.fpo_linear_workspace.argtypes = [_i64, _i64, _i64, _i32]
_lib.fpo_linear_workspace.restype = _sz
_lib.fpo_linear.argtypes = [_i64, _i64, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.fpo_linear.restype = _i32
_lib.fpo_linear_vjp_workspace.argtypes = [_i64, _i64, _i64, _i32, _i32]
_lib.fpo_linear_vjp_workspace.restype = _sz
_lib.fpo_linear_vjp.argtypes = [_i64, _i64, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp,
                                _vp, _vp, _sz, _vp]
_lib.fpo_linear_vjp.restype = _i32


class AdamwTensor(ctypes.Structure):
    """Mirror of fpo_adamw_tensor."""
    _fields_ = [("n", _i64), ("G", _vp), ("W_master", _vp), ("W_out", _vp), ("state1", _vp),
                ("state2", _vp), ("scale1", _vp), ("scale2", _vp), ("g_dtype", _i32),
                ("w_dtype", _i32), ("state_bits", _i32), ("weight_decay", _f32)]


_ADAMW_TENSOR = struct.Struct("@q7Piiif")  # the same, packed
assert _ADAMW_TENSOR.size == ctypes.sizeof(AdamwTensor)


class AdamwDesc(ctypes.Structure):
    """Mirror of fpo_adamw_desc."""
    _fields_ = [("lr", _f64), ("beta1", _f64), ("beta2", _f64), ("eps", _f64), ("clip_frac", _f64),
                ("step", _i64), ("clip", _i32)]


ADAMW_BLOCK = 256  # FPO_ADAMW_BLOCK: elements that share the scales of their 8-bit moments
_lib.fpo_adamw_workspace.argtypes = [_i32, ctypes.POINTER(_i64), _i32]
_lib.fpo_adamw_workspace.restype = _sz
_lib.fpo_adamw_grouped.argtypes = [_i32, ctypes.POINTER(AdamwTensor), ctypes.POINTER(AdamwDesc),
                                   ctypes.c_uint64, _vp, _sz, _vp]
_lib.fpo_adamw_grouped.restype = _i32
_lib.fpo_adamw_state_values.argtypes = [_i64, _i32, _vp, _vp, _i32, _vp, _vp]
_lib.fpo_adamw_state_values.restype = _i32


class MuonDesc(ctypes.Structure):
    """Mirror of fpo_muon_desc."""
    _fields_ = [("lr", _f32), ("momentum", _f32), ("weight_decay", _f32), ("scale", _f32),
                ("eps", _f32), ("nesterov", _i32), ("steps", _i32),
                ("coeffs", ctypes.POINTER(_f32))]


_lib.fpo_orthogonalize_workspace.argtypes = [_i32, _i64, _i64, _i32]
_lib.fpo_orthogonalize_workspace.restype = _sz
_lib.fpo_orthogonalize_grouped.argtypes = [_i32, _i64, _i64, _i32, ctypes.POINTER(_vp), _i32,
                                           ctypes.POINTER(_f32), _f32, ctypes.POINTER(_vp), _vp,
                                           _sz, _vp]
_lib.fpo_orthogonalize_grouped.restype = _i32
_lib.fpo_layer_muon_workspace.argtypes = [_i32, _i64, _i64, _i32]
_lib.fpo_layer_muon_workspace.restype = _sz
_lib.fpo_layer_muon_grouped.argtypes = [_i32, _i64, _i64, _i64, _i32, ctypes.POINTER(_vp),
                                        ctypes.POINTER(_vp), ctypes.POINTER(MuonDesc),
                                        ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                        ctypes.POINTER(_vp), _vp, _sz, _vp]
_lib.fpo_layer_muon_grouped.restype = _i32
_lib.fpo_gate_up_signals.argtypes = [_i64, _i64, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                     _sz, _vp]
_lib.fpo_gate_up_signals.restype = _i32
_lib.fpo_cosine_workspace.argtypes = [_i64]
_lib.fpo_cosine_workspace.restype = _sz
_lib.fpo_cosine.argtypes = [_i64, _i32, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.fpo_cosine.restype = _i32
_lib.fpo_get_device_status.argtypes = [_vp, _vp]
_lib.fpo_get_device_status.restype = _i32
_lib.fpo_cosine_grouped_workspace.argtypes = [_i32, _i64]
_lib.fpo_cosine_grouped_workspace.restype = _sz
_lib.fpo_cosine_grouped.argtypes = [_i32, _i64, _i32, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                    _vp, _vp, _sz, _vp]
_lib.fpo_cosine_grouped.restype = _i32
_lib.fpo_layer_grad_cosine_workspace.argtypes = [_i32, _i64, _i64]
_lib.fpo_layer_grad_cosine_workspace.restype = _sz
_lib.fpo_layer_grad_cosine_grouped.argtypes = [_i32, _i64, _i64, _i64, _i32, _vp,
                                               ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                               ctypes.POINTER(_vp), _vp, _vp, _sz, _vp]
_lib.fpo_layer_grad_cosine_grouped.restype = _i32
_lib.fpo_norm_ratio_workspace.argtypes = [_i32, _i64]
_lib.fpo_norm_ratio_workspace.restype = _sz
_lib.fpo_norm_ratio.argtypes = [_i32, _i64, _i32, ctypes.POINTER(_vp), _i32, ctypes.POINTER(_vp),
                                ctypes.c_double, _vp, _vp, _sz, _vp]
_lib.fpo_norm_ratio.restype = _i32
_lib.fpo_h2d_copy.argtypes = [_i32, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                              ctypes.POINTER(_sz), _vp]
_lib.fpo_h2d_copy.restype = _i32
_lib.fpo_testing_direct_fixup_rows.argtypes = [ctypes.POINTER(ErrorSignalDesc), _vp, _vp]
_lib.fpo_testing_direct_fixup_rows.restype = _i64
_lib.fpo_testing_kernel_launches.argtypes = []
_lib.fpo_testing_kernel_launches.restype = ctypes.c_uint64
_lib.fpo_testing_set_gemm_variant.argtypes = [_i32]
_lib.fpo_testing_set_gemm_variant.restype = _i32


class FpoError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {status_string(code)}")
        self.code = code


def status_string(code: int) -> str:
    return _lib.fpo_status_string(int(code)).decode()


def abi_version() -> int:
    return _lib.fpo_abi_version()


def set_wait_limit_ns(ns: int) -> None:
    _lib.fpo_set_wait_limit_ns(int(ns))


def kernel_launches() -> int:
    """fpo_testing_kernel_launches: kernels this library has launched in this process."""
    return int(_lib.fpo_testing_kernel_launches())


def set_gemm_variant(variant: int) -> int:
    """fpo_testing_set_gemm_variant: 0 single-CTA, 1 CTA-pair tiles, 2 CTA-pair tiles with a
    256 x 512 projection (the default); a negative value only reads the current setting.  Returns the setting in
    force before the call."""
    if variant < 0:
        cur = _lib.fpo_testing_set_gemm_variant(0)
        _lib.fpo_testing_set_gemm_variant(cur)
        return cur
    return _lib.fpo_testing_set_gemm_variant(int(variant))


def set_simt_tile(tile: int) -> int:
    """fpo_testing_set_simt_tile: fp32 GEMM tiles of 128 or 64, 0 for the estimated faster
    (the default).  Returns the setting in force before the call."""
    return _lib.fpo_testing_set_simt_tile(int(tile))


def _check(code: int, where: str) -> None:
    if code != OK:
        raise FpoError(code, where)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on_current_device(t: torch.Tensor) -> None:
    """Kernels run on the current device, where another one's memory may not be mapped."""
    device = t.get_device()  # -1: not CUDA memory, which _ptr refuses
    if device >= 0 and device != _current_device():
        raise ValueError(f"libfpo runs on the current device, cuda:{_current_device()}; "
                         f"got a tensor of cuda:{device}")


def _dtype_code(t: torch.Tensor) -> int:
    """The type of a call, that of its leading tensor."""
    _on_current_device(t)
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}; libfpo takes bfloat16 or float32")


def _ptr(t):
    # an int: ctypes passes it through a c_void_p argument or array slot
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libfpo takes CUDA tensors")
    if not t.is_contiguous():
        raise ValueError("libfpo takes contiguous tensors")
    return t.data_ptr()


_is_contiguous, _data_ptr, _numel = (
    torch.Tensor.is_contiguous, torch.Tensor.data_ptr, torch.Tensor.numel)


def _ptrs(ts):
    """_ptr of every entry of a list (0 for None), all on the current device."""
    some = [t for t in ts if t is not None]
    devices = {t.get_device() for t in some}
    if (len(devices) > 1 or -1 in devices or devices - {_current_device()}
            or not all(map(_is_contiguous, some))):
        for t in some:
            _on_current_device(t)
            _ptr(t)
    ptrs = list(map(_data_ptr, some))
    if len(some) == len(ts):
        return ptrs
    it = iter(ptrs)
    return [0 if t is None else next(it) for t in ts]


# torch's private call for a stream's handle, where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without building a torch Stream object (3 us a call, a
    # tenth of the host time of a small step)
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A tensor that belongs to the stream the call runs on.  Taken on the current stream while the
    call is given another one, its memory could still be in use by earlier work of the current
    stream, and would go to the next allocation there while the call's kernels still run."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):  # anything with a handle
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _workspace(nbytes: int, device, stream) -> torch.Tensor:
    return _empty(max(int(nbytes), 256), torch.uint8, device, stream)


def _result(shape, device, stream) -> torch.Tensor:
    """An fp64 result that the caller will read, also on the current stream."""
    t = _empty(shape, torch.float64, device, stream)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _expect(t, shape, dtype, name):
    """The C entry points see pointers only: a tensor's shape and type are checked here."""
    if t is not None and (t.shape != shape or t.dtype != dtype):
        raise ValueError(f"{name}: expected {dtype} of shape {tuple(shape)}, "
                         f"got {t.dtype} of {tuple(t.shape)}")


# --------------------------------------------------------------------------- error signal
def error_signal_desc(T, d, V, dtype=BF16, *, eps=1e-6, min_rms=0.5, loss_scale=None, t_chunk=0,
                      stage_events=None, algo=ES_AUTO, per_chunk_events=False):
    """fpo_error_signal_desc; ``stage_events`` is None or torch.cuda.Event objects that have
    been recorded once (so their CUDA handles exist): STAGE_EVENTS of them, or with
    ``per_chunk_events`` stage_event_count() of them (every token chunk's stages)."""
    s = (1.0 / T if T > 0 else 1.0) if loss_scale is None else loss_scale
    d = ErrorSignalDesc(int(T), int(d), int(V), int(dtype), float(eps), float(min_rms), float(s),
                        int(algo), int(t_chunk), None, 1 if per_chunk_events else 0)
    if stage_events is not None:
        need = stage_event_count(d)
        if len(stage_events) != need:
            raise ValueError(f"stage_events needs {need} events")
        ev = (_vp * need)(*[e.cuda_event for e in stage_events])
        d.stage_events = ctypes.cast(ev, ctypes.POINTER(_vp))
        d._keep = ev
    return d


def stage_event_count(desc: ErrorSignalDesc) -> int:
    """fpo_error_signal_stage_events: events the descriptor's stage-event layout needs."""
    return int(_lib.fpo_error_signal_stage_events(ctypes.byref(desc)))


def error_signal_workspace(desc: ErrorSignalDesc) -> int:
    return int(_lib.fpo_error_signal_workspace(ctypes.byref(desc)))


def error_signal(h, norm_w, W_U, targets, g_out, *, eps=1e-6, min_rms=0.5, loss_scale=None,
                 t_chunk=0, lse_out=None, loss_out=None, workspace=None, stream=None,
                 stage_events=None, algo=ES_AUTO, per_chunk_events=False):
    """fpo_error_signal: g~ = final-RMSNorm VJP of (softmax(z) - 1_y) W_U into ``g_out``.

    Returns the workspace tensor (its first word holds the device status).
    """
    T, d = h.shape
    V = W_U.shape[0]
    desc = error_signal_desc(T, d, V, _dtype_code(h), eps=eps, min_rms=min_rms,
                             loss_scale=loss_scale, t_chunk=t_chunk, stage_events=stage_events,
                             algo=algo, per_chunk_events=per_chunk_events)
    if workspace is None:
        workspace = _workspace(error_signal_workspace(desc), h.device, stream)
    rc = _lib.fpo_error_signal(ctypes.byref(desc), _ptr(h), _ptr(norm_w), _ptr(W_U), _ptr(targets),
                               _ptr(g_out), _ptr(lse_out), _ptr(loss_out), _ptr(workspace),
                               _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_error_signal")
    return workspace


def direct_fixup_rows(h, W_U, workspace, *, t_chunk=0, algo=ES_AUTO, stream=None) -> int:
    """fpo_testing_direct_fixup_rows: rows of the last token chunk of the latest error_signal
    call on ``workspace`` that the direct algorithm recomputed (-1: not the direct algorithm)."""
    T, d = h.shape
    desc = error_signal_desc(T, d, W_U.shape[0], _dtype_code(h), t_chunk=t_chunk, algo=algo)
    return int(_lib.fpo_testing_direct_fixup_rows(ctypes.byref(desc), _ptr(workspace),
                                                  _stream(stream)))


# --------------------------------------------------------------------------- layer update
def layer_update_workspace() -> int:
    return int(_lib.fpo_layer_update_workspace())


def layer_update(g, A, lr, *, W_master=None, W_out=None, G_out=None, workspace=None, stream=None):
    """fpo_layer_update: G = g~^T A ; W_master -= lr G ; W_out = cast(W_master)."""
    T, d = g.shape
    d_ff = A.shape[1]
    if workspace is None:
        workspace = _workspace(layer_update_workspace(), g.device, stream)
    rc = _lib.fpo_layer_update(T, d, d_ff, _dtype_code(g), _ptr(g), _ptr(A), float(lr),
                               _ptr(W_master), _ptr(W_out), _ptr(G_out), _ptr(workspace),
                               _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_layer_update")
    return workspace


def _ptr_array(ts, n):
    if ts is None:
        return None
    return (_vp * n)(*[_ptr(t) for t in ts])


def layer_update_grouped(g, As, lr, *, W_masters=None, W_outs=None, G_outs=None, workspace=None,
                         stream=None):
    """fpo_layer_update_grouped over len(As) target layers in one launch."""
    n = len(As)
    T, d = g.shape
    d_ff = As[0].shape[1]
    if workspace is None:
        workspace = _workspace(layer_update_workspace(), g.device, stream)
    rc = _lib.fpo_layer_update_grouped(n, T, d, d_ff, _dtype_code(g), _ptr(g), _ptr_array(As, n),
                                       float(lr), _ptr_array(W_masters, n), _ptr_array(W_outs, n),
                                       _ptr_array(G_outs, n), _ptr(workspace), _nbytes(workspace),
                                       _stream(stream))
    _check(rc, "fpo_layer_update_grouped")
    return workspace


def layer_update_grouped_signals(gs, As, lr, *, W_masters=None, W_outs=None, G_outs=None,
                                 workspace=None, stream=None):
    """fpo_layer_update_grouped_signals: layer l uses its own signal gs[l]."""
    n = len(As)
    T, d = gs[0].shape
    d_ff = As[0].shape[1]
    if workspace is None:
        workspace = _workspace(layer_update_workspace(), gs[0].device, stream)
    rc = _lib.fpo_layer_update_grouped_signals(
        n, T, d, d_ff, _dtype_code(gs[0]), _ptr_array(gs, n), _ptr_array(As, n), float(lr),
        _ptr_array(W_masters, n), _ptr_array(W_outs, n), _ptr_array(G_outs, n), _ptr(workspace),
        _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_layer_update_grouped_signals")
    return workspace


def optimizer_desc(kind=OPT_ADAMW, *, lr=1e-4, momentum=0.9, beta1=0.9, beta2=0.999, eps=1e-8,
                   weight_decay=0.01, clip=CLIP_STEP, clip_frac=0.01, step=1):
    d = OptimizerDesc(int(kind), int(clip), float(lr), float(momentum), float(beta1),
                      float(beta2), float(eps), float(weight_decay), float(clip_frac), int(step))
    # the rates as given, for the entry points that take them in double
    d.exact = dict(lr=float(lr), beta1=float(beta1), beta2=float(beta2), eps=float(eps),
                   weight_decay=float(weight_decay), clip_frac=float(clip_frac))
    return d


def layer_optimize_workspace(n_layers, d, d_ff) -> int:
    return int(_lib.fpo_layer_optimize_workspace(int(n_layers), int(d), int(d_ff)))


def layer_optimize_grouped(gs, As, opt, W_masters, *, W_outs=None, states1=None, states2=None,
                           workspace=None, stream=None):
    """fpo_layer_optimize_grouped: G_l = g_l^T A_l, relative clip, optimizer step."""
    n = len(As)
    T, d = gs[0].shape
    d_ff = As[0].shape[1]
    if workspace is None:
        workspace = _workspace(layer_optimize_workspace(n, d, d_ff), gs[0].device, stream)
    rc = _lib.fpo_layer_optimize_grouped(
        n, T, d, d_ff, _dtype_code(gs[0]), _ptr_array(gs, n), _ptr_array(As, n), ctypes.byref(opt),
        _ptr_array(W_masters, n), _ptr_array(W_outs, n), _ptr_array(states1, n),
        _ptr_array(states2, n), _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_layer_optimize_grouped")
    return workspace


def _coeffs(coeffs, steps):
    """None, or steps triples (a, b, c) as a C array; the caller keeps it alive."""
    if coeffs is None:
        return None
    flat = [float(v) for row in coeffs for v in row]
    if len(coeffs) != steps or len(flat) != 3 * steps:
        raise ValueError("coeffs needs one (a, b, c) per step")
    return (_f32 * len(flat))(*flat)


def _expect_all(ts, n, shape, dtype, name):
    if ts is None:
        return
    if len(ts) != n:
        raise ValueError(f"{name}: one entry per layer expected")
    for t in ts:
        _expect(t, shape, dtype, name)


def orthogonalize_workspace(n_layers, rows, cols, dtype=BF16) -> int:
    return int(_lib.fpo_orthogonalize_workspace(int(n_layers), int(rows), int(cols), int(dtype)))


def orthogonalize_grouped(Gs, Os, *, steps=5, coeffs=None, eps=1e-7, workspace=None, stream=None):
    """fpo_orthogonalize_grouped: Os[l] = Newton-Schulz orthogonalisation of Gs[l] (one shape
    and dtype; Os[l] may be Gs[l]).  coeffs: None, or ``steps`` triples (a, b, c).  Returns the
    workspace tensor (its first word holds the device status)."""
    n = len(Gs)
    if n == 0:
        raise ValueError("Gs and Os need one tensor per layer")
    G = Gs[0]
    rows, cols = G.shape
    _expect_all(Gs, n, G.shape, G.dtype, "Gs")
    _expect_all(Os, n, G.shape, G.dtype, "Os")
    dt = _dtype_code(G)
    if workspace is None:
        workspace = _workspace(orthogonalize_workspace(n, rows, cols, dt), G.device, stream)
    co = _coeffs(coeffs, steps)
    rc = _lib.fpo_orthogonalize_grouped(n, rows, cols, dt, _ptr_array(Gs, n), int(steps), co,
                                        float(eps), _ptr_array(Os, n), _ptr(workspace),
                                        _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_orthogonalize_grouped")
    return workspace


def muon_desc(*, lr=1e-4, momentum=0.95, weight_decay=0.0, scale=1.0, nesterov=True, steps=5,
              coeffs=None, eps=1e-7):
    """fpo_muon_desc; coeffs as in orthogonalize_grouped."""
    co = _coeffs(coeffs, steps)
    d = MuonDesc(float(lr), float(momentum), float(weight_decay), float(scale), float(eps),
                 1 if nesterov else 0, int(steps),
                 None if co is None else ctypes.cast(co, ctypes.POINTER(_f32)))
    d._keep = co
    return d


def layer_muon_workspace(n_layers, d, d_ff, dtype=BF16) -> int:
    return int(_lib.fpo_layer_muon_workspace(int(n_layers), int(d), int(d_ff), int(dtype)))


def layer_muon_grouped(gs, As, opt, W_masters, momenta, *, W_outs=None, workspace=None,
                       stream=None):
    """fpo_layer_muon_grouped: G_l = gs[l]^T As[l], momentum, orthogonalisation, weight step."""
    n = len(As)
    if n == 0 or n != len(gs):
        raise ValueError("gs and As need one tensor per layer")
    T, d = gs[0].shape
    d_ff = As[0].shape[1]
    dtype = gs[0].dtype
    _expect_all(gs, n, (T, d), dtype, "gs")
    _expect_all(As, n, (T, d_ff), dtype, "As")
    _expect_all(W_masters, n, (d, d_ff), torch.float32, "W_masters")
    _expect_all(momenta, n, (d, d_ff), torch.float32, "momenta")
    _expect_all(W_outs, n, (d, d_ff), dtype, "W_outs")
    dt = _dtype_code(gs[0])
    if workspace is None:
        workspace = _workspace(layer_muon_workspace(n, d, d_ff, dt), gs[0].device, stream)
    rc = _lib.fpo_layer_muon_grouped(n, T, d, d_ff, dt, _ptr_array(gs, n), _ptr_array(As, n),
                                     ctypes.byref(opt), _ptr_array(W_masters, n),
                                     _ptr_array(W_outs, n), _ptr_array(momenta, n),
                                     _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_layer_muon_grouped")
    return workspace


def gate_up_signals(g, W3_init, a, b, dA, dB, *, workspace=None, stream=None):
    """fpo_gate_up_signals: SwiGLU W1/W2 signals through the cached W3_init feedback."""
    T, d = g.shape
    d_ff = W3_init.shape[1]
    if workspace is None:
        workspace = _workspace(layer_update_workspace(), g.device, stream)
    rc = _lib.fpo_gate_up_signals(T, d, d_ff, _dtype_code(g), _ptr(g), _ptr(W3_init), _ptr(a),
                                  _ptr(b), _ptr(dA), _ptr(dB), _ptr(workspace), _nbytes(workspace),
                                  _stream(stream))
    _check(rc, "fpo_gate_up_signals")
    return workspace


def layer_signals(g, g_outs, *, m=None, gamma_post=None, x=None, gamma_pre=None, eps=1e-6,
                  min_rms=0.5, stream=None):
    """fpo_layer_signals: g_outs[l] = pre-MLP VJP at x[l] of (post-FFN VJP at m[l] of g);
    m / gamma_post and x / gamma_pre are lists with one entry per layer, or None."""
    n = len(g_outs)
    T, d = g.shape

    def arr(ts):
        if ts is None:
            return None
        if len(ts) != n:
            raise ValueError("one entry per layer expected")
        return _ptr_array(ts, n)

    rc = _lib.fpo_layer_signals(n, T, d, _dtype_code(g), _ptr(g), arr(m), arr(gamma_post), arr(x),
                                arr(gamma_pre), float(eps), float(min_rms), _ptr_array(g_outs, n),
                                _stream(stream))
    _check(rc, "fpo_layer_signals")
    return g_outs


def rmsnorm_vjp(g, x, gamma, g_out, *, eps=1e-6, min_rms=0.5, stream=None):
    """fpo_rmsnorm_vjp: the RMSNorm Jacobian (with the min-RMS clamp) applied to g at x."""
    T, d = x.shape
    rc = _lib.fpo_rmsnorm_vjp(T, d, _dtype_code(x), _ptr(g), _ptr(x), _ptr(gamma), float(eps),
                              float(min_rms), _ptr(g_out), _stream(stream))
    _check(rc, "fpo_rmsnorm_vjp")
    return g_out


# --------------------------------------------------------------------------- LayerNorm
def layernorm(x, gamma, beta, y, *, eps=1e-5, mean_out=None, rstd_out=None, stream=None):
    """fpo_layernorm: y = gamma (x - mean) / sqrt(var + eps) + beta over the rows of x [T, d];
    gamma and beta may be None, mean_out and rstd_out are fp32 [T] or None."""
    T, d = x.shape
    _expect(y, x.shape, x.dtype, "y")
    _expect(gamma, (d,), x.dtype, "gamma")
    _expect(beta, (d,), x.dtype, "beta")
    _expect(mean_out, (T,), torch.float32, "mean_out")
    _expect(rstd_out, (T,), torch.float32, "rstd_out")
    rc = _lib.fpo_layernorm(T, d, _dtype_code(x), _ptr(x), _ptr(gamma), _ptr(beta), float(eps),
                            _ptr(y), _ptr(mean_out), _ptr(rstd_out), _stream(stream))
    _check(rc, "fpo_layernorm")
    return y


def layernorm_vjp_workspace(T, d, dtype=BF16) -> int:
    return int(_lib.fpo_layernorm_vjp_workspace(int(T), int(d), int(dtype)))


def layernorm_vjp(g, x, gamma, g_out, *, eps=1e-5, min_rms=0.5, dgamma=None, dbeta=None,
                  workspace=None, stream=None):
    """fpo_layernorm_vjp: the LayerNorm Jacobian (with the min-RMS clamp; 0 for the exact
    gradient) applied to g at x into g_out, and the fp32 weight and bias gradients into dgamma
    and dbeta where given.  gamma and g_out may be None."""
    T, d = x.shape
    _expect(g, x.shape, x.dtype, "g")
    _expect(gamma, (d,), x.dtype, "gamma")
    _expect(g_out, x.shape, x.dtype, "g_out")
    _expect(dgamma, (d,), torch.float32, "dgamma")
    _expect(dbeta, (d,), torch.float32, "dbeta")
    if workspace is None and (dgamma is not None or dbeta is not None):
        need = layernorm_vjp_workspace(T, d, _dtype_code(x))
        if need:  # (0: a short batch)
            workspace = _workspace(need, x.device, stream)
    rc = _lib.fpo_layernorm_vjp(T, d, _dtype_code(x), _ptr(g), _ptr(x), _ptr(gamma), float(eps),
                                float(min_rms), _ptr(g_out), _ptr(dgamma), _ptr(dbeta),
                                _ptr(workspace), 0 if workspace is None else _nbytes(workspace),
                                _stream(stream))
    _check(rc, "fpo_layernorm_vjp")
    return g_out


def _entry(fn):
    """Marks an entry point all of whose tensors, not the leading one alone, are looked at for their
    device (_at).  It becomes a callable object with fn's name, documentation and signature, which
    inspect.isfunction does not find: who lists entry points looks for callables."""
    kind = type("entry", (), {"__call__": staticmethod(fn), "__doc__": fn.__doc__})
    return functools.update_wrapper(kind(), fn)


def _at(here, t):
    """_ptr of a tensor that is to lie on device `here`, the leading tensor's (-1: none)."""
    if t is None:
        return None
    if t.get_device() != here or here < 0 or not t.is_contiguous():
        _on_current_device(t)
        _ptr(t)
    return t.data_ptr()


def _fits(t, shape, dtype, name):
    if t is not None and (t.shape != shape or t.dtype is not dtype):
        _expect(t, shape, dtype, name)


# --------------------------------------------------------------------------- linear layers
def linear_workspace(T, d_out, d_in, dtype=BF16) -> int:
    return int(_lib.fpo_linear_workspace(int(T), int(d_out), int(d_in), int(dtype)))


@_entry
def linear(x, W, y, *, bias=None, act=ACT_NONE, residual=None, z_out=None, workspace=None,
           stream=None):
    """fpo_linear: y = act(x W^T + bias) + residual, for x [T, d_in] and W [d_out, d_in] of one
    dtype; residual may be y.  z_out takes the pre-activation, which linear_vjp reads.  Returns the
    workspace tensor (its first word holds the device status)."""
    T, d_in = x.shape
    d_out = W.shape[0]
    _fits(W, (d_out, d_in), x.dtype, "W")
    _fits(y, (T, d_out), x.dtype, "y")
    _fits(bias, (d_out,), x.dtype, "bias")
    _fits(residual, (T, d_out), x.dtype, "residual")
    _fits(z_out, (T, d_out), x.dtype, "z_out")
    dt = _dtype_code(x)
    here = x.get_device()
    xp, Wp, bp, rp, yp, zp = (_at(here, x), _at(here, W), _at(here, bias), _at(here, residual),
                              _at(here, y), _at(here, z_out))
    if workspace is None:
        workspace = _workspace(_lib.fpo_linear_workspace(T, d_out, d_in, dt), x.device, stream)
    rc = _lib.fpo_linear(T, d_out, d_in, dt, act, xp, Wp, bp, rp, yp, zp, _at(here, workspace),
                         _nbytes(workspace), _stream(stream))
    if rc:
        _check(rc, "fpo_linear")
    return workspace


def linear_vjp_workspace(T, d_out, d_in, dtype=BF16, act=ACT_NONE) -> int:
    return int(_lib.fpo_linear_vjp_workspace(int(T), int(d_out), int(d_in), int(dtype), int(act)))


@_entry
def linear_vjp(dy, x, W, dx, *, act=ACT_NONE, z=None, act_in=ACT_NONE, z_in=None, dW=None,
               dbias=None, workspace=None, stream=None):
    """fpo_linear_vjp: with dz = dy act'(z), dx = (dz W) act_in'(z_in), dW = dz^T x and the fp32
    dbias = sum_t dz; dx, dW and dbias may be None (not all), x is read for dW, W for dx.  Returns
    the workspace tensor (its first word holds the device status)."""
    T, d_out = dy.shape
    for t, name in ((W, "W"), (dW, "dW"), (x, "x"), (dx, "dx"), (z_in, "z_in")):
        if t is not None:
            d_in = t.shape[1]
            break
    else:
        d_in = 8  # the bias gradient alone
    _fits(x, (T, d_in), dy.dtype, "x")
    _fits(W, (d_out, d_in), dy.dtype, "W")
    _fits(dx, (T, d_in), dy.dtype, "dx")
    _fits(z, (T, d_out), dy.dtype, "z")
    _fits(z_in, (T, d_in), dy.dtype, "z_in")
    _fits(dW, (d_out, d_in), dy.dtype, "dW")
    _fits(dbias, (d_out,), torch.float32, "dbias")
    dt = _dtype_code(dy)
    here = dy.get_device()
    dyp, zp, xp, Wp, zip_, dxp, dWp, dbp = (
        _at(here, dy), _at(here, z), _at(here, x), _at(here, W), _at(here, z_in), _at(here, dx),
        _at(here, dW), _at(here, dbias))
    if workspace is None:
        workspace = _workspace(_lib.fpo_linear_vjp_workspace(T, d_out, d_in, dt, act), dy.device, stream)
    rc = _lib.fpo_linear_vjp(T, d_out, d_in, dt, act, dyp, zp, xp, Wp, act_in, zip_, dxp, dWp, dbp,
                             _at(here, workspace), _nbytes(workspace), _stream(stream))
    if rc:
        _check(rc, "fpo_linear_vjp")
    return workspace


# --------------------------------------------------------------------------- AdamW over many tensors
def adamw_workspace(sizes, clip=CLIP_NONE) -> int:
    return int(_lib.fpo_adamw_workspace(len(sizes), (_i64 * len(sizes))(*sizes), int(clip)))


_DTYPES = {torch.bfloat16: BF16}


@_entry
def adamw_grouped(Gs, opt, W_masters, states1, states2, *, scales1=None, scales2=None, W_outs=None,
                  weight_decays=None, seed=0, workspace=None, stream=None):
    """fpo_adamw_grouped: one AdamW step (optimizer_desc, per-tensor relative clip) on any number of
    tensors with given gradients; what belongs to a tensor has its number of elements, in any shape.
    Gs: fp32 or bf16, each its own; W_masters: fp32; states1 and
    states2: fp32, or float8_e4m3fn and uint8 with fp32 scales1 and scales2 of one element per
    ADAMW_BLOCK (None entries where the states are fp32; zeros are a valid start).  W_outs: fp32 or
    bf16, the list or an entry may be None; weight_decays: one per tensor, by default the
    descriptor's.  seed: of the 8-bit states' rounding.  Returns the workspace (None without a clip)."""
    n = len(Gs)
    rest = (W_masters, states1, states2, scales1, scales2, W_outs, weight_decays)
    if n == 0 or any(ts is not None and len(ts) != n for ts in rest):
        raise ValueError("one entry per tensor expected in every list")
    sizes = list(map(_numel, Gs))
    m_types = [m.dtype for m in states1]
    small = [dt != torch.float32 for dt in m_types]
    none = [None] * n
    scales1 = none if scales1 is None else scales1
    scales2 = none if scales2 is None else scales2
    W_outs = none if W_outs is None else W_outs

    def check(name, ts, counts, types):
        if list(map(_numel, ts)) != counts or [t.dtype for t in ts] != types:
            for t, c, want in zip(ts, counts, types):
                if t.dtype != want or t.numel() != c:
                    raise ValueError(f"{name}: expected {c} elements of {want}, got {t.numel()} of {t.dtype}")

    def given(ts, xs):
        return [x for t, x in zip(ts, xs) if t is not None]

    f32 = [torch.float32] * n
    check("W_masters", W_masters, sizes, f32)
    check("states1", states1, sizes, [torch.float8_e4m3fn if s else torch.float32 for s in small])
    check("states2", states2, sizes, [torch.uint8 if s else torch.float32 for s in small])
    outs = given(W_outs, W_outs)
    check("W_outs", outs, given(W_outs, sizes), [t.dtype for t in outs])
    blocks = [-(-c // ADAMW_BLOCK) for c in sizes]
    check("scales1", given(scales1, scales1), given(scales1, blocks), given(scales1, f32))
    check("scales2", given(scales2, scales2), given(scales2, blocks), given(scales2, f32))
    if any(s and (a is None or b is None) for s, a, b in zip(small, scales1, scales2)):
        raise ValueError("8-bit states need scales1 and scales2")
    if opt.kind != OPT_ADAMW:
        raise ValueError("adamw_grouped takes the descriptor of OPT_ADAMW")

    def rate(name, field=None):  # as given to optimizer_desc, or the field if it was set since
        v = getattr(opt, field or name)
        given = getattr(opt, "exact", {}).get(name, v)
        return given if _f32(given).value == v else v

    desc = AdamwDesc(rate("lr"), rate("beta1"), rate("beta2"), rate("eps", "adam_eps"), rate("clip_frac"),
                     opt.step, opt.clip)
    g_types = [_DTYPES.get(G.dtype) or _dtype_code(G) for G in Gs]
    w_types = [F32 if t is None else _DTYPES.get(t.dtype) or _dtype_code(t) for t in W_outs]
    decays = [rate("weight_decay")] * n if weight_decays is None else [float(w) for w in weight_decays]
    cols = [_ptrs(ts) for ts in (Gs, W_masters, W_outs, states1, states2, scales1, scales2)]
    table = b"".join(map(_ADAMW_TENSOR.pack, sizes, *cols, g_types, w_types,
                         [8 if s else 32 for s in small], decays))
    if workspace is None and opt.clip != CLIP_NONE:
        workspace = _workspace(adamw_workspace(sizes, opt.clip), Gs[0].device, stream)
    rc = _lib.fpo_adamw_grouped(n, ctypes.cast(table, ctypes.POINTER(AdamwTensor)),
                                ctypes.byref(desc), int(seed) & 0xffffffffffffffff,
                                _at(Gs[0].get_device(), workspace),
                                0 if workspace is None else _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_adamw_grouped")
    return workspace


@_entry
def adamw_state_values(codes, scales, out, *, stream=None):
    """fpo_adamw_state_values: the values of 8-bit moments (float8_e4m3fn: first, uint8: second)
    with their scales, into out (fp32 or bf16, the same shape)."""
    if codes.dtype not in (torch.float8_e4m3fn, torch.uint8):
        raise TypeError("codes are float8_e4m3fn (first moments) or uint8 (second moments)")
    n = codes.numel()
    dt = _dtype_code(out)
    _expect(out, codes.shape, out.dtype, "out")
    _expect(scales, (-(-n // ADAMW_BLOCK),), torch.float32, "scales")
    moment = 1 if codes.dtype == torch.float8_e4m3fn else 2
    here = out.get_device()
    _check(_lib.fpo_adamw_state_values(n, moment, _at(here, codes), _at(here, scales), dt, _at(here, out),
                                       _stream(stream)), "fpo_adamw_state_values")
    return out


# --------------------------------------------------------------------------- cosine
def cosine_workspace(n: int) -> int:
    return int(_lib.fpo_cosine_workspace(int(n)))


def cosine(X, Y, out=None, *, workspace=None, stream=None):
    """fpo_cosine: returns a device fp64 tensor [<X,Y>, |X|^2, |Y|^2, cos]."""
    n = X.numel()
    if out is None:
        out = _result(4, X.device, stream)
    if workspace is None:
        workspace = _workspace(cosine_workspace(n), X.device, stream)
    rc = _lib.fpo_cosine(n, _dtype_code(X), _ptr(X), _ptr(Y), _ptr(out), _ptr(workspace),
                         _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_cosine")
    return out


def cosine_grouped_workspace(n_layers: int, n: int) -> int:
    return int(_lib.fpo_cosine_grouped_workspace(int(n_layers), int(n)))


def cosine_grouped(X, Y, out=None, *, workspace=None, stream=None):
    """fpo_cosine_grouped: per layer [<X_l,Y_l>, |X_l|^2, |Y_l|^2, cos_l] as a device fp64
    tensor [len(X), 4]; X and Y are lists of same-size tensors of one dtype."""
    n_layers = len(X)
    if n_layers != len(Y) or n_layers == 0:
        raise ValueError("X and Y need one tensor per layer")
    n = X[0].numel()
    if any(t.numel() != n for t in list(X) + list(Y)):
        raise ValueError("every X_l and Y_l must have the same number of elements")
    if any(t.dtype != X[0].dtype for t in list(X) + list(Y)):
        raise TypeError("X and Y share one dtype")
    if out is None:
        out = _result((n_layers, 4), X[0].device, stream)
    if workspace is None:
        workspace = _workspace(cosine_grouped_workspace(n_layers, n), X[0].device, stream)
    xarr = (_vp * n_layers)(*[_ptr(t) for t in X])
    yarr = (_vp * n_layers)(*[_ptr(t) for t in Y])
    rc = _lib.fpo_cosine_grouped(n_layers, n, _dtype_code(X[0]), xarr, yarr, _ptr(out),
                                 _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_cosine_grouped")
    return out


def layer_grad_cosine_workspace(n_layers: int, d: int, d_ff: int) -> int:
    return int(_lib.fpo_layer_grad_cosine_workspace(int(n_layers), int(d), int(d_ff)))


def layer_grad_cosine_grouped(g, As, Ys, G_outs, out=None, *, workspace=None, stream=None):
    """fpo_layer_grad_cosine_grouped: G_outs[l] = g^T As[l] and, per layer,
    [<G_l,Y_l>, |G_l|^2, |Y_l|^2, cos_l] as a device fp64 tensor [len(As), 4]."""
    n = len(As)
    if n == 0 or n != len(Ys) or n != len(G_outs):
        raise ValueError("As, Ys and G_outs need one tensor per layer")
    T, d = g.shape
    d_ff = As[0].shape[1]
    if out is None:
        out = _result((n, 4), g.device, stream)
    if workspace is None:
        workspace = _workspace(layer_grad_cosine_workspace(n, d, d_ff), g.device, stream)
    arr = lambda ts: (_vp * n)(*[_ptr(t) for t in ts])  # noqa: E731
    rc = _lib.fpo_layer_grad_cosine_grouped(n, T, d, d_ff, _dtype_code(g), _ptr(g), arr(As),
                                            arr(Ys), arr(G_outs), _ptr(out), _ptr(workspace),
                                            _nbytes(workspace), _stream(stream))
    _check(rc, "fpo_layer_grad_cosine_grouped")
    return out


def norm_ratio_workspace(n_layers: int, n: int) -> int:
    return int(_lib.fpo_norm_ratio_workspace(int(n_layers), int(n)))


def norm_ratio(G, W, rel_step=0.01, out=None, *, workspace=None, stream=None):
    """fpo_norm_ratio: per layer [||G_l||^2, ||W_l||^2, ||G_l||/||W_l||, rel_step/ratio] as a
    device fp64 tensor [len(G), 4]; G and W are lists of same-size tensors."""
    n_layers = len(G)
    if n_layers != len(W) or n_layers == 0:
        raise ValueError("G and W need one tensor per layer")
    n = G[0].numel()
    if any(t.numel() != n for t in list(G) + list(W)):
        raise ValueError("every G_l and W_l must have the same number of elements")
    if any(t.dtype != G[0].dtype for t in G) or any(t.dtype != W[0].dtype for t in W):
        raise TypeError("the G_l share one dtype and the W_l share one dtype")
    if out is None:
        out = _result((n_layers, 4), G[0].device, stream)
    if workspace is None:
        workspace = _workspace(norm_ratio_workspace(n_layers, n), G[0].device, stream)
    garr = (_vp * n_layers)(*[_ptr(t) for t in G])
    warr = (_vp * n_layers)(*[_ptr(t) for t in W])
    rc = _lib.fpo_norm_ratio(n_layers, n, _dtype_code(G[0]), garr, _dtype_code(W[0]), warr,
                             float(rel_step), _ptr(out), _ptr(workspace), _nbytes(workspace),
                             _stream(stream))
    _check(rc, "fpo_norm_ratio")
    return out


MAX_COPY_BUFFERS = 64


def h2d_copy(dsts, srcs, *, stream=None):
    """fpo_h2d_copy: copy page-locked host tensors srcs[i] into device tensors dsts[i]
    (contiguous, equal byte sizes) by SM loads, one kernel launch per MAX_COPY_BUFFERS
    pairs."""
    if len(dsts) != len(srcs):
        raise ValueError("h2d_copy takes as many destinations as sources")
    for d_t, s_t in zip(dsts, srcs):
        if s_t.is_cuda or not s_t.is_contiguous():
            raise ValueError("h2d_copy sources are contiguous host tensors")
        if d_t.numel() * d_t.element_size() != s_t.numel() * s_t.element_size():
            raise ValueError("h2d_copy source and destination sizes differ")
    for c in range(0, len(srcs), MAX_COPY_BUFFERS):
        ds, ss = dsts[c:c + MAX_COPY_BUFFERS], srcs[c:c + MAX_COPY_BUFFERS]
        n = len(ss)
        _on_current_device(ds[0])
        darr = (_vp * n)(*[_ptr(t) for t in ds])
        sarr = (_vp * n)(*[t.data_ptr() for t in ss])
        barr = (_sz * n)(*[t.numel() * t.element_size() for t in ss])
        _check(_lib.fpo_h2d_copy(n, darr, sarr, barr, _stream(stream)), "fpo_h2d_copy")


def get_device_status(workspace, stream=None) -> int:
    """fpo_get_device_status: synchronise, read and clear the workspace's status word."""
    return int(_lib.fpo_get_device_status(_ptr(workspace), _stream(stream)))
