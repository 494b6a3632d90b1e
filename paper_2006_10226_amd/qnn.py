"""Python binding of libqnn (ctypes): argument marshalling only.

Every computation runs in the HIP kernels of ``libqnn.so``; PyTorch supplies
device memory and the current stream.  The library must have been built
(``python -m paper_2006_10226_amd.build`` or ``__graft_entry__.build()``);
the first call into it raises ImportError when it is missing -- there is no
CPU fallback.

Conventions follow include/qnn.h: activations NHWC, conv weights OHWI,
depthwise weights [R][S][C], dense weights [N][K]; scales and zero points are
Python numbers or sequences (per tensor or per output channel).
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple, Union

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqnn.so")

UINT8, INT8, INT32, FLOAT16, BFLOAT16 = 0, 1, 2, 3, 4
HALF_UP, HALF_AWAY, TWO_STAGE = 0, 1, 2
_TORCH_DT = {torch.uint8: UINT8, torch.int8: INT8, torch.int32: INT32}
_NAME_DT = {"u8": UINT8, "i8": INT8, "i32": INT32}
_DT_TORCH = {UINT8: torch.uint8, INT8: torch.int8, INT32: torch.int32}
_ROUND = {"half_up": HALF_UP, "half_away": HALF_AWAY, "two_stage": TWO_STAGE}
INT32_MIN, INT32_MAX = -(2**31), 2**31 - 1

STATUS = ["QNN_OK", "QNN_ERR_NULL", "QNN_ERR_SHAPE", "QNN_ERR_DTYPE", "QNN_ERR_QPARAM",
          "QNN_ERR_OVERFLOW", "QNN_ERR_UNSUPPORTED", "QNN_ERR_HIP", "QNN_ERR_ALLOC"]

# Every symbol the public header declares.
EXPORTS = [
    "qnn_abi_version", "qnn_last_error", "qnn_status_string", "qnn_quantize_multiplier",
    "qnn_conv2d", "qnn_depthwise_conv2d", "qnn_dense", "qnn_requantize", "qnn_add",
    "qnn_pool2d",
    "qnn_cache4_page_bytes", "qnn_cache4_append", "qnn_cache4_read", "qnn_attention4_workspace_size",
    "qnn_attention4", "qnn_pages_workspace_size", "qnn_pages_resize",
    "qnn_conv2d_plan_create", "qnn_depthwise_conv2d_plan_create", "qnn_dense_plan_create",
    "qnn_conv2d_plan_create_wt", "qnn_depthwise_conv2d_plan_create_wt", "qnn_dense_plan_create_wt",
    "qnn_requantize_plan_create", "qnn_plan_run", "qnn_plan_run_timed", "qnn_time_next_kernel", "qnn_plan_run_noalloc",
    "qnn_plan_set_residual", "qnn_plan_run_residual", "qnn_plan_set_activation", "qnn_activation_table", "qnn_lookup", "qnn_plan_workspace_size",
    "qnn_plan_describe", "qnn_set_tuning_file", "qnn_plan_destroy",
]


class QnnError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        self.status_name = STATUS[status] if 0 <= status < len(STATUS) else f"status {status}"
        super().__init__(f"{self.status_name}: {message}")


class QParams(ctypes.Structure):
    _fields_ = [("scale", ctypes.POINTER(ctypes.c_float)),
                ("zero_point", ctypes.POINTER(ctypes.c_int32)),
                ("n", ctypes.c_int32)]


class ConvParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("stride_h", "stride_w", "pad_top", "pad_left", "pad_bottom", "pad_right", "dil_h", "dil_w")]


class Clamp(ctypes.Structure):
    _fields_ = [("lo", ctypes.c_int32), ("hi", ctypes.c_int32)]


class Cache4Desc(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("pages", "page_size", "heads", "head_dim")]


class AttentionParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("tokens", "q_heads", "requests", "table_width")] +
                [(n, ctypes.c_int64) for n in ("q_ld", "o_ld", "table_ld")] +
                [(n, ctypes.c_int32) for n in ("max_q", "max_ctx", "causal", "window")] + [("scale", ctypes.c_float)])


_lib = None


def lib() -> ctypes.CDLL:
    """Load libqnn.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2006_10226_amd.build)")
    L = ctypes.CDLL(LIB_PATH)
    P, i32, i64, st = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int
    L.qnn_abi_version.restype = i32
    L.qnn_last_error.restype = ctypes.c_char_p
    L.qnn_status_string.restype = ctypes.c_char_p
    L.qnn_status_string.argtypes = [st]
    L.qnn_quantize_multiplier.argtypes = [ctypes.c_double, P, P]
    L.qnn_quantize_multiplier.restype = st
    conv_args = [P, st, i32, i32, i32, i32, QParams, P, i32, i32, i32, QParams, P, ConvParams,
                 P, st, QParams, Clamp, st, i32, i32]
    L.qnn_conv2d.argtypes = [P] + conv_args
    L.qnn_conv2d.restype = st
    dw_args = [P, st, i32, i32, i32, i32, QParams, P, i32, i32, QParams, P, ConvParams,
               P, st, QParams, Clamp, st, i32, i32]
    L.qnn_depthwise_conv2d.argtypes = [P] + dw_args
    L.qnn_depthwise_conv2d.restype = st
    L.qnn_dense.argtypes = [P, P, st, i32, i32, QParams, P, i32, QParams, P, P, st, QParams, Clamp, st, i32]
    L.qnn_dense.restype = st
    L.qnn_requantize.argtypes = [P, P, st, i64, i32, QParams, P, st, QParams, Clamp, st]
    L.qnn_requantize.restype = st
    L.qnn_add.argtypes = [P, P, st, QParams, P, st, QParams, i64, P, st, QParams, Clamp, st]
    L.qnn_add.restype = st
    L.qnn_pool2d.argtypes = [P, P, st, i32, i32, i32, i32, i32, i32, ConvParams, st, i32, i32, P, st]
    L.qnn_pool2d.restype = st
    L.qnn_cache4_page_bytes.argtypes = [i32, i32, i32]
    L.qnn_cache4_page_bytes.restype = ctypes.c_size_t
    L.qnn_cache4_append.argtypes = [P, Cache4Desc, P, P, st, QParams, QParams, i32, i64, i64, P]
    L.qnn_cache4_append.restype = st
    L.qnn_cache4_read.argtypes = [P, Cache4Desc, P, i32, P, P, st, i64, i64]
    L.qnn_cache4_read.restype = st
    L.qnn_attention4_workspace_size.argtypes = [Cache4Desc, AttentionParams]
    L.qnn_attention4_workspace_size.restype = ctypes.c_size_t
    L.qnn_attention4.argtypes = [P, P, st, QParams, Cache4Desc, P, P, P, AttentionParams, P, st, QParams, P,
                                 ctypes.c_size_t]
    L.qnn_attention4.restype = st
    L.qnn_pages_workspace_size.argtypes = [i32]
    L.qnn_pages_workspace_size.restype = ctypes.c_size_t
    L.qnn_pages_resize.argtypes = [P, i32, i32, P, P, P, i32, i64, P, i32, P, P, P, P, i32, P, P]
    L.qnn_pages_resize.restype = st
    PP = ctypes.POINTER(ctypes.c_void_p)
    L.qnn_conv2d_plan_create.argtypes = [PP, P, st, i32, i32, i32, i32, QParams, P, i32, i32, i32,
                                         QParams, P, ConvParams, st, QParams, Clamp, st, i32, i32]
    L.qnn_conv2d_plan_create.restype = st
    L.qnn_depthwise_conv2d_plan_create.argtypes = [PP, P, st, i32, i32, i32, i32, QParams, P, i32, i32,
                                                   QParams, P, ConvParams, st, QParams, Clamp, st, i32, i32]
    L.qnn_depthwise_conv2d_plan_create.restype = st
    L.qnn_dense_plan_create.argtypes = [PP, P, st, i32, i32, QParams, P, i32, QParams, P, st, QParams,
                                        Clamp, st, i32]
    L.qnn_dense_plan_create.restype = st
    L.qnn_conv2d_plan_create_wt.argtypes = [PP, P, st, i32, i32, i32, i32, QParams, P, st, i32, i32, i32,
                                            QParams, P, ConvParams, st, QParams, Clamp, st, i32, i32]
    L.qnn_conv2d_plan_create_wt.restype = st
    L.qnn_depthwise_conv2d_plan_create_wt.argtypes = [PP, P, st, i32, i32, i32, i32, QParams, P, st, i32, i32,
                                                      QParams, P, ConvParams, st, QParams, Clamp, st, i32, i32]
    L.qnn_depthwise_conv2d_plan_create_wt.restype = st
    L.qnn_dense_plan_create_wt.argtypes = [PP, P, st, i32, i32, QParams, P, st, i32, QParams, P, st, QParams,
                                           Clamp, st, i32]
    L.qnn_dense_plan_create_wt.restype = st
    L.qnn_requantize_plan_create.argtypes = [PP, P, st, i64, i32, QParams, st, QParams, Clamp, st]
    L.qnn_requantize_plan_create.restype = st
    L.qnn_plan_run.argtypes = [P, P, P, P, P]
    L.qnn_plan_run.restype = st
    L.qnn_plan_run_timed.argtypes = [P, P, P, P, P, P, P]
    L.qnn_plan_run_timed.restype = st
    L.qnn_time_next_kernel.argtypes = [P, P]
    L.qnn_time_next_kernel.restype = st
    L.qnn_plan_run_noalloc.argtypes = [P, P, P, P]
    L.qnn_plan_run_noalloc.restype = st
    L.qnn_plan_set_residual.argtypes = [P, st, QParams, i32, i32, st, QParams, Clamp, st]
    L.qnn_plan_set_residual.restype = st
    L.qnn_plan_set_activation.argtypes = [P, P, st, QParams]
    L.qnn_plan_set_activation.restype = st
    L.qnn_activation_table.argtypes = [st, st, QParams, st, QParams, P]
    L.qnn_activation_table.restype = st
    L.qnn_lookup.argtypes = [P, P, P, i64, P]
    L.qnn_lookup.restype = st
    L.qnn_plan_run_residual.argtypes = [P, P, P, P, P, P]
    L.qnn_plan_run_residual.restype = st
    L.qnn_plan_workspace_size.argtypes = [P]
    L.qnn_plan_workspace_size.restype = ctypes.c_size_t
    L.qnn_plan_describe.argtypes = [P]
    L.qnn_plan_describe.restype = ctypes.c_char_p
    L.qnn_set_tuning_file.argtypes = [ctypes.c_char_p]
    L.qnn_set_tuning_file.restype = st
    L.qnn_plan_destroy.argtypes = [P]
    L.qnn_plan_destroy.restype = None
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise QnnError(status, lib().qnn_last_error().decode())


class _Q:
    """Host arrays behind a qnn_qparams (kept alive for the call)."""

    def __init__(self, scale, zp, n: Optional[int] = None):
        s = np.atleast_1d(np.asarray(scale, dtype=np.float32))
        z = np.atleast_1d(np.asarray(zp, dtype=np.int32))
        if n is None:
            n = max(s.size, z.size)
        if s.size == 1 and n > 1:
            s = np.full(n, s[0], np.float32)
        if z.size == 1 and n > 1:
            z = np.full(n, z[0], np.int32)
        self.s = np.ascontiguousarray(s)
        self.z = np.ascontiguousarray(z)
        self.q = QParams(self.s.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                         self.z.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), int(n))


def _per_tensor_or_channel(scale, zp):
    s = np.atleast_1d(np.asarray(scale, dtype=np.float32))
    z = np.atleast_1d(np.asarray(zp, dtype=np.int32))
    return _Q(s, z, max(s.size, z.size))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


# The current stream's handle without the Stream object that
# torch.cuda.current_stream() builds (about 3 of the 7.5 us that a plan's run
# took on the host); None where this torch doesn't offer it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_handle(stream=None) -> int:
    """_stream as a plain integer."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _dt(t: torch.Tensor) -> int:
    if t.dtype not in _TORCH_DT:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return _TORCH_DT[t.dtype]


def _clamp(act: Optional[Tuple[int, int]]) -> Clamp:
    if act is None:
        return Clamp(INT32_MIN, INT32_MAX)
    return Clamp(int(max(INT32_MIN, act[0])), int(min(INT32_MAX, act[1])))


def _cp(stride, pads, dil) -> ConvParams:
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    dh, dw = (dil, dil) if isinstance(dil, int) else dil
    pt, pl, pb, pr = (pads,) * 4 if isinstance(pads, int) else pads
    return ConvParams(sh, sw, pt, pl, pb, pr, dh, dw)


def out_hw(H, W, R, S, stride=1, pads=0, dil=1):
    cp = _cp(stride, pads, dil)
    Ho = (H + cp.pad_top + cp.pad_bottom - cp.dil_h * (R - 1) - 1) // cp.stride_h + 1
    Wo = (W + cp.pad_left + cp.pad_right - cp.dil_w * (S - 1) - 1) // cp.stride_w + 1
    return Ho, Wo


def _contig(t: torch.Tensor, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _check_out(out: torch.Tensor, lead, ydt, whole=False):
    shape = tuple(out.shape) if whole else tuple(out.shape[:-1])
    if shape != tuple(lead) or out.dtype != _DT_TORCH[ydt]:
        raise ValueError(f"out is {tuple(out.shape)} {out.dtype}; expected leading dims {tuple(lead)} "
                         f"and dtype {_DT_TORCH[ydt]}")


def quantize_multiplier(M: float) -> Tuple[int, int]:
    m, s = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().qnn_quantize_multiplier(float(M), ctypes.byref(m), ctypes.byref(s)))
    return m.value, s.value


def time_next_kernel(start, stop):
    """The next main kernel launched from this thread records the two
    torch.cuda.Event objects at its own start and end."""
    for e in (start, stop):
        if not e.cuda_event:   # torch creates its events on first record
            e.record()
    _check(lib().qnn_time_next_kernel(ctypes.c_void_p(start.cuda_event), ctypes.c_void_p(stop.cuda_event)))


def set_tuning_file(path: Optional[str]):
    """Read kernel choices from, and append timed ones to, a text file
    (None: stop); see qnn_set_tuning_file."""
    _check(lib().qnn_set_tuning_file(None if path is None else os.fsencode(path)))


def abi_version() -> int:
    return lib().qnn_abi_version()


# ---------------------------------------------------------------- plans

class Plan:
    """A prepared conv / depthwise / dense / requantize (owns device memory)."""

    def __init__(self, handle: ctypes.c_void_p, in_shape, in_dtype, out_shape, out_dtype, y_ldc_shape=None, out_q=None):
        self._h = handle
        self.in_shape = tuple(in_shape)
        self.in_dtype = in_dtype
        self.out_shape = tuple(out_shape)
        self.out_dtype = out_dtype
        self.y_ldc_shape = tuple(y_ldc_shape or out_shape)
        self.residual = None   # (shape, dtype) of a fused add's residual
        self.out_q = out_q     # (scale, zp) of an 8-bit output

    @property
    def handle(self):
        return self._h

    @property
    def workspace_size(self) -> int:
        return int(lib().qnn_plan_workspace_size(self._h))

    def describe(self) -> str:
        return lib().qnn_plan_describe(self._h).decode()

    def set_residual(self, r_dtype, r_scale, r_zp, o_scale, o_zp, o_dtype="u8", act=None, rounding="half_up",
                     r_ldc=None, r_coff=0):
        """qnn_plan_set_residual: the plan then stores qnn.add(its conv
        output, a residual of the output's pixels) with the output qparams
        o_*; run it with run(x, out, workspace, residual=r), r of shape
        (N, Ho, Wo, r_ldc), dense: (M, r_ldc) (r_ldc defaults to the output channels)."""
        *pixels, K = self.out_shape
        r_ldc = K if r_ldc is None else r_ldc
        rdt, odt = _NAME_DT[r_dtype], _NAME_DT[o_dtype]
        rq, oq = _Q(r_scale, r_zp, 1), _Q(o_scale, o_zp, 1)
        _check(lib().qnn_plan_set_residual(self._h, rdt, rq.q, r_ldc, r_coff, odt, oq.q, _clamp(act),
                                           _ROUND[rounding]))
        self.out_dtype = _DT_TORCH[odt]
        self.residual = ((*pixels, r_ldc), _DT_TORCH[rdt])
        return self

    def set_activation(self, kind, y_scale, y_zp, y_dtype="i8"):
        """qnn_plan_set_activation: the plan then stores the activation of its
        output, with the qparams y_*; kind is one of ACTIVATIONS, or a table of
        256 bytes (numpy uint8, by the output's byte).  A set_residual may
        follow."""
        if isinstance(kind, str):
            if self.out_q is None:
                raise ValueError("an activation needs a plan with 8-bit outputs")
            scale, zp = self.out_q
            table = activation_table(kind, {v: k for k, v in _NAME_DT.items()}[_TORCH_DT[self.out_dtype]], scale, zp,
                                     y_dtype, y_scale, y_zp)
        else:
            table = _byte_table(kind)
        yq = _Q(y_scale, y_zp, 1)
        _check(lib().qnn_plan_set_activation(self._h, table.ctypes.data_as(ctypes.c_void_p), _NAME_DT[y_dtype], yq.q))
        self.out_dtype = _DT_TORCH[_NAME_DT[y_dtype]]
        self.out_q = (y_scale, y_zp)
        return self

    def new_output(self, device="cuda"):
        return torch.empty(self.y_ldc_shape or self.out_shape, dtype=self.out_dtype, device=device)

    def run(self, x: torch.Tensor, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
            stream=None, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Run on x (shape and dtype fixed at creation); the kernels trust the
        sizes, so they are checked here.  A plan with a fused add
        (set_residual) takes its residual tensor."""
        # Small plans are bound by this path: no Stream or c_void_p objects,
        # no shape copies, no library call for a workspace that isn't given.
        _contig(x, "x")
        if x.shape != self.in_shape or x.dtype != self.in_dtype:
            raise ValueError(f"x is {tuple(x.shape)} {x.dtype}, the plan expects {self.in_shape} {self.in_dtype}")
        if out is None:
            out = self.new_output(x.device)
        _contig(out, "out")
        if out.shape != self.y_ldc_shape or out.dtype != self.out_dtype:
            raise ValueError(f"out is {tuple(out.shape)} {out.dtype}, the plan writes {self.y_ldc_shape} "
                             f"{self.out_dtype}")
        ws = None
        if workspace is not None:
            if workspace.numel() * workspace.element_size() < self.workspace_size:
                raise ValueError("workspace is smaller than the plan needs")
            ws = workspace.data_ptr()
        fused = self.residual
        if (fused is None) != (residual is None):
            raise ValueError("a residual goes with a plan that has a fused add (set_residual), and only with one")
        if fused is not None:
            _contig(residual, "residual")
            if residual.shape != fused[0] or residual.dtype != fused[1]:
                raise ValueError(f"residual is {tuple(residual.shape)} {residual.dtype}, the plan expects "
                                 f"{fused[0]} {fused[1]}")
            status = lib().qnn_plan_run_residual(self._h, _stream_handle(stream), x.data_ptr(), residual.data_ptr(),
                                                 out.data_ptr(), ws)
        else:
            status = lib().qnn_plan_run(self._h, _stream_handle(stream), x.data_ptr(), out.data_ptr(), ws)
        if status:
            _check(status)
        return out

    def run_timed(self, x: torch.Tensor, out: torch.Tensor, workspace, start, stop, stream=None):
        """qnn_plan_run_timed: start / stop (torch.cuda.Event with timing)
        are recorded at the main kernel's own start and end."""
        for e in (start, stop):
            if not e.cuda_event:   # torch creates its events on first record
                e.record()
        _check(lib().qnn_plan_run_timed(self._h, _stream(stream), _ptr(x), _ptr(out), _ptr(workspace),
                                        ctypes.c_void_p(start.cuda_event), ctypes.c_void_p(stop.cuda_event)))
        return out

    def run_noalloc(self, x: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
        """qnn_plan_run_noalloc: the workspace is the library's static device
        array; out must be given (nothing is allocated)."""
        _contig(x, "x")
        _contig(out, "out")
        if tuple(x.shape) != self.in_shape or x.dtype != self.in_dtype:
            raise ValueError(f"x is {tuple(x.shape)} {x.dtype}, the plan expects {self.in_shape} {self.in_dtype}")
        if tuple(out.shape) != self.y_ldc_shape or out.dtype != self.out_dtype:
            raise ValueError(f"out is {tuple(out.shape)} {out.dtype}, the plan writes {self.y_ldc_shape} "
                             f"{self.out_dtype}")
        _check(lib().qnn_plan_run_noalloc(self._h, _stream(stream), _ptr(x), _ptr(out)))
        return out

    def close(self):
        if self._h:
            lib().qnn_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def conv2d_plan(x_shape, x_dtype, x_scale, x_zp, w: torch.Tensor, w_scale, w_zp, bias=None,
                stride=1, pads=0, dil=1, y_scale=1.0, y_zp=0, y_dtype="u8", act=None,
                rounding="half_up", y_ldc=None, y_coff=0, stream=None) -> Plan:
    N, H, W, C = x_shape
    _contig(w, "w")
    K, R, S, Cw = w.shape
    if Cw != C:
        raise ValueError("weight Cin does not match x")
    cp = _cp(stride, pads, dil)
    Ho, Wo = out_hw(H, W, R, S, stride, pads, dil)
    y_ldc = K if y_ldc is None else y_ldc
    xq, wq, yq = _Q(x_scale, x_zp, 1), _per_tensor_or_channel(w_scale, w_zp), _Q(y_scale, y_zp, 1)
    h = ctypes.c_void_p()
    if w.dtype == torch.uint8:   # asymmetric uint8 weights, legalised at creation
        _check(lib().qnn_conv2d_plan_create_wt(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], N, H, W, C,
                                               xq.q, _ptr(w), UINT8, K, R, S, wq.q, _ptr(bias), cp,
                                               _NAME_DT[y_dtype], yq.q, _clamp(act), _ROUND[rounding], y_ldc,
                                               y_coff))
    else:
        _check(lib().qnn_conv2d_plan_create(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], N, H, W, C, xq.q,
                                            _ptr(w), K, R, S, wq.q, _ptr(bias), cp, _NAME_DT[y_dtype], yq.q,
                                            _clamp(act), _ROUND[rounding], y_ldc, y_coff))
    return Plan(h, x_shape, _DT_TORCH[_NAME_DT[x_dtype]], (N, Ho, Wo, K), _DT_TORCH[_NAME_DT[y_dtype]],
                (N, Ho, Wo, y_ldc), None if y_dtype == "i32" else (y_scale, y_zp))


def depthwise_conv2d_plan(x_shape, x_dtype, x_scale, x_zp, w: torch.Tensor, w_scale, w_zp, bias=None,
                          stride=1, pads=0, dil=1, y_scale=1.0, y_zp=0, y_dtype="u8", act=None,
                          rounding="half_up", y_ldc=None, y_coff=0, stream=None) -> Plan:
    N, H, W, C = x_shape
    _contig(w, "w")
    R, S, Cw = w.shape
    if Cw != C:
        raise ValueError("depthwise weight channels do not match x")
    cp = _cp(stride, pads, dil)
    Ho, Wo = out_hw(H, W, R, S, stride, pads, dil)
    y_ldc = C if y_ldc is None else y_ldc
    xq, wq, yq = _Q(x_scale, x_zp, 1), _per_tensor_or_channel(w_scale, w_zp), _Q(y_scale, y_zp, 1)
    h = ctypes.c_void_p()
    if w.dtype == torch.uint8:
        _check(lib().qnn_depthwise_conv2d_plan_create_wt(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], N, H,
                                                         W, C, xq.q, _ptr(w), UINT8, R, S, wq.q, _ptr(bias), cp,
                                                         _NAME_DT[y_dtype], yq.q, _clamp(act), _ROUND[rounding],
                                                         y_ldc, y_coff))
    else:
        _check(lib().qnn_depthwise_conv2d_plan_create(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], N, H, W,
                                                      C, xq.q, _ptr(w), R, S, wq.q, _ptr(bias), cp,
                                                      _NAME_DT[y_dtype], yq.q, _clamp(act), _ROUND[rounding],
                                                      y_ldc, y_coff))
    return Plan(h, x_shape, _DT_TORCH[_NAME_DT[x_dtype]], (N, Ho, Wo, C), _DT_TORCH[_NAME_DT[y_dtype]],
                (N, Ho, Wo, y_ldc), None if y_dtype == "i32" else (y_scale, y_zp))


def dense_plan(M, K, x_dtype, x_scale, x_zp, w: torch.Tensor, w_scale, w_zp, bias=None, y_scale=1.0, y_zp=0,
               y_dtype="i8", act=None, rounding="half_up", y_ldc=None, stream=None) -> Plan:
    _contig(w, "w")
    Nd, Kw = w.shape
    if Kw != K:
        raise ValueError("dense weight K does not match x")
    y_ldc = Nd if y_ldc is None else y_ldc
    xq, wq, yq = _Q(x_scale, x_zp, 1), _per_tensor_or_channel(w_scale, w_zp), _Q(y_scale, y_zp, 1)
    h = ctypes.c_void_p()
    if w.dtype == torch.uint8:
        _check(lib().qnn_dense_plan_create_wt(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], M, K, xq.q,
                                              _ptr(w), UINT8, Nd, wq.q, _ptr(bias), _NAME_DT[y_dtype], yq.q,
                                              _clamp(act), _ROUND[rounding], y_ldc))
    else:
        _check(lib().qnn_dense_plan_create(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], M, K, xq.q, _ptr(w),
                                           Nd, wq.q, _ptr(bias), _NAME_DT[y_dtype], yq.q, _clamp(act),
                                           _ROUND[rounding], y_ldc))
    return Plan(h, (M, K), _DT_TORCH[_NAME_DT[x_dtype]], (M, Nd), _DT_TORCH[_NAME_DT[y_dtype]], (M, y_ldc),
                None if y_dtype == "i32" else (y_scale, y_zp))


def requantize_plan(shape, x_dtype, x_scale, x_zp, y_scale, y_zp, y_dtype="u8", act=None,
                    rounding="half_up", stream=None) -> Plan:
    channels = shape[-1] if len(shape) else 1
    count = int(np.prod(shape)) if len(shape) else 1
    xq, yq = _per_tensor_or_channel(x_scale, x_zp), _per_tensor_or_channel(y_scale, y_zp)
    h = ctypes.c_void_p()
    _check(lib().qnn_requantize_plan_create(ctypes.byref(h), _stream(stream), _NAME_DT[x_dtype], count, channels,
                                            xq.q, _NAME_DT[y_dtype], yq.q, _clamp(act), _ROUND[rounding]))
    return Plan(h, shape, _DT_TORCH[_NAME_DT[x_dtype]], shape, _DT_TORCH[_NAME_DT[y_dtype]])


# ---------------------------------------------------------------- one-shot ops

def conv2d(x: torch.Tensor, x_scale, x_zp, w: torch.Tensor, w_scale, w_zp, bias=None, stride=1, pads=0,
           dil=1, y_scale=1.0, y_zp=0, y_dtype="u8", act=None, rounding="half_up",
           out: Optional[torch.Tensor] = None, y_coff=0, stream=None) -> torch.Tensor:
    """qnn.conv2d + bias + requantize + clamp; NHWC x, OHWI w (device tensors).

    With ``out`` given (NHWC, last dim = row stride), the result is written to
    channels [y_coff, y_coff + K) of it (a concat slice)."""
    _contig(x, "x")
    _contig(w, "w")
    N, H, W, C = x.shape
    K, R, S, _ = w.shape
    Ho, Wo = out_hw(H, W, R, S, stride, pads, dil)
    ydt = _NAME_DT[y_dtype]
    if out is None:
        out = torch.empty((N, Ho, Wo, K), dtype=_DT_TORCH[ydt], device=x.device)
    _contig(out, "out")
    _check_out(out, (N, Ho, Wo), ydt)
    xq, wq, yq = _Q(x_scale, x_zp, 1), _per_tensor_or_channel(w_scale, w_zp), _Q(y_scale, y_zp, 1)
    _check(lib().qnn_conv2d(_stream(stream), _ptr(x), _dt(x), N, H, W, C, xq.q, _ptr(w), K, R, S, wq.q,
                            _ptr(bias), _cp(stride, pads, dil), _ptr(out), ydt, yq.q, _clamp(act),
                            _ROUND[rounding], out.shape[-1], y_coff))
    return out


def depthwise_conv2d(x: torch.Tensor, x_scale, x_zp, w: torch.Tensor, w_scale, w_zp, bias=None, stride=1,
                     pads=0, dil=1, y_scale=1.0, y_zp=0, y_dtype="u8", act=None, rounding="half_up",
                     out: Optional[torch.Tensor] = None, y_coff=0, stream=None) -> torch.Tensor:
    _contig(x, "x")
    _contig(w, "w")
    N, H, W, C = x.shape
    R, S, _ = w.shape
    Ho, Wo = out_hw(H, W, R, S, stride, pads, dil)
    ydt = _NAME_DT[y_dtype]
    if out is None:
        out = torch.empty((N, Ho, Wo, C), dtype=_DT_TORCH[ydt], device=x.device)
    _contig(out, "out")
    _check_out(out, (N, Ho, Wo), ydt)
    xq, wq, yq = _Q(x_scale, x_zp, 1), _per_tensor_or_channel(w_scale, w_zp), _Q(y_scale, y_zp, 1)
    _check(lib().qnn_depthwise_conv2d(_stream(stream), _ptr(x), _dt(x), N, H, W, C, xq.q, _ptr(w), R, S, wq.q,
                                      _ptr(bias), _cp(stride, pads, dil), _ptr(out), ydt, yq.q, _clamp(act),
                                      _ROUND[rounding], out.shape[-1], y_coff))
    return out


def dense(x: torch.Tensor, x_scale, x_zp, w: torch.Tensor, w_scale, w_zp, bias=None, y_scale=1.0, y_zp=0,
          y_dtype="i8", act=None, rounding="half_up", out: Optional[torch.Tensor] = None,
          stream=None) -> torch.Tensor:
    _contig(x, "x")
    _contig(w, "w")
    M, K = x.shape
    Nd = w.shape[0]
    ydt = _NAME_DT[y_dtype]
    if out is None:
        out = torch.empty((M, Nd), dtype=_DT_TORCH[ydt], device=x.device)
    _contig(out, "out")
    _check_out(out, (M,), ydt)
    xq, wq, yq = _Q(x_scale, x_zp, 1), _per_tensor_or_channel(w_scale, w_zp), _Q(y_scale, y_zp, 1)
    _check(lib().qnn_dense(_stream(stream), _ptr(x), _dt(x), M, K, xq.q, _ptr(w), Nd, wq.q, _ptr(bias),
                           _ptr(out), ydt, yq.q, _clamp(act), _ROUND[rounding], out.shape[-1]))
    return out


def requantize(x: torch.Tensor, x_scale, x_zp, y_scale, y_zp, y_dtype="u8", act=None, rounding="half_up",
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Standalone requantize; qparams per tensor or per innermost channel."""
    _contig(x, "x")
    channels = x.shape[-1] if x.dim() else 1
    ydt = _NAME_DT[y_dtype]
    if out is None:
        out = torch.empty(x.shape, dtype=_DT_TORCH[ydt], device=x.device)
    _contig(out, "out")
    _check_out(out, tuple(x.shape), ydt, whole=True)
    xq, yq = _per_tensor_or_channel(x_scale, x_zp), _per_tensor_or_channel(y_scale, y_zp)
    _check(lib().qnn_requantize(_stream(stream), _ptr(x), _dt(x), x.numel(), channels, xq.q, _ptr(out), ydt, yq.q,
                                _clamp(act), _ROUND[rounding]))
    return out


def add(a: torch.Tensor, a_scale, a_zp, b: torch.Tensor, b_scale, b_zp, y_scale, y_zp, y_dtype="u8", act=None,
        rounding="half_up", out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """qnn.add of two same-shape tensors with different per-tensor qparams."""
    _contig(a, "a")
    _contig(b, "b")
    if a.shape != b.shape:
        raise ValueError("add operands must have the same shape")
    ydt = _NAME_DT[y_dtype]
    if out is None:
        out = torch.empty(a.shape, dtype=_DT_TORCH[ydt], device=a.device)
    _contig(out, "out")
    _check_out(out, tuple(a.shape), ydt, whole=True)
    aq, bq, yq = _Q(a_scale, a_zp, 1), _Q(b_scale, b_zp, 1), _Q(y_scale, y_zp, 1)
    _check(lib().qnn_add(_stream(stream), _ptr(a), _dt(a), aq.q, _ptr(b), _dt(b), bq.q, a.numel(), _ptr(out), ydt,
                         yq.q, _clamp(act), _ROUND[rounding]))
    return out


# Activations by name (qnn_activation).
ACTIVATIONS = {"gelu": 0, "gelu_tanh": 1, "silu": 2, "sigmoid": 3, "tanh": 4, "hard_swish": 5}


def _byte_table(table) -> np.ndarray:
    t = np.ascontiguousarray(table)
    if t.dtype not in (np.uint8, np.int8) or t.shape != (256,):
        raise ValueError("a table is 256 bytes (uint8 or int8)")
    return t.view(np.uint8)


def activation_table(kind: str, x_dtype, x_scale, x_zp, y_dtype, y_scale, y_zp) -> np.ndarray:
    """qnn_activation_table: the 256 output bytes (uint8), by the input's byte."""
    table = np.zeros(256, np.uint8)
    xq, yq = _Q(x_scale, x_zp, 1), _Q(y_scale, y_zp, 1)
    _check(lib().qnn_activation_table(ACTIVATIONS[kind], _NAME_DT[x_dtype], xq.q, _NAME_DT[y_dtype], yq.q,
                                      table.ctypes.data_as(ctypes.c_void_p)))
    return table


def lookup(x: torch.Tensor, table, y_dtype="i8", out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """y = table[x] by bytes (x u8 or i8, `table` 256 bytes on the host): an
    activation where a plan has none in its epilogue."""
    _contig(x, "x")
    if x.dtype not in (torch.uint8, torch.int8):
        raise TypeError(f"lookup takes u8 or i8, not {x.dtype}")
    ydt = _NAME_DT[y_dtype]
    if ydt == INT32:
        raise TypeError("lookup gives u8 or i8")
    if out is None:
        out = torch.empty(x.shape, dtype=_DT_TORCH[ydt], device=x.device)
    _contig(out, "out")
    _check_out(out, tuple(x.shape), ydt, whole=True)
    _check(lib().qnn_lookup(_stream(stream), _ptr(x), _byte_table(table).ctypes.data_as(ctypes.c_void_p), x.numel(),
                            _ptr(out)))
    return out


_POOL_MODE = {"avg": 0, "max": 1}


def pool2d(x: torch.Tensor, mode="avg", kernel=(3, 3), stride=(1, 1), pads=0, count_pad=False, zp=0,
           rounding="half_away", out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Quantized pool2d of Eq. (4): NHWC u8/i8 in, same dtype out, scale and
    zero point unchanged.  "avg" rounds sum / count to nearest (ties by
    ``rounding``, "half_up" or "half_away"; padded cells count as ``zp`` when
    ``count_pad``), "max" takes the largest in-input cell.  Enqueued on the
    stream, no synchronization."""
    _contig(x, "x")
    if x.dim() != 4:
        raise ValueError("pool2d input must be NHWC")
    N, H, W, C = x.shape
    R, S = (kernel, kernel) if isinstance(kernel, int) else kernel
    cp = _cp(stride, pads, 1)
    Ho = (H + cp.pad_top + cp.pad_bottom - R) // cp.stride_h + 1
    Wo = (W + cp.pad_left + cp.pad_right - S) // cp.stride_w + 1
    if out is None:
        out = torch.empty((N, max(Ho, 0), max(Wo, 0), C), dtype=x.dtype, device=x.device)
    _contig(out, "out")
    if out.dtype != x.dtype or tuple(out.shape) != (N, Ho, Wo, C):
        raise ValueError(f"pool2d out must be {x.dtype} of shape {(N, Ho, Wo, C)}")
    _check(lib().qnn_pool2d(_stream(stream), _ptr(x), _dt(x), N, H, W, C, R, S, cp, _POOL_MODE[mode],
                            int(bool(count_pad)), int(zp), _ptr(out), _ROUND[rounding]))
    return out


# ---------------------------------------------------------------- 4-bit cache

# Element types of the cache's operators; those above stay with whole numbers.
_FLOAT_DT = {**{k: v for k, v in _TORCH_DT.items() if k != torch.int32},
             torch.float16: FLOAT16, torch.bfloat16: BFLOAT16}
_FLOAT_NAME = {"u8": torch.uint8, "i8": torch.int8, "f16": torch.float16, "bf16": torch.bfloat16}
_NO_Q = QParams(None, None, 0)


def _i32(*values):
    """Numbers that become C ints: ctypes cuts longer ones off without a word."""
    if max(values) > INT32_MAX or min(values) < INT32_MIN:
        raise ValueError(f"{[v for v in values if not INT32_MIN <= v <= INT32_MAX]} does not fit 32 bits")


def _one_q(scale, zp) -> QParams:
    """Per-tensor qparams of two numbers (a tenth of _Q's time, which small calls see)."""
    _i32(zp)
    return QParams(ctypes.pointer(ctypes.c_float(scale)), ctypes.pointer(ctypes.c_int32(zp)), 1)


def _here(index: int, *tensors):
    """Every given tensor on device `index`, which must be the current one.
    (These checks are most of a small call's time on the host: no names or
    formatting unless something is wrong.)"""
    if index < 0:
        raise ValueError("the tensors must be device tensors")
    if index != (torch.cuda.current_device() if _raw_device is None else _raw_device()):
        raise ValueError(f"tensors on cuda:{index}, the current device is cuda:{torch.cuda.current_device()}")
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError(f"a tensor of {tuple(t.shape)} {t.dtype} is on {t.device}, not on cuda:{index}")


def _ints(t: Optional[torch.Tensor], name: str, count: Optional[int] = None):
    """A contiguous int32 vector (of `count` entries)."""
    if t is None:
        return
    if t.dtype is not torch.int32 or t.dim() != 1 or not t.is_contiguous() or (count is not None and
                                                                               t.numel() != count):
        raise ValueError(f"{name} must be a contiguous int32 vector" + ("" if count is None else f" of {count} entries")
                         + f", not {tuple(t.shape)} {t.dtype}")


def _heads(t: torch.Tensor, name: str, shape) -> int:
    """Row stride of a [tokens][heads][head_dim] tensor whose rows are contiguous."""
    if t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, expected {tuple(shape)}")
    T, H, D = shape
    if T == 0:
        return H * D
    row, head, one = t.stride()
    if D > 1 and one != 1 or H > 1 and head != D:
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    if T == 1:
        return H * D
    if row < H * D:
        raise ValueError(f"{name}: rows overlap (stride {row})")
    return row


def _table(t: torch.Tensor, rows: int) -> int:
    if t.dtype != torch.int32 or t.dim() != 2 or t.shape[0] != rows or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"the block table must be int32 [{rows}][pages] with contiguous rows, not {tuple(t.shape)} "
                         f"{t.dtype}")
    width = t.shape[1]
    if rows <= 1:
        return width
    ld = t.stride(0)
    if ld < width:
        raise ValueError(f"the block table's rows overlap (stride {ld})")
    return ld


class Cache4:
    """Keys and values of an attention as 4-bit codes, in pages (qnn_cache4):
    `data` is a uint8 tensor [num_pages][bytes of a page], allocated here unless
    given."""

    def __init__(self, num_pages: int, page_size: int, heads: int, head_dim: int, device="cuda",
                 data: Optional[torch.Tensor] = None):
        _i32(num_pages, page_size, heads, head_dim)
        per_page = int(lib().qnn_cache4_page_bytes(page_size, heads, head_dim))
        if per_page == 0 or num_pages < 1:
            raise ValueError(f"no cache of {num_pages} pages of {page_size} tokens, {heads} heads of {head_dim}: "
                             "page_size is 16, 32, 64, 128 or 256, head_dim a multiple of 8 up to 256")
        if data is None:
            data = torch.empty((num_pages, per_page), dtype=torch.uint8, device=device)
        if data.dtype != torch.uint8 or tuple(data.shape) != (num_pages, per_page) or not data.is_contiguous():
            raise ValueError(f"data must be contiguous uint8 {(num_pages, per_page)}, not {tuple(data.shape)} "
                             f"{data.dtype}")
        if not data.is_cuda:
            raise ValueError("data must be a device tensor")
        self.data, self.num_pages, self.page_size = data, num_pages, page_size
        self.heads, self.head_dim, self.device = heads, head_dim, data.get_device()
        self.desc = Cache4Desc(data.data_ptr(), num_pages, page_size, heads, head_dim)


def cache4_append(cache: Cache4, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, k_scale=1.0, k_zp=0,
                  v_scale=1.0, v_zp=0, stream=None) -> None:
    """Quantizes k and v ([tokens][heads][head_dim], f16, bf16, or u8 / i8 with
    their scale and zero point) to 4 bits at `slots` (int32; below 0: skipped);
    see qnn_cache4_append.  k and v may be slices of a wider tensor of rows."""
    T = k.shape[0]
    _i32(T)
    if stream is not None and stream.device_index != cache.device:
        raise ValueError(f"the stream is one of cuda:{stream.device_index}, the cache is on cuda:{cache.device}")
    _here(cache.device, k, v, slots)
    if k.dtype not in _FLOAT_DT or v.dtype != k.dtype:
        raise TypeError(f"k and v must both be f16, bf16, u8 or i8, not {k.dtype} and {v.dtype}")
    k_ld, v_ld = (_heads(t, n, (T, cache.heads, cache.head_dim)) for t, n in ((k, "k"), (v, "v")))
    _ints(slots, "slots", T)
    whole = k.dtype in (torch.uint8, torch.int8)
    status = lib().qnn_cache4_append(_stream_handle(stream), cache.desc, k.data_ptr(), v.data_ptr(),
                                     _FLOAT_DT[k.dtype], _one_q(k_scale, k_zp) if whole else _NO_Q,
                                     _one_q(v_scale, v_zp) if whole else _NO_Q, T, k_ld, v_ld, slots.data_ptr())
    if status:
        _check(status)


def cache4_read(cache: Cache4, slots: torch.Tensor, dtype="f16", stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(k, v) at `slots` as [slots][heads][head_dim] of dtype "f16" or "bf16";
    slots outside the cache give zeros.  See qnn_cache4_read."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return cache4_read(cache, slots, dtype)
    _here(cache.device, slots)
    _ints(slots, "slots")
    T = slots.numel()
    _i32(T)
    dt = _FLOAT_NAME[dtype]
    k, v = cache.data.new_empty((2, T, cache.heads, cache.head_dim), dtype=dt).unbind(0)
    ld = cache.heads * cache.head_dim
    status = lib().qnn_cache4_read(_stream_handle(), cache.desc, slots.data_ptr(), T, k.data_ptr(), v.data_ptr(),
                                   _FLOAT_DT[dt], ld, ld)
    if status:
        _check(status)
    return k, v


def attention4(q: torch.Tensor, cache: Cache4, block_table: torch.Tensor, ctx: torch.Tensor,
               cu_q: Optional[torch.Tensor] = None, max_q: Optional[int] = None, max_ctx: int = 0, scale: Optional[float] = None,
               causal=True, window: int = 0, q_scale=1.0, q_zp=0, y_scale=1.0, y_zp=0, y_dtype: Optional[str] = None,
               out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """Attention of q ([tokens][q_heads][head_dim], f16, bf16, or u8 / i8 with
    q_scale and q_zp) over the cache; see qnn_attention4.  Request b's queries
    are rows cu_q[b] .. cu_q[b + 1] - 1 (cu_q None: one each), the last of its
    ctx[b] tokens; block_table is int32 [requests][pages].  max_q is at least any
    request's queries, the rest of which stays uncomputed (None: that isn't known,
    all of q, for which the grid is that much larger), max_ctx (0: unknown) about
    the longest ctx.  scale defaults to head_dim ** -0.5.  Rows of q behind the last
    request's stay as they are in the output (in a new one: anything).  The output
    has y_dtype ("f16", "bf16", "u8", "i8"; q's by default), 8-bit ones with y_scale
    and y_zp.  `workspace` is a uint8 tensor of attention4_workspace_size() bytes,
    allocated here if not given; two calls that may overlap need one each."""
    if stream is not None:   # what is allocated here belongs to the stream that uses it
        with torch.cuda.stream(stream):
            return attention4(q, cache, block_table, ctx, cu_q, max_q, max_ctx, scale, causal, window, q_scale, q_zp,
                              y_scale, y_zp, y_dtype, out, workspace)
    if q.dim() != 3:
        raise ValueError("q must be [tokens][heads][head_dim]")
    T, Hq, D = q.shape
    B = ctx.numel()
    _here(cache.device, q, block_table, ctx, cu_q, out, workspace)
    if q.dtype not in _FLOAT_DT:
        raise TypeError(f"q must be f16, bf16, u8 or i8, not {q.dtype}")
    _ints(ctx, "ctx")
    _ints(cu_q, "cu_q", B + 1)
    q_ld = _heads(q, "q", (T, Hq, cache.head_dim))
    odt = q.dtype if y_dtype is None else _FLOAT_NAME[y_dtype]
    if out is None:
        out = q.new_empty((T, Hq, D), dtype=odt)
    elif out.dtype != odt:
        raise ValueError(f"out is {out.dtype}, not {odt}")
    table_ld = _table(block_table, B)
    if max_q is None:
        max_q = 1 if cu_q is None else max(T, 1)
    _i32(T, Hq, B, block_table.shape[1], max_q, max_ctx, window)
    p = AttentionParams(T, Hq, B, block_table.shape[1], q_ld, _heads(out, "out", (T, Hq, D)), table_ld, max_q, max_ctx,
                        1 if causal else 0, window, D ** -0.5 if scale is None else scale)
    need = lib().qnn_attention4_workspace_size(cache.desc, p)
    if workspace is None and need:
        workspace = cache.data.new_empty(need)
    have = 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        have = workspace.numel() * workspace.element_size()
    qq = _one_q(q_scale, q_zp) if q.dtype in (torch.uint8, torch.int8) else _NO_Q
    oq = _one_q(y_scale, y_zp) if odt in (torch.uint8, torch.int8) else _NO_Q
    status = lib().qnn_attention4(_stream_handle(), q.data_ptr(), _FLOAT_DT[q.dtype], qq, cache.desc,
                                  block_table.data_ptr(), ctx.data_ptr(), None if cu_q is None else cu_q.data_ptr(),
                                  p, out.data_ptr(), _FLOAT_DT[odt], oq,
                                  None if workspace is None else workspace.data_ptr(), have)
    if status:
        _check(status)
    return out


def attention4_workspace_size(cache: Cache4, tokens: int, q_heads: int, requests: int, table_width: int,
                              max_q: Optional[int] = None, max_ctx: int = 0, causal=True, window: int = 0) -> int:
    """Bytes of workspace of attention4 calls of these sizes (0: none)."""
    if max_q is None:
        max_q = max(tokens, 1)
    _i32(tokens, q_heads, requests, table_width, max_q, max_ctx, window)
    ld = q_heads * cache.head_dim
    p = AttentionParams(tokens, q_heads, requests, table_width, ld, ld, table_width, max_q, max_ctx, int(bool(causal)),
                        window, 1.0)
    return int(lib().qnn_attention4_workspace_size(cache.desc, p))


def pages_resize(lens: torch.Tensor, new_lens: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
                 free_count: torch.Tensor, page_size: int, token_capacity: int,
                 workspace: Optional[torch.Tensor] = None, stream=None):
    """Resizes requests of lens[b] tokens to new_lens[b]: block_table, lens, and
    the free stack (free_pages, free_count[0]) are updated, and every new token
    gets a slot; see qnn_pages_resize.  Returns (cu, slots, positions, status):
    request b's new tokens are slots[cu[b]:cu[b + 1]], unused entries -1; status
    (a device int32) is 0, or says why nothing was changed.  All arguments are
    int32 device tensors."""
    if stream is not None:   # what is allocated here belongs to the stream that uses it
        with torch.cuda.stream(stream):
            return pages_resize(lens, new_lens, block_table, free_pages, free_count, page_size, token_capacity, workspace)
    B = lens.numel()
    _here(lens.get_device(), new_lens, block_table, free_pages, free_count, workspace)
    _ints(lens, "lens")
    _ints(new_lens, "new_lens", B)
    _ints(free_pages, "free_pages")
    _ints(free_count, "free_count", 1)
    ld = _table(block_table, B)
    L = lib()
    _i32(B, page_size, block_table.shape[1], free_pages.numel(), token_capacity)
    need = L.qnn_pages_workspace_size(B)
    if token_capacity < 0:
        raise ValueError("token_capacity must be >= 0")
    if workspace is None:   # one allocation with the outputs
        work, cu, status, slots, positions = lens.new_empty(need // 4 + B + 2 + 2 * token_capacity).split_with_sizes(
            (need // 4, B + 1, 1, token_capacity, token_capacity))
        work = work.data_ptr()
    else:
        if not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
            raise ValueError("workspace must be contiguous and of qnn_pages_workspace_size() bytes")
        cu, status, slots, positions = lens.new_empty(B + 2 + 2 * token_capacity).split_with_sizes(
            (B + 1, 1, token_capacity, token_capacity))
        work = workspace.data_ptr()
    code = L.qnn_pages_resize(_stream_handle(), B, page_size, lens.data_ptr(), new_lens.data_ptr(),
                              block_table.data_ptr(), block_table.shape[1], ld, free_pages.data_ptr(),
                              free_pages.numel(), free_count.data_ptr(), cu.data_ptr(), slots.data_ptr(),
                              positions.data_ptr(), token_capacity, status.data_ptr(), work)
    if code:
        _check(code)
    return cu, slots, positions, status
