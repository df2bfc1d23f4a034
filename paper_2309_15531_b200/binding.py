"""ctypes binding of libadadim.so.

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  Functions take torch CUDA tensors (used purely as device buffers),
pass their data pointers and the current stream, and raise AdadimError on a
non-zero status.  There is no CPU fallback: if the library cannot be loaded,
every call fails with an ImportError naming the missing file.
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple
import os
from typing import Optional

import torch

OK = 0
F32, F16, BF16 = 0, 1, 2
DIM_OC, DIM_IC, DIM_BOTH, DIM_CHOSEN = 0, 1, 2, 3
WS_HESSIAN, WS_GPTQ, WS_SCORE, WS_FACTOR, WS_GPTQ_ROWS, WS_GEMV, WS_FP4 = 0, 1, 2, 3, 4, 5, 6
MXFP4, NVFP4 = 0, 1
DIM_NAMES = {DIM_OC: "oc", DIM_IC: "ic"}

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libadadim.so")
_lib = None


class AdadimError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({strerror(status)})")


class QTensorC(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("zeros", C.c_void_p)]


class Fp4TensorC(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("amax", C.c_void_p), ("ld", C.c_int64)]


class GptqLayerC(C.Structure):
    _fields_ = [("W", C.c_void_p), ("out", C.c_int64), ("ldw", C.c_int64), ("q_oc", C.POINTER(QTensorC)),
                ("q_ic", C.POINTER(QTensorC)), ("dim", C.c_int), ("chosen", C.c_void_p), ("gptq_loss", C.c_void_p)]


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2309_15531_b200.build` "
                              "(there is no CPU fallback)")
        L = C.CDLL(_LIB_PATH)
        i64, vp, sz = C.c_int64, C.c_void_p, C.c_size_t
        qp = C.POINTER(QTensorC)
        L.adadim_version.restype = C.c_int
        L.adadim_strerror.restype = C.c_char_p
        L.adadim_strerror.argtypes = [C.c_int]
        L.adadim_workspace_bytes.restype = sz
        L.adadim_workspace_bytes.argtypes = [C.c_int, i64, i64, C.c_int, C.c_int]
        L.adadim_hessian_accumulate.restype = C.c_int
        L.adadim_hessian_accumulate.argtypes = [vp, C.c_int, i64, i64, i64, vp, C.POINTER(i64), vp, vp, sz, vp]
        L.adadim_quantize_rtn.restype = C.c_int
        L.adadim_quantize_rtn.argtypes = [vp, C.c_int, i64, i64, i64, C.c_int, C.c_int, C.c_int, qp, qp, vp]
        L.adadim_cholesky_inverse_factor.restype = C.c_int
        L.adadim_cholesky_inverse_factor.argtypes = [vp, i64, C.c_double, vp, vp, vp, sz, vp]
        L.adadim_quantize_gptq.restype = C.c_int
        L.adadim_quantize_gptq.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, C.c_int, C.c_int, C.c_int, C.c_double,
                                           C.c_int, qp, qp, vp, vp, vp, sz, vp]
        L.adadim_quantize_gptq_batched.restype = C.c_int
        L.adadim_quantize_gptq_batched.argtypes = [C.POINTER(GptqLayerC), C.c_int, C.c_int, i64, vp, vp, C.c_int,
                                                   C.c_int, C.c_double, C.c_int, vp, vp, sz, vp]
        L.adadim_quantize_gptq_reordered.restype = C.c_int
        L.adadim_quantize_gptq_reordered.argtypes = [vp, C.c_int, i64, i64, i64, vp, C.c_int, C.c_int, C.c_int,
                                                     C.c_double, C.c_int, qp, qp, vp, vp, vp, vp, sz, vp]
        L.adadim_score_select.restype = C.c_int
        L.adadim_score_select.argtypes = [vp, C.c_int, i64, i64, i64, vp, C.c_int, C.c_int, qp, qp, vp, vp, vp, vp,
                                          sz, vp]
        L.adadim_score_select_static.restype = C.c_int
        L.adadim_score_select_static.argtypes = [vp, C.c_int, i64, i64, i64, vp, C.c_int, C.c_int, qp, qp, vp, vp,
                                                 vp, vp]
        L.adadim_static_scratch_bytes.restype = sz
        L.adadim_dequant_gemv.restype = C.c_int
        L.adadim_dequant_gemv.argtypes = [qp, C.c_int, i64, i64, C.c_int, C.c_int, vp, vp, vp, sz, vp]
        fp, ci = C.POINTER(Fp4TensorC), C.c_int
        L.adadim_fp4_scale_bytes.restype = sz
        L.adadim_fp4_scale_bytes.argtypes = [ci, i64, i64, ci]
        L.adadim_absmax.restype = ci
        L.adadim_absmax.argtypes = [vp, ci, i64, i64, i64, vp, vp]
        L.adadim_quantize_fp4.restype = ci
        L.adadim_quantize_fp4.argtypes = [vp, ci, i64, i64, i64, i64, ci, vp, vp, ci, fp, vp, ci, i64, vp]
        L.adadim_quantize_fp4_amax.restype = ci
        L.adadim_quantize_fp4_amax.argtypes = L.adadim_quantize_fp4.argtypes[:-1] + [vp, vp]
        L.adadim_fp4_matmul.restype = ci
        L.adadim_fp4_matmul.argtypes = [fp, i64, fp, i64, i64, ci, vp, ci, i64, vp, vp]
        L.adadim_fp4_matmul_grouped.restype = ci
        L.adadim_fp4_matmul_grouped.argtypes = [fp, i64, vp, ci, fp, i64, i64, ci, vp, ci, i64, vp, vp]
        L.adadim_fp4_linear.restype = ci
        L.adadim_fp4_linear.argtypes = [vp, ci, i64, i64, i64, vp, fp, i64, ci, vp, ci, i64, vp, vp, sz, vp]
        L.adadim_fp4_linear_grouped.restype = ci
        L.adadim_fp4_linear_grouped.argtypes = [vp, ci, i64, i64, i64, vp, vp, vp, ci, i64, fp, i64, ci, vp, ci, i64,
                                                vp, vp, sz, vp]
        L.adadim_fp4_plan.restype = ci
        L.adadim_fp4_plan.argtypes = [i64, i64, i64, ci, ci, ci, ci, C.POINTER(C.c_int)]
        L.adadim_unpack_codes.restype = C.c_int
        L.adadim_unpack_codes.argtypes = [vp, i64, i64, C.c_int, vp, vp]
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().adadim_strerror(int(status)).decode()


def version() -> int:
    return lib().adadim_version()


def workspace_bytes(kind: int, out: int, inp: int, bits: int = 0, group: int = 0) -> int:
    return int(lib().adadim_workspace_bytes(kind, out, inp, bits, group))


_DT = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# The current device, and the handle of a device's current stream without a Stream object (3.5 us on the measured host).
_device, _raw_stream = (getattr(torch._C, name, None) for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))


def _check(rc: int, where: str):
    if rc != OK:
        raise AdadimError(rc, where)


class QTensor:
    """Device buffers of one quantized tensor (see include/adadim.h for the layout)."""

    def __init__(self, out: int, inp: int, bits: int, group: int, dim: int, device="cuda"):
        self.out, self.inp, self.bits, self.group, self.dim = out, inp, bits, group, dim
        self.codes = torch.zeros(out, inp * bits // 32, dtype=torch.int32, device=device)
        shape = (out, inp // group) if dim == DIM_OC else (out // group, inp)
        self.scales = torch.zeros(shape, dtype=torch.float16, device=device)
        self.zeros = torch.zeros(shape, dtype=torch.float16, device=device)

    def c(self) -> QTensorC:
        return QTensorC(self.codes.data_ptr(), self.scales.data_ptr(), self.zeros.data_ptr())

    def unpacked(self) -> torch.Tensor:
        dst = torch.empty(self.out, self.inp, dtype=torch.uint8, device=self.codes.device)
        _check(lib().adadim_unpack_codes(self.codes.data_ptr(), self.out, self.inp, self.bits, dst.data_ptr(),
                                         _stream()), "adadim_unpack_codes")
        return dst


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def hessian_accumulate(X: torch.Tensor, H: torch.Tensor, status: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, tensor_cores: bool = True) -> None:
    """H += 2 X^T X for X[n_tokens, in] (bf16 or fp32), H[in, in] fp32.  fp32 X runs on the tensor cores
    through a workspace (allocated here if none is given); tensor_cores=False selects the plain kernel."""
    assert X.is_cuda and H.is_cuda and X.stride(1) == 1 and H.is_contiguous()
    ws_ptr, ws_len = None, 0
    if X.dtype == torch.float32 and tensor_cores and X.shape[0] > 0:
        if workspace is None:
            workspace = _ws(workspace_bytes(WS_HESSIAN, X.shape[0], X.shape[1]), X.device)
        ws_ptr, ws_len = workspace.data_ptr(), workspace.numel()
    rc = lib().adadim_hessian_accumulate(X.data_ptr(), _DT[X.dtype], X.shape[0], X.shape[1], X.stride(0),
                                         H.data_ptr(), None, status.data_ptr() if status is not None else None,
                                         ws_ptr, ws_len, _stream())
    _check(rc, "adadim_hessian_accumulate")


def quantize_rtn(W: torch.Tensor, bits: int, group: int, dim: int = DIM_BOTH,
                 q_oc: Optional[QTensor] = None, q_ic: Optional[QTensor] = None):
    assert W.is_cuda and W.stride(1) == 1
    out, inp = W.shape
    if dim != DIM_IC and q_oc is None:
        q_oc = QTensor(out, inp, bits, group, DIM_OC, W.device)
    if dim != DIM_OC and q_ic is None:
        q_ic = QTensor(out, inp, bits, group, DIM_IC, W.device)
    coc = q_oc.c() if q_oc is not None else None
    cic = q_ic.c() if q_ic is not None else None
    rc = lib().adadim_quantize_rtn(W.data_ptr(), _DT[W.dtype], out, inp, W.stride(0), bits, group, dim,
                                   C.byref(coc) if coc is not None else None,
                                   C.byref(cic) if cic is not None else None, _stream())
    _check(rc, "adadim_quantize_rtn")
    return q_oc, q_ic


def cholesky_inverse_factor(H: torch.Tensor, percdamp: float = 0.01, status: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None, U: Optional[torch.Tensor] = None) -> torch.Tensor:
    n = H.shape[0]
    if U is None:
        U = torch.empty(n, n, dtype=torch.float64, device=H.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_FACTOR, 0, n), H.device)
    rc = lib().adadim_cholesky_inverse_factor(H.data_ptr(), n, percdamp, U.data_ptr(),
                                              status.data_ptr() if status is not None else None,
                                              workspace.data_ptr(), workspace.numel(), _stream())
    _check(rc, "adadim_cholesky_inverse_factor")
    return U


def quantize_gptq(W: torch.Tensor, H: torch.Tensor, bits: int, group: int, dim: int = DIM_BOTH,
                  percdamp: float = 0.01, U: Optional[torch.Tensor] = None,
                  q_oc: Optional[QTensor] = None, q_ic: Optional[QTensor] = None,
                  loss: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None):
    assert W.is_cuda and W.stride(1) == 1 and H.is_contiguous()
    out, inp = W.shape
    if dim != DIM_IC and q_oc is None:
        q_oc = QTensor(out, inp, bits, group, DIM_OC, W.device)
    if dim != DIM_OC and q_ic is None:
        q_ic = QTensor(out, inp, bits, group, DIM_IC, W.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_GPTQ, out, inp, bits, group), W.device)
    coc = q_oc.c() if q_oc is not None else None
    cic = q_ic.c() if q_ic is not None else None
    rc = lib().adadim_quantize_gptq(W.data_ptr(), _DT[W.dtype], out, inp, W.stride(0), H.data_ptr(),
                                    U.data_ptr() if U is not None else None, bits, group, dim, percdamp, 128,
                                    C.byref(coc) if coc is not None else None,
                                    C.byref(cic) if cic is not None else None,
                                    loss.data_ptr() if loss is not None else None,
                                    status.data_ptr() if status is not None else None,
                                    workspace.data_ptr(), workspace.numel(), _stream())
    _check(rc, "adadim_quantize_gptq")
    return q_oc, q_ic


def quantize_gptq_batched(Ws, H: torch.Tensor, bits: int, group: int, dims, percdamp: float = 0.01,
                          U: Optional[torch.Tensor] = None, chosen=None, qs=None, losses=None,
                          status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """GPTQ for layers that share H (and U): one call, one chain of column steps for all of them.
    Ws: list of weights [out_l, in] of one dtype; dims: one of DIM_OC / DIM_IC / DIM_BOTH / DIM_CHOSEN per
    layer; chosen: per layer a device int32[1] (required for DIM_CHOSEN, e.g. score_select's output);
    qs: optional list of (q_oc, q_ic) to write into.  Returns the list of (q_oc, q_ic); with DIM_CHOSEN
    both are allocated and the one named by the device word is written."""
    n = len(Ws)
    inp = Ws[0].shape[1]
    assert all(w.is_cuda and w.stride(1) == 1 and w.shape[1] == inp and w.dtype == Ws[0].dtype for w in Ws)
    out_qs, keep, arr = [], [], (GptqLayerC * n)()
    rows = 0
    for l, W in enumerate(Ws):
        out, dim = W.shape[0], dims[l]
        q_oc, q_ic = qs[l] if qs is not None else (None, None)
        if dim != DIM_IC and q_oc is None:
            q_oc = QTensor(out, inp, bits, group, DIM_OC, W.device)
        if dim != DIM_OC and q_ic is None:
            q_ic = QTensor(out, inp, bits, group, DIM_IC, W.device)
        coc = q_oc.c() if q_oc is not None else None
        cic = q_ic.c() if q_ic is not None else None
        keep.append((coc, cic))
        arr[l].W, arr[l].out, arr[l].ldw, arr[l].dim = W.data_ptr(), out, W.stride(0), dim
        arr[l].q_oc = C.pointer(coc) if coc is not None else None
        arr[l].q_ic = C.pointer(cic) if cic is not None else None
        arr[l].chosen = chosen[l].data_ptr() if chosen is not None and chosen[l] is not None else None
        arr[l].gptq_loss = losses[l].data_ptr() if losses is not None and losses[l] is not None else None
        out_qs.append((q_oc, q_ic))
        rows += out * (2 if dim == DIM_BOTH else 1)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_GPTQ_ROWS, rows, inp, bits, group), Ws[0].device)
    rc = lib().adadim_quantize_gptq_batched(arr, n, _DT[Ws[0].dtype], inp, H.data_ptr(),
                                            U.data_ptr() if U is not None else None, bits, group, percdamp, 128,
                                            status.data_ptr() if status is not None else None,
                                            workspace.data_ptr(), workspace.numel(), _stream())
    _check(rc, "adadim_quantize_gptq_batched")
    return out_qs


def quantize_gptq_reordered(W: torch.Tensor, H: torch.Tensor, bits: int, group: int, dim: int = DIM_BOTH,
                            percdamp: float = 0.01,
                            q_oc: Optional[QTensor] = None, q_ic: Optional[QTensor] = None,
                            loss: Optional[torch.Tensor] = None, perm: Optional[torch.Tensor] = None,
                            status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """GPTQ with activation reordering (per-IC: dynamic groups; per-OC: static groups).
    `perm`, if given, is an int32[in] device tensor that receives the column order."""
    assert W.is_cuda and W.stride(1) == 1 and H.is_contiguous()
    out, inp = W.shape
    if dim != DIM_IC and q_oc is None:
        q_oc = QTensor(out, inp, bits, group, DIM_OC, W.device)
    if dim != DIM_OC and q_ic is None:
        q_ic = QTensor(out, inp, bits, group, DIM_IC, W.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_GPTQ, out, inp, bits, group), W.device)
    coc = q_oc.c() if q_oc is not None else None
    cic = q_ic.c() if q_ic is not None else None
    rc = lib().adadim_quantize_gptq_reordered(W.data_ptr(), _DT[W.dtype], out, inp, W.stride(0), H.data_ptr(),
                                              bits, group, dim, percdamp, 128,
                                              C.byref(coc) if coc is not None else None,
                                              C.byref(cic) if cic is not None else None,
                                              loss.data_ptr() if loss is not None else None,
                                              perm.data_ptr() if perm is not None else None,
                                              status.data_ptr() if status is not None else None,
                                              workspace.data_ptr(), workspace.numel(), _stream())
    _check(rc, "adadim_quantize_gptq_reordered")
    return q_oc, q_ic


def score_select(W: torch.Tensor, H: torch.Tensor, bits: int, group: int,
                 q_oc: Optional[QTensor], q_ic: Optional[QTensor],
                 err: Optional[torch.Tensor] = None, chosen: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Returns (err float64[2] = (E_oc, E_ic), chosen int32[1]) as device tensors."""
    assert W.is_cuda and W.stride(1) == 1 and H.is_contiguous()
    out, inp = W.shape
    if err is None:
        err = torch.empty(2, dtype=torch.float64, device=W.device)
    if chosen is None:
        chosen = torch.empty(1, dtype=torch.int32, device=W.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_SCORE, out, inp, bits, group), W.device)
    coc = q_oc.c() if q_oc is not None else None
    cic = q_ic.c() if q_ic is not None else None
    rc = lib().adadim_score_select(W.data_ptr(), _DT[W.dtype], out, inp, W.stride(0), H.data_ptr(), bits, group,
                                   C.byref(coc) if coc is not None else None,
                                   C.byref(cic) if cic is not None else None,
                                   err.data_ptr(), chosen.data_ptr(),
                                   status.data_ptr() if status is not None else None,
                                   workspace.data_ptr(), workspace.numel(), _stream())
    _check(rc, "adadim_score_select")
    return err, chosen


def dequant_gemv(codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, bits: int, group: int,
                 x: torch.Tensor, y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = Q x for a per-IC quantized layer: codes int32 [out, in*bits/32], scales / zeros fp16
    [out/group, in], x fp16 [in]; returns y fp16 [out]."""
    out, inp = codes.shape[0], scales.shape[1]
    assert x.dtype == torch.float16 and x.is_contiguous() and codes.is_contiguous()
    if y is None:
        y = torch.empty(out, dtype=torch.float16, device=x.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_GEMV, out, inp, bits, group), x.device)
    qc = QTensorC(codes.data_ptr(), scales.data_ptr(), zeros.data_ptr())
    rc = lib().adadim_dequant_gemv(C.byref(qc), DIM_IC, out, inp, bits, group, x.data_ptr(), y.data_ptr(),
                                   workspace.data_ptr(), workspace.numel(), _stream())
    _check(rc, "adadim_dequant_gemv")
    return y


class _TensorScale:
    """The amax that NVFP4's tensor scale is taken from, of a matrix or of a stack of experts: a copy of its value on the
    device, so that what the caller does with an amax later changes no product, and which of the matrices were quantized
    with it."""

    def __init__(self, device, shared: bool):
        self.shared = shared                              # by the experts of a stack
        self.value = torch.empty(1, dtype=torch.float32, device=device)
        self.present = False                              # False: no amax, tensor scale 1
        self.fixed = False                                # a stack has one; its first expert or set_amax fixes it
        self.given: Optional[torch.Tensor] = None         # the tensor that a stack's was copied from, and its version
        self.version = 0
        self.done: set = set()                            # matrices that were quantized with it
        self.stale: set = set()                           # .. and with an earlier one, not again since
        self.state = object()                             # another one whenever `present` or `stale` changes

    @staticmethod
    def _version(t: torch.Tensor) -> int:
        return 0 if t.is_inference() else t._version

    def same(self, amax: Optional[torch.Tensor]) -> bool:
        """Whether it is known that amax holds the value kept here."""
        if amax is None or not self.present:
            return amax is None and not self.present
        p = amax.data_ptr()
        return p == self.value.data_ptr() or (self.given is not None and p == self.given.data_ptr()
                                              and self._version(amax) == self.version)

    def _fix(self, amax: Optional[torch.Tensor]) -> None:
        self.present, self.fixed, self.state = amax is not None, True, object()
        if self.shared and amax is not None and amax.data_ptr() != self.value.data_ptr():
            self.given, self.version = amax, self._version(amax)

    def change(self, amax: Optional[torch.Tensor]) -> None:
        if not self.same(amax):
            self.stale |= self.done
            self.done.clear()
        if amax is not None and amax.data_ptr() != self.value.data_ptr():
            self.value.copy_(amax.reshape(1))
        self._fix(amax)

    def quantized(self, k: int, amax: Optional[torch.Tensor]) -> None:
        """Matrix k was quantized with amax, and a call that had to fix the amax has copied it."""
        self.done.add(k)
        self.stale.discard(k)
        self._fix(amax)


class Fp4Tensor:
    """Device buffers of a matrix in microscaled 4-bit floating point (see include/adadim.h for the layout).
    `groups` > 0: the rows are in that many groups given by an offsets tensor (activations sorted by
    expert).  `experts` > 0: a stack of that many [rows, cols] weights; expert(e) is a view of one."""

    def __init__(self, rows: int, cols: int, fmt: int, groups: int = 0, experts: int = 0, device="cuda"):
        if rows < 0 or cols < 0 or fmt not in (MXFP4, NVFP4) or groups < 0 or experts < 0 or (groups and experts):
            raise ValueError("Fp4Tensor: bad sizes or format")
        self.rows, self.cols, self.fmt, self.groups, self.experts = rows, cols, fmt, groups, experts
        n = max(experts, 1)
        self.scale_bytes = int(lib().adadim_fp4_scale_bytes(fmt, rows, cols, groups))
        ld = ((cols + 1) // 2 + 15) // 16 * 16
        self._buffers = (torch.zeros(n * rows, ld, dtype=torch.uint8, device=device),
                         torch.zeros(n * self.scale_bytes, dtype=torch.uint8, device=device))
        self.dev = self._buffers[0].get_device()
        self.stack: Optional["Fp4Tensor"] = None          # of an expert's view
        self._index = 0                                   # of this matrix in the stack
        self._scale = _TensorScale(device, experts > 0)
        self._c = self._c_of = self._product = self._state = None

    def expert(self, e: int) -> "Fp4Tensor":
        if not 0 <= e < self.experts:
            raise IndexError(e)
        one = object.__new__(Fp4Tensor)
        one.rows, one.cols, one.fmt, one.groups, one.experts = self.rows, self.cols, self.fmt, 0, 0
        one.scale_bytes, one.dev, one.stack, one._index, one._scale = self.scale_bytes, self.dev, self, e, self._scale
        one._c = one._c_of = one._product = one._state = None
        return one

    # Buffers may be replaced (by ones that were loaded, say), in a stack those of all experts together; views follow.
    @property
    def codes(self) -> torch.Tensor:
        if self.stack is not None:
            return self.stack.codes[self._index * self.rows:(self._index + 1) * self.rows]
        return self._buffers[0]

    @codes.setter
    def codes(self, t: torch.Tensor) -> None:
        old = self._replaceable(t)[0]
        if t.shape != old.shape or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError("Fp4Tensor: codes of another shape or order")
        self._replace(t, self._buffers[1])

    @property
    def scales(self) -> torch.Tensor:
        if self.stack is not None:
            return self.stack.scales[self._index * self.scale_bytes:(self._index + 1) * self.scale_bytes]
        return self._buffers[1]

    @scales.setter
    def scales(self, t: torch.Tensor) -> None:
        old = self._replaceable(t)[1]
        if t.shape != old.shape or not t.is_contiguous():
            raise ValueError("Fp4Tensor: scales of another shape or order")
        self._replace(self._buffers[0], t)

    def _replaceable(self, t: torch.Tensor):
        if self.stack is not None:
            raise ValueError("Fp4Tensor: replace the buffers of the stack")
        if t.dtype != torch.uint8 or t.get_device() != self.dev:
            raise ValueError("Fp4Tensor: a buffer of another type or device")
        return self._buffers

    def _replace(self, codes: torch.Tensor, scales: torch.Tensor) -> None:
        self._buffers = (codes, scales)
        self._scale.state = object()
        self._scale.done.clear()                          # the caller answers for what comes from elsewhere
        self._scale.stale.clear()

    @property
    def amax(self) -> Optional[torch.Tensor]:
        """float32[1], the largest magnitude that NVFP4's tensor scale is taken from; None: tensor scale 1 (or MXFP4)."""
        return self._scale.value if self._scale.present else None

    @amax.setter
    def amax(self, amax: Optional[torch.Tensor]) -> None:
        self.set_amax(amax)

    def set_amax(self, amax: Optional[torch.Tensor]) -> None:
        """Sets the amax (its value is copied).  Matrices that were quantized with another have to be quantized again:
        a product that needs one of them raises ValueError until then.  A stack has one amax for all its experts: the
        first expert that is quantized sets it, or a call on the stack itself."""
        if amax is not None:
            assert amax.is_cuda
            _amax(amax, self.dev)
        if self.fmt != NVFP4:
            return                                        # MXFP4 has no tensor scale
        if self.stack is not None and self._scale.fixed and not self._scale.same(amax):
            raise ValueError("the experts of a stack share one amax: set_amax on the stack first")
        self._scale.change(amax)

    def _both(self):
        """What the quantizer takes: without an amax, and with the one that is kept."""
        buffers = (self.stack or self)._buffers
        if self._c_of is not buffers:
            codes, scales = self.codes, self.scales
            p, s, ld = codes.data_ptr(), scales.data_ptr(), codes.stride(0)
            self._c, self._c_of = (Fp4TensorC(p, s, None, ld), Fp4TensorC(p, s, self._scale.value.data_ptr(), ld)), buffers
        return self._c

    def c(self) -> Fp4TensorC:
        return self._both()[self._scale.present]

    def _operand(self):
        """What a product takes, by reference."""
        scale = self._scale
        if self._state is not scale.state:
            if scale.stale and (self.experts or self._index in scale.stale):
                raise ValueError("the amax was changed after this was quantized: quantize it again")
            self._product, self._state = C.byref(self.c()), scale.state
        return self._product


def _amax(t: Optional[torch.Tensor], dev: int):
    if t is None:
        return None
    assert t.get_device() == dev and t.dtype == torch.float32 and t.numel() == 1
    return t.data_ptr()


def _status(t: Optional[torch.Tensor], dev: int):
    if t is None:
        return None
    p = t.data_ptr()                                      # 0 if it is empty
    assert p and t.get_device() == dev and t.dtype == torch.int32
    return p


def _i32(t: torch.Tensor, dev: int) -> torch.Tensor:
    assert t.get_device() == dev and t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous()
    return t


def _matrix_in(X: torch.Tensor):
    """(pointer, dtype code, rows, columns, pitch, device index) of a row-major matrix; as few tensor queries as
    possible, for the small products whose time is the caller's."""
    rows, cols = X.shape
    ld, step = X.stride()
    dev = X.get_device()
    assert dev >= 0 and (cols <= 1 or step == 1)
    return X.data_ptr(), _DT[X.dtype], rows, cols, (ld if rows > 1 or ld > cols else cols), dev


def absmax(X: torch.Tensor, amax: Optional[torch.Tensor] = None) -> torch.Tensor:
    """float32[1] = max(amax, max |X|); pass the same tensor for several chunks."""
    xp, xdt, rows, cols, ldx, dev = _matrix_in(X)
    if amax is None:
        amax = torch.zeros(1, dtype=torch.float32, device=X.device)
    if dev != _device():
        with torch.cuda.device(dev):
            return absmax(X, amax)
    _check(lib().adadim_absmax(xp, xdt, rows, cols, ldx, _amax(amax, dev), _raw_stream(dev)), "adadim_absmax")
    torch.autograd.graph.increment_version(amax)         # as any operation in place does
    return amax


def quantize_fp4(X: torch.Tensor, fmt: int, amax: Optional[torch.Tensor] = None, q: Optional[Fp4Tensor] = None,
                 values: Optional[torch.Tensor] = None, row_index: Optional[torch.Tensor] = None,
                 offsets: Optional[torch.Tensor] = None) -> Fp4Tensor:
    """Quantize X[rows, cols] (fp32, fp16 or bf16) to MXFP4 or NVFP4.  amax: float32[1], NVFP4's tensor scale is
    taken from it (None: 1) and the result keeps a copy of it.  values (bf16 or fp32 [rows, cols]): receives the
    quantized values.  row_index int32[rows]: take row r from X[row_index[r]].  offsets int32[n + 1]: the rows are in
    n groups (see Fp4Tensor)."""
    xp, xdt, x_rows, cols, ldx, dev = _matrix_in(X)
    if dev != _device():
        with torch.cuda.device(dev):
            return quantize_fp4(X, fmt, amax, q, values, row_index, offsets)
    rows, ip = (x_rows, None) if row_index is None else (_i32(row_index, dev).numel(), row_index.data_ptr())
    groups, op = (0, None) if offsets is None else (_i32(offsets, dev).numel() - 1, offsets.data_ptr())
    if q is None:
        q = Fp4Tensor(rows, cols, fmt, groups=groups, device=X.device)
    if q.rows != rows or q.cols != cols or q.fmt != fmt or q.groups != groups or q.experts or q.dev != dev:
        raise ValueError("quantize_fp4: q was made for another shape, format or device")
    vp, vdt, ldv = None, BF16, 0
    if values is not None:
        vp, vdt, v_rows, v_cols, ldv, v_dev = _matrix_in(values)
        assert v_rows == rows and v_cols == cols and v_dev == dev
    scale, nv, alone = q._scale, fmt == NVFP4, q.stack is None
    given = _amax(amax, dev)
    if not nv:
        given = None
    if alone or not scale.fixed:
        source = given                                    # the call copies its value to where q keeps it
    elif not nv or scale.same(amax):
        source = None
    else:
        raise ValueError("the experts of a stack share one amax: set_amax on the stack first")
    rc = (_lib or lib()).adadim_quantize_fp4_amax(xp, xdt, rows, cols, ldx, x_rows, fmt, ip, op, groups,
                                                  C.byref(q._both()[given is not None]), vp, vdt, ldv, source,
                                                  _raw_stream(dev))
    if rc:
        _check(rc, "adadim_quantize_fp4")
    if nv and not (alone and scale.done and scale.present == (given is not None)):
        scale.quantized(q._index, amax)
    return q


def _fp4_operands(X: Fp4Tensor, W: Fp4Tensor, y: Optional[torch.Tensor]):
    """The result of a product of two 4-bit matrices, with its pointer, dtype code and pitch."""
    if W.dev != X.dev:
        raise ValueError("X and W are on different devices")
    if y is None:
        y = torch.empty(X.rows, W.rows, dtype=torch.bfloat16, device=X.codes.device)
    yp, ydt, rows, cols, ldy, dev = _matrix_in(y)
    assert rows == X.rows and cols == W.rows and dev == X.dev
    return y, yp, ydt, ldy


def fp4_linear(X, W: Fp4Tensor, x_amax: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = Q(X) W^T for activations X[n_tokens, in] (fp32, fp16, bf16; quantized in the call with x_amax) or for an
    Fp4Tensor X that is quantized already (y is bf16 then unless given).  y has X's type unless given.  NVFP4 without an
    x_amax has tensor scale 1: what lies above 2688 saturates.  For inference: no gradient passes to X."""
    if W.experts:
        raise ValueError("fp4_linear: W is a stack of experts")
    if isinstance(X, Fp4Tensor):
        if X.fmt != W.fmt or X.cols != W.cols or X.groups or X.experts:
            raise ValueError("fp4_linear: X and W do not match")
        y, yp, ydt, ldy = _fp4_operands(X, W, y)
        with torch.cuda.device(X.dev):
            _check(lib().adadim_fp4_matmul(X._operand(), X.rows, W._operand(), W.rows, W.cols, W.fmt, yp, ydt, ldy,
                                           _status(status, X.dev), _raw_stream(X.dev)), "adadim_fp4_matmul")
        return y
    xp, xdt, rows, inp, ldx, dev = _matrix_in(X)
    if inp != W.cols or dev != W.dev:
        raise ValueError("fp4_linear: X and W do not match")
    if dev != _device():
        with torch.cuda.device(dev):
            return fp4_linear(X, W, x_amax, y, workspace, status)
    if y is None:
        y = torch.empty(rows, W.rows, dtype=X.dtype, device=X.device)
    yp, ydt, y_rows, out, ldy, y_dev = _matrix_in(y)
    assert y_rows == rows and out == W.rows and y_dev == dev
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_FP4, rows, inp, 4, 0), X.device)
    assert workspace.get_device() == dev and workspace.dtype == torch.uint8
    rc = (_lib or lib()).adadim_fp4_linear(xp, xdt, rows, inp, ldx, _amax(x_amax, dev), W._operand(), out, W.fmt, yp, ydt,
                                           ldy, _status(status, dev), workspace.data_ptr(), workspace.numel(),
                                           _raw_stream(dev))
    if rc:
        _check(rc, "adadim_fp4_linear")
    return y


def fp4_linear_grouped(X, offsets: torch.Tensor, W: Fp4Tensor, row_index: Optional[torch.Tensor] = None,
                       x_amax: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The product for rows sorted by expert: rows offsets[e] .. offsets[e+1]-1 (int32 on the device) are
    multiplied by expert e of the stack W.  Row r is X[row_index[r]] (None: X[r]); X may be an Fp4Tensor with
    groups.  Rows of no expert are not written.  For inference: no gradient passes to X."""
    n = _i32(offsets, W.dev).numel() - 1
    if W.experts != n or n < 1:
        raise ValueError("fp4_linear_grouped: offsets do not match the stack of experts")
    if isinstance(X, Fp4Tensor):
        if X.fmt != W.fmt or X.cols != W.cols or X.groups != n or row_index is not None:
            raise ValueError("fp4_linear_grouped: X and W do not match")
        y, yp, ydt, ldy = _fp4_operands(X, W, y)
        with torch.cuda.device(X.dev):
            _check(lib().adadim_fp4_matmul_grouped(X._operand(), X.rows, offsets.data_ptr(), n, W._operand(), W.rows, W.cols,
                                                   W.fmt, yp, ydt, ldy, _status(status, X.dev), _raw_stream(X.dev)),
                   "adadim_fp4_matmul_grouped")
        return y
    xp, xdt, x_rows, inp, ldx, dev = _matrix_in(X)
    if inp != W.cols or dev != W.dev:
        raise ValueError("fp4_linear_grouped: X and W do not match")
    if dev != _device():
        with torch.cuda.device(dev):
            return fp4_linear_grouped(X, offsets, W, row_index, x_amax, y, workspace, status)
    rows, ip = (x_rows, None) if row_index is None else (_i32(row_index, dev).numel(), row_index.data_ptr())
    if y is None:
        y = torch.empty(rows, W.rows, dtype=X.dtype, device=X.device)
    yp, ydt, y_rows, out, ldy, y_dev = _matrix_in(y)
    assert y_rows == rows and out == W.rows and y_dev == dev
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_FP4, rows, inp, 4, n), X.device)
    assert workspace.get_device() == dev and workspace.dtype == torch.uint8
    rc = (_lib or lib()).adadim_fp4_linear_grouped(xp, xdt, x_rows, inp, ldx, _amax(x_amax, dev), ip, offsets.data_ptr(), n,
                                                   rows, W._operand(), out, W.fmt, yp, ydt, ldy, _status(status, dev),
                                                   workspace.data_ptr(), workspace.numel(), _raw_stream(dev))
    if rc:
        _check(rc, "adadim_fp4_linear_grouped")
    return y


Fp4Plan = namedtuple("Fp4Plan", "many token_tile splits ctas_per_sm fused")


def fp4_plan(rows: int, out: int, inp: int, fmt: int, experts: int = 0, quantized: bool = False, aligned: bool = True) -> Fp4Plan:
    """How fp4_linear lays out a product (fp4_linear_grouped with `experts`): see include/adadim.h.  Host only."""
    plan = (C.c_int * 5)()
    _check(lib().adadim_fp4_plan(rows, out, inp, experts, fmt, quantized, aligned, plan), "adadim_fp4_plan")
    return Fp4Plan(bool(plan[0]), plan[1], plan[2], plan[3], bool(plan[4]))


def static_scratch_bytes() -> int:
    return int(lib().adadim_static_scratch_bytes())


def score_select_static(W: torch.Tensor, H: torch.Tensor, bits: int, group: int,
                        q_oc: Optional[QTensor], q_ic: Optional[QTensor],
                        err: torch.Tensor, chosen: torch.Tensor, status: Optional[torch.Tensor] = None) -> None:
    """score_select on the library's built-in scratch array, for callers that cannot allocate
    device memory.  The caller passes every buffer, outputs included (err float64[2], chosen
    int32[1]); this wrapper creates no tensor.  Layers whose scoring workspace exceeds
    static_scratch_bytes() raise AdadimError(status 6).  Calls on one device must not overlap
    on the GPU: they share the array."""
    out, inp = W.shape
    coc = q_oc.c() if q_oc is not None else None
    cic = q_ic.c() if q_ic is not None else None
    rc = lib().adadim_score_select_static(W.data_ptr(), _DT[W.dtype], out, inp, W.stride(0), H.data_ptr(), bits, group,
                                          C.byref(coc) if coc is not None else None,
                                          C.byref(cic) if cic is not None else None,
                                          err.data_ptr(), chosen.data_ptr(),
                                          status.data_ptr() if status is not None else None, _stream())
    _check(rc, "adadim_score_select_static")
