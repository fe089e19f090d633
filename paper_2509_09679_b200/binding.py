"""ctypes binding of libbfq.so: the same names as the C ABI, argument marshalling only.

Every step of the path runs in the CUDA kernels behind these calls.  There is no CPU
fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os

import torch

from .kv_cache import KVCache

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbfq.so")

BFQ_F32, BFQ_BF16 = 0, 1
BFQ_OK = 0
STATUS_NAMES = {
    0: "BFQ_OK", -1: "BFQ_ERR_NULL", -2: "BFQ_ERR_UNSUPPORTED_N", -3: "BFQ_ERR_BITS", -4: "BFQ_ERR_ALIGN",
    -5: "BFQ_ERR_STRIDE", -6: "BFQ_ERR_DTYPE", -7: "BFQ_ERR_WORKSPACE", -8: "BFQ_ERR_CUDA",
    -9: "BFQ_ERR_DEVICE_TIMEOUT", -10: "BFQ_ERR_TOO_LARGE", -11: "BFQ_ERR_INDEX",
}

# name -> (restype, argtypes); must list every symbol include/bfq.h declares
_i, _i64, _p = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
SIGNATURES = {
    "bfq_plan_create": (_i, [ctypes.POINTER(_p), _i, _i64, _i]),
    "bfq_plan_destroy": (_i, [_p]),
    "bfq_set_angles": (_i, [_p, _p, _p]),
    "bfq_forward": (_i, [_p, _p, _i, _i64, _i64, _p, _i, _i64, _p]),
    "bfq_forward_quant": (_i, [_p, _p, _i, _i64, _i64, _i, _p, _p, _p]),
    "bfq_forward_quant_stats": (_i, [_p, _p, _i, _i64, _i64, _i, _p, _p, _p, _p, _p]),
    "bfq_inverse": (_i, [_p, _p, _i, _i64, _i64, _p, _i, _i64, _p]),
    "bfq_hadamard": (_i, [_p, _p, _i, _i64, _i64, _p, _i, _i64, _p]),
    "bfq_hadamard_quant": (_i, [_p, _p, _i, _i64, _i64, _i, _p, _p, _p]),
    "bfq_backward": (_i, [_p, _p, _i, _p, _i, _i64, _i64, _p, _i, _p, _p]),
    "bfq_fold_weights": (_i, [_p, _p, _i, _i64, _i64, _i, _p, _p, _p, _i, _p]),
    "bfq_composite_backward": (_i, [_p, _p, _i, _p, _i, _p, _i, _i64, _i64, _p, _p, _p, _p]),
    "bfq_cayley_backward": (_i, [_p, _p, _i, _p, _p, _p, _p]),
    "bfq_device_status": (_i, [_p]),
    "bfq_last_cuda_error": (_i, [_p]),
    "bfq_status_string": (ctypes.c_char_p, [_i]),
    "bfq_backward_partials": (_i, [_p]),
    "bfq_forward_quant_host": (_i, [_p, _p, _i, _i64, _i64, _i, _p, _p, _p, ctypes.c_size_t, _p]),
    "bfq_forward_quant_host_workspace": (ctypes.c_size_t, [_p, _i, _i, _i64]),
    "bfq_measure_fma_rates": (_i, [_p]),
    "bfq_measure_mma_rates": (_i, [_p]),
    "bfq_dequant_gemm": (_i, [_p, _i64, _i64, _i64, ctypes.c_float, _p, _i, _i, _i64, _p, _p, _i, _i, _i64, _p, _p, _i64, _p]),
    "bfq_dequant_gemm_workspace": (ctypes.c_size_t, [_p, _i64, _i64, _i64, _i, _i, _i, _i]),
    "bfq_dequant_gemm_split": (_i, [_p, _i64, _i64, _i64, ctypes.c_float, _p, _i, _i, _i64, _p, _p, _i, _i, _i64, _p, _p, _i64, _p,
                                    ctypes.c_size_t, _p]),
    "bfq_stage_form": (_i, [_p]),
    "bfq_test_stuck_wait": (_i, [_p, _i]),
    "bfq_backward_noalloc": (_i, [_i, _p, _p, _i, _p, _i, _i64, _i64, _p, _i, _p, _p]),
    "bfq_cayley": (_i, [_p, _p, _i, _p, _p]),
    "bfq_composite_forward": (_i, [_p, _p, _i, _p, _i, _i64, _i64, _p, _i, _i64, _p]),
    "bfq_composite_forward_quant": (_i, [_p, _p, _i, _p, _i, _i64, _i64, _i, _p, _p, _p]),
    "bfq_composite_inverse": (_i, [_p, _p, _i, _p, _i, _i64, _i64, _p, _i, _i64, _p]),
    "bfq_kv_append": (_i, [_p, _p, _p, _i64, _i, _p, _p, _p, _p, _p, _p]),
    "bfq_kv_read": (_i, [_p, _p, _p, _i64, _i, _p, _p, _p]),
    "bfq_kv_attend_workspace": (ctypes.c_size_t, [_p, _p, _p]),
    "bfq_kv_attend": (_i, [_p, _p, _p, _p, ctypes.c_size_t, _p]),
}


class _CKVCache(ctypes.Structure):
    _fields_ = [("k_codes", _p), ("k_scales", _p), ("v_codes", _p), ("v_scales", _p), ("k_codes_page", _i64), ("k_scales_page", _i64),
                ("v_codes_page", _i64), ("v_scales_page", _i64), ("pages", _i64), ("heads", _i), ("page_size", _i), ("bits", _i)]


class _CHeads(ctypes.Structure):
    _fields_ = [("data", _p), ("token", _i64), ("head", _i64), ("heads", _i)]


class _CPositions(ctypes.Structure):
    _fields_ = [("positions", _p), ("table", _p), ("rows", _i64), ("dims", _i), ("interleaved", _i), ("q_norm", _p), ("k_norm", _p), ("eps", ctypes.c_float)]


class _CQueries(ctypes.Structure):
    _fields_ = [("q", _CHeads), ("out", _CHeads), ("lse", _p), ("tokens", _i64), ("batch", _i), ("block_table", _p), ("table_ld", _i64), ("table_width", _i),
                ("lengths", _p), ("q_starts", _p), ("max_new", _i), ("prefix", _p), ("prefix_pages", _i), ("prefix_length", _i64), ("scale", ctypes.c_float)]

_lib = None


def _not_native(*args):
    return None


class _Interpreted:
    """In the place of fast_calls: every call is done by the methods below."""
    forward = forward_quant = inverse = append_kv = read_kv = attend_kv = staticmethod(_not_native)


_fast = _Interpreted  # set by lib()


def _native_calls():
    """fast_calls, the plain forms of the smallest calls in C++ (a result, a status, or None for "not plain, done below"), attached to
    the library; or, where it is not built or built against another torch, what answers None to everything."""
    try:
        from . import fast_calls
    except ImportError:
        return _Interpreted
    if getattr(fast_calls, "torch_version", None) != torch.__version__:  # its calls into torch could do anything
        return _Interpreted
    fast_calls.attach(LIB_PATH)
    return fast_calls


class BfqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().bfq_status_string(status).decode()
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({msg})")


def lib() -> ctypes.CDLL:
    """Loads libbfq.so (raises if it has not been built: there is no fallback)."""
    global _lib, _fast
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: run `python -m paper_2509_09679_b200.build` "
                               "(the CUDA library is the only implementation)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _fast = _native_calls()
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != BFQ_OK:
        raise BfqError(status, where)


_DTYPES = {torch.float32: BFQ_F32, torch.bfloat16: BFQ_BF16}


def _dt(t: torch.Tensor) -> int:
    kind = _DTYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return kind


# A call of a few microseconds on the GPU is bound by what happens here, so each property of a tensor is asked for once,
# buffers allocated here are not checked again, and the stream is read as the raw handle (the Stream object that
# torch.cuda.current_stream builds takes longer than the rest of a call).
def _rows(t: torch.Tensor, n: int, device=None, rows=None, what: str = "rows"):
    """Checks a [rows][n] row tensor (unit inner stride; on `device` when given; `rows` rows when given) and returns
    (rows, leading dimension).  Only this layer knows the buffers' sizes: the C ABI takes bare pointers."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what}: expected a [rows][{n}] tensor with unit inner stride, got {type(t)}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[1] != n or stride[1] != 1:
        raise ValueError(f"{what}: expected a [rows][{n}] tensor with unit inner stride, got {tuple(shape)}")
    if device is not None:
        _on(t, device, what)
    count, ld = shape[0], stride[0]
    if rows is not None and count != rows:
        raise ValueError(f"{what}: expected {rows} rows, got {count}")
    if ld < n:
        if count > 1:
            raise ValueError(f"{what}: rows overlap (row stride {ld} < {n})")
        ld = n
    return count, ld


def _on(t: torch.Tensor, device, what: str):
    if t.get_device() != device.index or not t.is_cuda:
        raise ValueError(f"{what}: tensor is on {t.device}, the plan works on {device}")


def _exact(t: torch.Tensor, dtype, shape, device, what: str):
    """A contiguous tensor of exactly this dtype and shape on `device` (tables, codes, scales, statistics)."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        got = (t.dtype, tuple(t.shape)) if isinstance(t, torch.Tensor) else type(t)
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {tuple(shape)}, got {got}")
    _on(t, device, what)
    return t


def _stream(t: torch.Tensor):
    return torch._C._cuda_getCurrentRawStream(t.get_device())


class GemmOperand:
    """One operand of Plan.dequant_gemm: rows of fp32 / bf16 numbers, or packed codes with the fp16 scales of their
    stored rows; `transposed` = stored [K][rows] instead of [rows][K]."""

    def __init__(self, data: torch.Tensor, scales: torch.Tensor | None = None, bits: int = 0, transposed: bool = False):
        shape, stride = data.shape, data.stride()
        if len(shape) != 2 or stride[1] != 1:
            raise ValueError("operand: expected a 2-D tensor with unit inner stride")
        self.data, self.scales, self.transposed = data, scales, bool(transposed)
        if scales is None:
            self.kind, per = _dt(data), 1
        else:
            if bits not in (2, 4, 8) or data.dtype != torch.uint8:
                raise ValueError("operand: codes are uint8 with bits in {2, 4, 8}")
            self.kind, per = bits, 8 // bits
            _exact(scales, torch.float16, (shape[0],), data.device, "operand scales")
        stored_rows, width = shape[0], shape[1] * per
        self.rows, self.k = (width, stored_rows) if transposed else (stored_rows, width)
        self.ld = (stride[0] if stored_rows > 1 else shape[1]) * per


class Plan:
    """Owns a bfq_plan for row length n on one CUDA device."""

    _id, _index = 0, -1  # of the plan and its device, for fast_calls

    def __init__(self, n: int, device=None, max_rows: int = 0):
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        if dev.type != "cuda":
            raise ValueError("bfq runs on CUDA devices only")
        self.n = int(n)
        self.L = self.n.bit_length() - 1
        self.device = torch.device("cuda", dev.index if dev.index is not None else torch.cuda.current_device())
        self._h = ctypes.c_void_p()
        self._c = lib()
        _check(lib().bfq_plan_create(ctypes.byref(self._h), self.n, int(max_rows), self.device.index),
               "bfq_plan_create")
        self._id, self._index = self._h.value, self.device.index

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._id = 0
            lib().bfq_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C ABI, one method per entry point ------------------------------------------------------
    def set_angles(self, theta: torch.Tensor):
        _exact(theta, torch.float32, (self.L, self.n // 2), self.device, "theta")
        _check(self._c.bfq_set_angles(self._h, theta.data_ptr(), _stream(theta)), "bfq_set_angles")

    def forward(self, x: torch.Tensor, out_dtype=None, out: torch.Tensor | None = None) -> torch.Tensor:
        if out is None and out_dtype is None:
            done = _fast.forward(self._id, self.n, self._index, x)
            if done is not None:
                return done if type(done) is not int else _check(done, "bfq_forward")
        n = self.n
        rows, ldx = _rows(x, n, self.device, what="x")
        y, ldy = self._row_output(x, rows, out_dtype, out)
        _check(self._c.bfq_forward(self._h, x.data_ptr(), _dt(x), rows, ldx, y.data_ptr(), _dt(y), ldy, _stream(x)), "bfq_forward")
        return y

    def _row_output(self, x: torch.Tensor, rows: int, out_dtype, out):
        """The caller's [rows][n] buffer, checked, or a new one; and its leading dimension."""
        n = self.n
        if out is not None:
            return out, _rows(out, n, self.device, rows, "out")[1]
        return torch.empty((rows, n), dtype=out_dtype or x.dtype, device=self.device), n

    def _outputs(self, rows: int, width: int, bits: int, codes, scales):
        """Allocates or checks the codes uint8 [rows][width * bits / 8] and scales fp16 [rows] buffers (the bit width
        itself is the C side's to reject, before any launch)."""
        shape = (rows, width * int(bits) // 8)
        if codes is None:
            codes = torch.empty(shape, dtype=torch.uint8, device=self.device)
        else:
            _exact(codes, torch.uint8, shape, self.device, "codes")
        if scales is None:
            scales = torch.empty(rows, dtype=torch.float16, device=self.device)
        else:
            _exact(scales, torch.float16, (rows,), self.device, "scales")
        return codes, scales

    def forward_quant(self, x: torch.Tensor, bits: int, codes=None, scales=None):
        if codes is None and scales is None:
            done = _fast.forward_quant(self._id, self.n, self._index, x, bits)
            if done is not None:
                return done if type(done) is not int else _check(done, "bfq_forward_quant")
        rows, ldx = _rows(x, self.n, self.device, what="x")
        codes, scales = self._outputs(rows, self.n, bits, codes, scales)
        _check(self._c.bfq_forward_quant(self._h, x.data_ptr(), _dt(x), rows, ldx, int(bits), codes.data_ptr(),
                                       scales.data_ptr(), _stream(x)), "bfq_forward_quant")
        return codes, scales

    # -- composite transform Q1 (x) Q2 for d = n1 * n (paper Sec. 3.3); this plan's butterfly is Q2 --------------
    def cayley(self, params: torch.Tensor, n1: int) -> torch.Tensor:
        """Q1 = (I - A)(I + A)^-1 from the n1 (n1 - 1) / 2 upper-triangle entries of the skew A -> fp32 [n1][n1]."""
        if params.dtype != torch.float32 or params.numel() != n1 * (n1 - 1) // 2 or not params.is_contiguous():
            raise ValueError("params must be a contiguous fp32 tensor of n1 (n1 - 1) / 2 entries")
        _on(params, self.device, "params")
        q1 = torch.empty((n1, n1), dtype=torch.float32, device=params.device)
        _check(self._c.bfq_cayley(self._h, params.data_ptr(), int(n1), q1.data_ptr(), _stream(params)), "bfq_cayley")
        return q1

    def _q1(self, q1: torch.Tensor) -> int:
        if q1.dtype != torch.float32 or q1.dim() != 2 or q1.shape[0] != q1.shape[1] or not q1.is_contiguous():
            raise ValueError("q1 must be a contiguous fp32 [n1][n1] tensor")
        _on(q1, self.device, "q1")
        return q1.shape[0]

    def composite_forward(self, q1: torch.Tensor, x: torch.Tensor, out_dtype=None, out=None) -> torch.Tensor:
        n1 = self._q1(q1)
        d = n1 * self.n
        rows, ldx = _rows(x, d, self.device, what="x")
        y = out if out is not None else torch.empty((rows, d), dtype=out_dtype or x.dtype, device=x.device)
        if _rows(y, d, self.device, rows, "out")[1] != d:
            raise ValueError("out: rows must be contiguous")
        _check(self._c.bfq_composite_forward(self._h, q1.data_ptr(), n1, x.data_ptr(), _dt(x), rows, ldx, y.data_ptr(),
                                           _dt(y), d, _stream(x)), "bfq_composite_forward")
        return y

    def composite_inverse(self, q1: torch.Tensor, y: torch.Tensor, out_dtype=None, out=None) -> torch.Tensor:
        n1 = self._q1(q1)
        d = n1 * self.n
        rows, ldy = _rows(y, d, self.device, what="y")
        x = out if out is not None else torch.empty((rows, d), dtype=out_dtype or y.dtype, device=y.device)
        if _rows(x, d, self.device, rows, "out")[1] != d:
            raise ValueError("out: rows must be contiguous")
        _check(self._c.bfq_composite_inverse(self._h, q1.data_ptr(), n1, y.data_ptr(), _dt(y), rows, ldy, x.data_ptr(),
                                           _dt(x), d, _stream(y)), "bfq_composite_inverse")
        return x

    def composite_forward_quant(self, q1: torch.Tensor, x: torch.Tensor, bits: int, codes=None, scales=None):
        n1 = self._q1(q1)
        d = n1 * self.n
        rows, ldx = _rows(x, d, self.device, what="x")
        codes, scales = self._outputs(rows, d, bits, codes, scales)
        _check(self._c.bfq_composite_forward_quant(self._h, q1.data_ptr(), n1, x.data_ptr(), _dt(x), rows, ldx, int(bits),
                                                 codes.data_ptr(), scales.data_ptr(), _stream(x)),
               "bfq_composite_forward_quant")
        return codes, scales

    def composite_backward(self, q1: torch.Tensor, x: torch.Tensor, g: torch.Tensor):
        """x, g: [tokens][n1 * n] contiguous.  Returns (dx in the type of x, dtheta of Q2, dQ1)."""
        n1 = self._q1(q1)
        d = n1 * self.n
        rows, ld = _rows(x, d, self.device, what="x")
        ld_g = _rows(g, d, self.device, rows, "g")[1]
        if rows > 1 and (ld != d or ld_g != d):  # a single row may come with any row stride
            raise ValueError("x and g must have contiguous rows")
        dx = torch.empty((rows, d), dtype=x.dtype, device=x.device)
        dtheta = torch.empty((self.L, self.n // 2), dtype=torch.float32, device=x.device)
        dq1 = torch.empty((n1, n1), dtype=torch.float32, device=x.device)
        _check(self._c.bfq_composite_backward(self._h, q1.data_ptr(), n1, x.data_ptr(), _dt(x), g.data_ptr(), _dt(g), rows, d, dx.data_ptr(),
                                            dtheta.data_ptr(), dq1.data_ptr(), _stream(x)), "bfq_composite_backward")
        return dx, dtheta, dq1

    def cayley_backward(self, params: torch.Tensor, q1: torch.Tensor, dq1: torch.Tensor) -> torch.Tensor:
        """dL/dparams of q1 = cayley(params) from dL/dQ1 (fp32, on the plan's device)."""
        n1 = self._q1(q1)
        _exact(params, torch.float32, (n1 * (n1 - 1) // 2,), self.device, "params")
        _exact(dq1, torch.float32, (n1, n1), self.device, "dq1")
        dparams = torch.empty_like(params)
        _check(self._c.bfq_cayley_backward(self._h, params.data_ptr(), n1, q1.data_ptr(), dq1.data_ptr(), dparams.data_ptr(), _stream(params)),
               "bfq_cayley_backward")
        return dparams

    def forward_quant_stats(self, x: torch.Tensor, bits: int):
        """-> (codes, scales, hist int64 [2^bits], rowstats fp32 [rows][2] = (sum y^2, sum y^4))."""
        rows, ldx = _rows(x, self.n, self.device, what="x")
        codes, scales = self._outputs(rows, self.n, bits, None, None)
        hist = torch.empty((1 << bits,), dtype=torch.int64, device=x.device)
        rowstats = torch.empty((rows, 2), dtype=torch.float32, device=x.device)
        _check(self._c.bfq_forward_quant_stats(self._h, x.data_ptr(), _dt(x), rows, ldx, int(bits), codes.data_ptr(),
                                             scales.data_ptr(), hist.data_ptr(), rowstats.data_ptr(), _stream(x)),
               "bfq_forward_quant_stats")
        return codes, scales, hist, rowstats

    def hadamard(self, x: torch.Tensor, out_dtype=None, out: torch.Tensor | None = None) -> torch.Tensor:
        rows, ldx = _rows(x, self.n, self.device, what="x")
        y, ldy = self._row_output(x, rows, out_dtype, out)
        _check(self._c.bfq_hadamard(self._h, x.data_ptr(), _dt(x), rows, ldx, y.data_ptr(), _dt(y), ldy, _stream(x)),
               "bfq_hadamard")
        return y

    def hadamard_quant(self, x: torch.Tensor, bits: int, codes=None, scales=None):
        rows, ldx = _rows(x, self.n, self.device, what="x")
        codes, scales = self._outputs(rows, self.n, bits, codes, scales)
        _check(self._c.bfq_hadamard_quant(self._h, x.data_ptr(), _dt(x), rows, ldx, int(bits), codes.data_ptr(),
                                        scales.data_ptr(), _stream(x)), "bfq_hadamard_quant")
        return codes, scales

    def inverse(self, y: torch.Tensor, out_dtype=None, out: torch.Tensor | None = None) -> torch.Tensor:
        if out is None and out_dtype is None:
            done = _fast.inverse(self._id, self.n, self._index, y)
            if done is not None:
                return done if type(done) is not int else _check(done, "bfq_inverse")
        rows, ldy = _rows(y, self.n, self.device, what="y")
        x, ldx = self._row_output(y, rows, out_dtype, out)
        _check(self._c.bfq_inverse(self._h, y.data_ptr(), _dt(y), rows, ldy, x.data_ptr(), _dt(x), ldx, _stream(y)),
               "bfq_inverse")
        return x

    def backward(self, x: torch.Tensor, g: torch.Tensor, dx_dtype=None, want_dx: bool = True, dx=None, dtheta=None):
        rows, ld = _rows(x, self.n, self.device, what="x")
        rows_g, ld_g = _rows(g, self.n, self.device, what="g")
        if rows_g != rows or ld_g != ld:
            raise ValueError("x and g must have the same shape and row stride")
        if want_dx and dx is None:
            dx = torch.empty_strided((rows, self.n), (ld, 1), dtype=dx_dtype or x.dtype, device=self.device)
        elif want_dx and _rows(dx, self.n, self.device, rows, "dx")[1] != ld:
            raise ValueError("dx must have the row stride of x")
        if dtheta is None:
            dtheta = torch.empty((self.L, self.n // 2), dtype=torch.float32, device=self.device)
        else:
            _exact(dtheta, torch.float32, (self.L, self.n // 2), self.device, "dtheta")
        _check(self._c.bfq_backward(self._h, x.data_ptr(), _dt(x), g.data_ptr(), _dt(g), rows, ld,
                                  dx.data_ptr() if want_dx else None, _dt(dx) if want_dx else BFQ_F32,
                                  dtheta.data_ptr(), _stream(x)), "bfq_backward")
        return (dx if want_dx else None), dtheta

    def forward_quant_host_workspace(self, dtype, bits: int, chunk_rows: int) -> int:
        """Bytes of device workspace for forward_quant_host in chunks of chunk_rows rows."""
        xt = BFQ_F32 if dtype == torch.float32 else BFQ_BF16
        return int(self._c.bfq_forward_quant_host_workspace(self._h, xt, int(bits), int(chunk_rows)))

    def forward_quant_host(self, x_host: torch.Tensor, bits: int, codes_host: torch.Tensor, scales_host: torch.Tensor,
                           workspace: torch.Tensor):
        """bfq_forward_quant_host: rows, codes and scales in (pinned) host memory, a uint8 device workspace; enqueued on
        the current stream of the plan's device."""
        if x_host.is_cuda or codes_host.is_cuda or scales_host.is_cuda:
            raise ValueError("x_host, codes_host and scales_host must be host tensors")
        if x_host.dim() != 2 or x_host.shape[1] != self.n or x_host.stride(1) != 1:
            raise ValueError(f"x_host must be [rows][{self.n}] with unit inner stride")
        if x_host.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("x_host must be float32 or bfloat16")
        rows = x_host.shape[0]
        for t, dtype, shape, what in ((codes_host, torch.uint8, (rows, self.n * int(bits) // 8), "codes_host"),
                                      (scales_host, torch.float16, (rows,), "scales_host")):
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
                raise ValueError(f"{what}: expected a contiguous {dtype} host tensor of shape {shape}")
        if not workspace.is_cuda or workspace.device != self.device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on the plan's device")
        with torch.cuda.device(self.device):
            stream = torch.cuda.current_stream(self.device).cuda_stream
            _check(self._c.bfq_forward_quant_host(self._h, x_host.data_ptr(), _dt(x_host), rows, x_host.stride(0), int(bits),
                                                codes_host.data_ptr(), scales_host.data_ptr(), workspace.data_ptr(),
                                                workspace.numel(), stream), "bfq_forward_quant_host")

    def fold_weights(self, W: torch.Tensor, bits: int, want_rotated: bool = False, rotated_dtype=None):
        m, ldw = _rows(W, self.n, self.device, what="W")
        codes, scales = self._outputs(m, self.n, bits, None, None)
        rot = torch.empty((m, self.n), dtype=rotated_dtype or W.dtype, device=W.device) if want_rotated else None
        _check(self._c.bfq_fold_weights(self._h, W.data_ptr(), _dt(W), m, ldw, int(bits), codes.data_ptr(),
                                      scales.data_ptr(), rot.data_ptr() if rot is not None else None,
                                      _dt(rot) if rot is not None else BFQ_F32, _stream(W)), "bfq_fold_weights")
        return codes, scales, rot

    def dequant_gemm(self, a: GemmOperand, b: GemmOperand, alpha: float = 1.0, out: torch.Tensor | None = None):
        """C[i][j] = alpha * sum_k A(i, k) B(j, k) on the tensor cores, low-bit operands dequantized on the fly -> fp32."""
        if a.k != b.k:
            raise ValueError(f"operands disagree on K: {a.k} and {b.k}")
        for op, what in ((a, "A"), (b, "B")):
            _on(op.data, self.device, what)
        if out is None:
            c = torch.empty((a.rows, b.rows), dtype=torch.float32, device=self.device)
        else:
            c = _exact(out, torch.float32, (a.rows, b.rows), self.device, "out")
        args = (self._h, a.rows, b.rows, a.k, float(alpha), a.data.data_ptr(), a.kind, int(a.transposed), a.ld,
                a.scales.data_ptr() if a.scales is not None else None, b.data.data_ptr(), b.kind, int(b.transposed), b.ld,
                b.scales.data_ptr() if b.scales is not None else None, c.data_ptr(), b.rows)
        if a.kind == BFQ_F32 or b.kind == BFQ_F32:  # room to split fp32 operands in, where that helps
            size = self._c.bfq_dequant_gemm_workspace(self._h, a.rows, b.rows, a.k, a.kind, int(a.transposed), b.kind, int(b.transposed))
            try:
                room = torch.empty(size + 256, dtype=torch.uint8, device=self.device) if size else None
            except torch.OutOfMemoryError:
                room = None  # the product does not need it
            if room is not None:
                _check(self._c.bfq_dequant_gemm_split(*args, (room.data_ptr() + 255) // 256 * 256, size, _stream(c)), "bfq_dequant_gemm_split")
                return c
        _check(self._c.bfq_dequant_gemm(*args, _stream(c)), "bfq_dequant_gemm")
        return c

    # -- paged low-bit cache of keys and values (kv_cache.py); this plan's n is the head dimension -------------------
    def _cache(self, cache: KVCache):
        if not isinstance(cache, KVCache) or cache.head_dim != self.n or cache.device != self.device:
            got = (cache.head_dim, str(cache.device)) if isinstance(cache, KVCache) else type(cache)
            raise ValueError(f"cache: expected a KVCache of heads of {self.n} elements on {self.device}, got {got}")
        pages = [t.stride(0) if cache.pages > 1 else t.shape[1:].numel() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
        return ctypes.byref(_CKVCache(cache.k_codes.data_ptr(), cache.k_scales.data_ptr(), cache.v_codes.data_ptr(), cache.v_scales.data_ptr(), *pages,
                                      cache.pages, cache.heads, cache.page_size, cache.bits))

    def _head_rows(self, t, tokens, heads, dtype, what: str):
        """Checks rows [tokens][heads][n] (unit inner stride, on the plan's device; tokens, heads, dtype where given) and describes them."""
        if not isinstance(t, torch.Tensor) or t.dim() != 3 or t.shape[2] != self.n or t.stride(2) != 1:
            raise ValueError(f"{what}: expected [tokens][heads][{self.n}] with unit inner stride, got {tuple(t.shape) if isinstance(t, torch.Tensor) else type(t)}")
        _on(t, self.device, what)
        shape, stride = t.shape, t.stride()
        if (tokens is not None and shape[0] != tokens) or (heads is not None and shape[1] != heads) or shape[1] < 1:
            raise ValueError(f"{what}: expected [{tokens}][{heads}][{self.n}], got {tuple(shape)}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
        head = stride[1] if shape[1] > 1 else self.n
        return _CHeads(t.data_ptr(), stride[0] if shape[0] > 1 else shape[1] * self.n, head, shape[1])

    def _apart(self, t, what: str):
        """Rows that are written: no two of them may share memory."""
        shape, stride = t.shape, t.stride()
        (few, near), (many, far) = sorted(zip(shape[:2], stride[:2]), key=lambda d: d[1])
        if t.numel() and ((few > 1 and near < self.n) or (many > 1 and far < (few - 1) * near + self.n)):
            raise ValueError(f"{what}: rows overlap (strides {stride})")

    def append_kv(self, cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, q: torch.Tensor | None = None,
                  positions: torch.Tensor | None = None, rope: torch.Tensor | None = None, interleaved: bool = False,
                  q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, eps: float = 1e-6, q_out: torch.Tensor | None = None):
        """A step's new tokens into the cache: k, v [tokens][heads][n] (bf16 or fp32), quantized at slots int64 [tokens] (negative: nowhere); before
        that queries and keys are normed per head (q_norm, k_norm fp32 [n]) and rotated by position (positions int32 [tokens], rope fp32
        [rows][dims]: cosines of dims / 2 frequencies, then sines; pairs (i, i + dims / 2), or (2 i, 2 i + 1) if interleaved), and all are rotated
        by Q.  Returns the queries as attend_kv takes them, bf16 (q_out, or a new tensor), or None without q."""
        if q_out is None and type(cache) is KVCache:
            done = _fast.append_kv(self._id, self.n, self._index, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales, cache.bits, k, v, slots, q,
                                   positions, rope, interleaved, q_norm, k_norm, eps)
            if done is not None:
                return None if done is True else (done if type(done) is not int else _check(done, "bfq_kv_append"))
        c = self._cache(cache)
        ck = self._head_rows(k, None, cache.heads, None, "k")
        tokens, xt = k.shape[0], _dt(k)
        cv = self._head_rows(v, tokens, cache.heads, k.dtype, "v")
        _exact(slots, torch.int64, (tokens,), self.device, "slots")
        cq = co = None
        if q is not None:
            cq = self._head_rows(q, tokens, None, k.dtype, "q")
            given = q_out is not None
            if not given:
                q_out = torch.empty((tokens, q.shape[1], self.n), dtype=torch.bfloat16, device=self.device)
            co = self._head_rows(q_out, tokens, q.shape[1], torch.bfloat16, "q_out")
            if given:
                self._apart(q_out, "q_out")
        elif q_out is not None or q_norm is not None:
            raise ValueError("q_out and q_norm are for calls with q")
        if (positions is None) != (rope is None):
            raise ValueError("positions and rope come together")
        at = _CPositions()
        if positions is not None:
            _exact(positions, torch.int32, (tokens,), self.device, "positions")
            if rope.dim() != 2 or not 16 <= rope.shape[1] <= self.n or rope.shape[1] % 16 or not rope.shape[0]:
                raise ValueError(f"rope: expected [positions][dims], dims a multiple of 16 up to {self.n}, got {tuple(rope.shape)}")
            _exact(rope, torch.float32, rope.shape, self.device, "rope")
            at.positions, at.table, at.rows, at.dims, at.interleaved = positions.data_ptr(), rope.data_ptr(), rope.shape[0], rope.shape[1], bool(interleaved)
        if q_norm is not None:
            at.q_norm = _exact(q_norm, torch.float32, (self.n,), self.device, "q_norm").data_ptr()
        if k_norm is not None:
            at.k_norm = _exact(k_norm, torch.float32, (self.n,), self.device, "k_norm").data_ptr()
        at.eps = eps
        ref = ctypes.byref
        _check(self._c.bfq_kv_append(self._h, c, slots.data_ptr(), tokens, xt, ref(ck), ref(cv), ref(cq) if cq is not None else None,
                                     ref(co) if co is not None else None, ref(at), _stream(k)), "bfq_kv_append")
        return q_out

    def read_kv(self, cache: KVCache, slots: torch.Tensor, dtype=torch.bfloat16):
        """-> (k, v) [tokens][heads][n] of `dtype` (bf16 or fp32): the rows at slots int64 [tokens], dequantized and in the model's basis;
        zeros for a negative slot."""
        if dtype is torch.bfloat16 and type(cache) is KVCache:
            done = _fast.read_kv(self._id, self.n, self._index, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales, cache.bits, slots)
            if done is not None:
                return done if type(done) is not int else _check(done, "bfq_kv_read")
        c = self._cache(cache)
        kind = _DTYPES.get(dtype)
        if kind is None:
            raise TypeError(f"unsupported dtype {dtype}")
        if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
            raise ValueError("slots: expected int64 [tokens]")
        tokens = slots.shape[0]
        _exact(slots, torch.int64, (tokens,), self.device, "slots")
        k, v = torch.empty((2, tokens, cache.heads, self.n), dtype=dtype, device=self.device).unbind(0)
        _check(self._c.bfq_kv_read(self._h, c, slots.data_ptr(), tokens, kind, k.data_ptr(), v.data_ptr(), _stream(slots)), "bfq_kv_read")
        return k, v

    def attend_kv(self, cache: KVCache, q: torch.Tensor, block_table: torch.Tensor, lengths: torch.Tensor, scale: float | None = None,
                  q_starts: torch.Tensor | None = None, max_new: int | None = None, prefix: torch.Tensor | None = None, prefix_length: int = 0,
                  want_lse: bool = False, out: torch.Tensor | None = None):
        """Attention of q, bf16 [tokens][heads][n] as append_kv gives it, over the cached keys and values of each sequence; out in the model's
        basis, bf16.  block_table int32 [batch][width]: a sequence's pages; lengths int32 [batch]: its cached keys, this call's tokens
        included.  q_starts int32 [batch + 1] with max_new, the most tokens that a sequence has in q: each sees the keys up to its own;
        without them token b is sequence b's only one.  prefix int32 [pages], prefix_length: keys in front of every sequence, read once for
        all.  scale: 1 / sqrt(n) by default.  want_lse: (out, fp32 [tokens][heads] log sum exp of the scaled scores).  Rows of tokens behind
        the last sequence are not written."""
        if out is None and not want_lse and type(cache) is KVCache:
            done = _fast.attend_kv(self._id, self.n, self._index, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales, cache.bits, q, block_table,
                                   lengths, scale, q_starts, max_new, prefix, prefix_length)
            if done is not None:
                return done if type(done) is not int else _check(done, "bfq_kv_attend")
        c = self._cache(cache)
        cq = self._head_rows(q, None, None, torch.bfloat16, "q")
        tokens, heads = q.shape[0], q.shape[1]
        if heads % cache.heads or heads // cache.heads > 128:
            raise ValueError(f"q: {heads} heads are not 1 to 128 for each of the cache's {cache.heads}")
        if not isinstance(lengths, torch.Tensor) or lengths.dim() != 1:
            raise ValueError("lengths: expected int32 [batch]")
        batch = lengths.shape[0]
        _exact(lengths, torch.int32, (batch,), self.device, "lengths")
        if not isinstance(block_table, torch.Tensor) or block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != batch or \
                (block_table.shape[1] > 1 and block_table.stride(1) != 1) or (batch > 1 and block_table.stride(0) < block_table.shape[1]):
            raise ValueError(f"block_table: expected int32 [{batch}][pages] with unit inner stride")
        _on(block_table, self.device, "block_table")
        if q_starts is not None:
            _exact(q_starts, torch.int32, (batch + 1,), self.device, "q_starts")
            if max_new is None or (tokens and not 1 <= max_new):
                raise ValueError("q_starts: max_new, the most tokens of a sequence, is needed and at least 1")
            max_new = min(int(max_new), max(tokens, 1))
        elif tokens < batch:
            raise ValueError(f"q: expected a token for each of {batch} sequences, got {tokens}")
        if prefix is None:
            if prefix_length:
                raise ValueError("prefix_length without prefix")
        else:
            if not isinstance(prefix, torch.Tensor) or prefix.dim() != 1:
                raise ValueError("prefix: expected int32 [pages]")
            _exact(prefix, torch.int32, (prefix.shape[0],), self.device, "prefix")
            if not 0 <= prefix_length <= prefix.shape[0] * cache.page_size:
                raise ValueError(f"prefix_length: {prefix_length} keys are not in {prefix.shape[0]} pages of {cache.page_size}")
        given = out is not None
        if not given:
            out = torch.empty((tokens, heads, self.n), dtype=torch.bfloat16, device=self.device)
        co = self._head_rows(out, tokens, heads, torch.bfloat16, "out")
        if given:
            self._apart(out, "out")
        lse = torch.empty((tokens, heads), dtype=torch.float32, device=self.device) if want_lse else None
        if tokens and batch:
            a = _CQueries(cq, co, lse.data_ptr() if want_lse else None, tokens, batch, block_table.data_ptr(),
                          block_table.stride(0) if batch > 1 else block_table.shape[1], block_table.shape[1], lengths.data_ptr(),
                          q_starts.data_ptr() if q_starts is not None else None, max_new or 1, prefix.data_ptr() if prefix is not None else None,
                          prefix.shape[0] if prefix is not None else 0, int(prefix_length), float(scale) if scale is not None else self.n ** -0.5)
            a = ctypes.byref(a)
            size = self._c.bfq_kv_attend_workspace(self._h, c, a)
            room = torch.empty(size + 256, dtype=torch.uint8, device=self.device)
            _check(self._c.bfq_kv_attend(self._h, c, a, (room.data_ptr() + 255) // 256 * 256, size, _stream(q)), "bfq_kv_attend")
        return (out, lse) if want_lse else out

    def device_status(self) -> int:
        return int(self._c.bfq_device_status(self._h))

    def stage_form(self) -> int:
        """bit 0 / bit 1: the forward / inverse tables of the tuned kernels use the three-shear fallback."""
        r = int(self._c.bfq_stage_form(self._h))
        if r < 0:
            raise BfqError(r, "bfq_stage_form")
        return r

    def test_stuck_wait(self, enable: bool):
        _check(self._c.bfq_test_stuck_wait(self._h, int(bool(enable))), "bfq_test_stuck_wait")

    def backward_partials(self) -> int:
        return int(self._c.bfq_backward_partials(self._h))


def backward_noalloc(theta: torch.Tensor, x: torch.Tensor, g: torch.Tensor, dx: torch.Tensor | None,
                     dtheta: torch.Tensor):
    """bfq_backward_noalloc: the backward pass without a plan and without any device allocation by the
    library (for hosts that must not call cudaMalloc; row length at most 1024).  Every buffer,
    outputs included, is the caller's; pass dx=None to skip dL/dx.  Runs on x's device, which is
    made current for the call.  Calls share one fixed scratch array per GPU: do not overlap them."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not x.is_cuda:
        raise ValueError("x must be a [rows][n] CUDA tensor")
    n = x.shape[1]
    L = n.bit_length() - 1
    if n < 16 or (1 << L) != n:
        raise ValueError("n must be a power of two >= 16")
    rows, ld = _rows(x, n, x.device, what="x")
    rows_g, ld_g = _rows(g, n, x.device, what="g")
    if rows_g != rows or ld_g != ld:
        raise ValueError("x and g must have the same shape and row stride")
    if dx is not None and _rows(dx, n, x.device, rows, "dx") != (rows, ld):
        raise ValueError("dx must have the shape and row stride of x")
    _exact(theta, torch.float32, (L, n // 2), x.device, "theta")
    _exact(dtheta, torch.float32, (L, n // 2), x.device, "dtheta")
    with torch.cuda.device(x.device):
        _check(lib().bfq_backward_noalloc(n, theta.data_ptr(), x.data_ptr(), _dt(x), g.data_ptr(), _dt(g), rows, ld,
                                          dx.data_ptr() if dx is not None else None,
                                          _dt(dx) if dx is not None else BFQ_F32, dtheta.data_ptr(), _stream(x)),
               "bfq_backward_noalloc")
    return dx, dtheta


def measure_fma_rates(device=None):
    """bfq_measure_fma_rates on `device` (default: the current one): SM cycles per FMA instruction per scheduler for
    (packed, three register operands), (packed, two), (scalar, three), (scalar, two)."""
    out = (ctypes.c_float * 4)()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(dev):
        _check(lib().bfq_measure_fma_rates(ctypes.cast(out, ctypes.c_void_p)), "bfq_measure_fma_rates")
    return {"packed_3reg": out[0], "packed_2reg": out[1], "scalar_3reg": out[2], "scalar_2reg": out[3]}


def measure_mma_rates(device=None):
    """bfq_measure_mma_rates on `device` (default: the current one): SM cycles per tcgen05.mma (bf16, M = 128, K = 16)
    for N = 16, 64, 128, 256."""
    out = (ctypes.c_float * 4)()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(dev):
        _check(lib().bfq_measure_mma_rates(ctypes.cast(out, ctypes.c_void_p)), "bfq_measure_mma_rates")
    return {"n16": out[0], "n64": out[1], "n128": out[2], "n256": out[3]}
