"""The operators next to the compressed layers in a transformer block: RMS norm with the residual's addition, 8-bit
matrices with a scale for each 128 values and their products, rotary positions (include/compact_block.h).

Argument marshalling only, as in `binding`: every step runs in the library's CUDA kernels, torch gives device memory and
streams, and a refused call raises binding.CompactError with the library's status.  The tensors are checked and handed
over by a small C++ module (csrc/block_py.cpp); if it or the library is missing, loading raises.

    x8 = RMSNorm(n).forward(x, gamma, residual=r, want_fp8=True).q     # what the next product reads
    w8, w8t = quantize_blocks(W)                                       # a layer's weight (n x m) and its transpose, once per update
    product = Fp8Product()                                             # kept: it is asked for its status now and then
    y = product(x8, w8t)                                               # Y = X W
    dx = product(quantize_rows(dy), w8)                                # dX = dY W^T
    q, k = Rotary(128).forward(q, k, positions)
"""
from __future__ import annotations

import ctypes as C
import functools
import math
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as cb
from .binding import BF16, ERR_DTYPE, ERR_INVALID_ARG, ERR_SHAPE, F32, CompactError
from .build import LIB_PATH, MODULE_PATH, module_fits, module_tag

E4M3, E5M2 = 0, 1
ROTARY_NONE, ROTARY_LINEAR, ROTARY_BASE, ROTARY_BY_PARTS = range(4)
RMS_NORM_MAX_N = 16384

EXPORTS = [
    "compact_fp8_scale_groups", "compact_quantize_rows", "compact_quantize_blocks", "compact_rms_norm_fwd",
    "compact_rms_norm_bwd_workspace_bytes", "compact_rms_norm_bwd", "compact_rotary_create", "compact_rotary_destroy",
    "compact_rotary_apply", "compact_fp8_product_create", "compact_fp8_product_destroy", "compact_fp8_product_run",
    "compact_fp8_product_status", "compact_fp8_product_set_kernel", "compact_debug_fp8_product_withhold",
    "compact_debug_fp8_product_plan",
]

_FLOATS = {torch.float32: F32, torch.bfloat16: BF16}
_FP8 = {torch.float8_e4m3fn: E4M3, torch.float8_e5m2: E5M2}
_SCALINGS = {"none": ROTARY_NONE, "linear": ROTARY_LINEAR, "base": ROTARY_BASE, "by_parts": ROTARY_BY_PARTS}


class RotaryConfig(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scaling", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("trained_length", C.c_double), ("attention_factor", C.c_float)]


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    L = cb.lib()
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    L.compact_fp8_scale_groups.argtypes = [i64]
    L.compact_fp8_scale_groups.restype = i64
    L.compact_quantize_rows.argtypes = [C.c_int, i64, i64, vp, i64, C.c_int, vp, i64, vp, i64, vp]
    L.compact_quantize_blocks.argtypes = [C.c_int, i64, i64, vp, i64, C.c_int, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    L.compact_rms_norm_fwd.argtypes = [C.c_int, i64, i32, C.c_float, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, C.c_int, vp, i64, vp, i64, vp]
    L.compact_rms_norm_bwd_workspace_bytes.argtypes = [C.c_int, i64, i32]
    L.compact_rms_norm_bwd_workspace_bytes.restype = C.c_size_t
    L.compact_rms_norm_bwd.argtypes = [C.c_int, i64, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, C.c_int, vp, C.c_size_t, vp]
    L.compact_rotary_create.argtypes = [C.POINTER(RotaryConfig), C.POINTER(vp)]
    L.compact_rotary_destroy.argtypes = [vp]
    L.compact_rotary_apply.argtypes = [vp, C.c_int, i64, i32, i32, vp, i64, i64, vp, i64, i64, vp, C.c_int, i64, C.c_int,
                                       vp, i64, i64, vp, i64, i64, vp]
    L.compact_fp8_product_create.argtypes = [C.POINTER(vp)]
    L.compact_fp8_product_destroy.argtypes = [vp]
    L.compact_fp8_product_run.argtypes = [vp, i64, i64, i64, C.c_int, vp, i64, vp, i64, C.c_int, vp, i64, vp, i64, C.c_int, vp, i64, vp]
    L.compact_fp8_product_status.argtypes = [vp]
    L.compact_fp8_product_set_kernel.argtypes = [C.c_int]
    L.compact_debug_fp8_product_withhold.argtypes = [vp, i32]
    L.compact_debug_fp8_product_plan.argtypes = [i64, i64, i64, C.POINTER(i32)]
    _lib = L
    return L


def _module():
    """The C++ module, on the library that `binding` has loaded."""
    global _mod
    if _mod is None:
        lib()
        if not module_fits():
            raise ImportError(f"{MODULE_PATH} is missing, or built for another Python or torch than {module_tag()}: build.build_module() makes it")
        from . import _block_py

        _block_py.open_library(LIB_PATH, CompactError)
        _mod = _block_py
    return _mod


_mod = None


def _check(code: int, where: str) -> None:
    if code != cb.OK:
        raise CompactError(code, where)


def _on_its_stream(call):
    """A call with `stream` runs with that stream current: what it allocates belongs to the stream that uses it."""

    @functools.wraps(call)
    def wrapped(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)

    return wrapped


def _float_code(dtype: torch.dtype, where: str) -> int:
    code = _FLOATS.get(dtype)
    if code is None:
        raise CompactError(ERR_DTYPE, where)
    return code


def _fp8_code(dtype: torch.dtype, where: str) -> int:
    code = _FP8.get(dtype)
    if code is None:
        raise CompactError(ERR_DTYPE, where)
    return code


# -- 8-bit matrices ---------------------------------------------------------------------------------
class Fp8Matrix(NamedTuple):
    """data (rows, cols) in float8_e4m3fn or float8_e5m2, rows on 16-byte boundaries; scales (ceil(cols / 512), rows, 4) in
    float8_e8m0fnu: scales[g, i, j] belongs to columns 128 (4 g + j) .. + 127 of row i."""

    data: torch.Tensor
    scales: torch.Tensor


def new_fp8(rows: int, cols: int, dtype: torch.dtype = torch.float8_e4m3fn, device="cuda") -> Fp8Matrix:
    """Memory for one.  Rows start on 128-byte boundaries where they are longer than that, which products read fastest; 16 is what
    they need."""
    unit = 128 if cols > 128 else 16
    return Fp8Matrix(torch.empty((rows, (cols + unit - 1) // unit * unit), dtype=dtype, device=device)[:, :cols],
                     torch.empty(((cols + 511) // 512, rows, 4), dtype=torch.float8_e8m0fnu, device=device))


@_on_its_stream
def quantize_rows(x: torch.Tensor, dtype: torch.dtype = torch.float8_e4m3fn, out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
    """x (rows, cols) to 8 bits with a scale for each 128 columns of a row: activations, gradients."""
    data, scales = (None, None) if out is None else out
    return Fp8Matrix(*_module().quantize_rows(x, _fp8_code(dtype, "compact_quantize_rows"), data, scales))


@_on_its_stream
def quantize_blocks(x: torch.Tensor, dtype: torch.dtype = torch.float8_e4m3fn, transpose: bool = True, out: Optional[Fp8Matrix] = None,
                    out_t: Optional[Fp8Matrix] = None) -> Tuple[Fp8Matrix, Optional[Fp8Matrix]]:
    """x (rows, cols) to 8 bits with a scale for each 128 x 128 block: weights.  Returns (x, its transpose) with the same
    values; without `transpose` the second is None."""
    data, scales = (None, None) if out is None else out
    data_t, scales_t = (None, None) if out_t is None else out_t
    q, s, qt, st = _module().quantize_blocks(x, _fp8_code(dtype, "compact_quantize_blocks"), data, scales, transpose, data_t, scales_t)
    return Fp8Matrix(q, s), None if qt is None else Fp8Matrix(qt, st)


class Fp8Product:
    """C = A B^T of 8-bit matrices: A (M, K), B (N, K).  The handle holds the status word of the kernels' bounded waits."""

    def __init__(self):
        self._h = C.c_void_p()
        _check(lib().compact_fp8_product_create(C.byref(self._h)), "compact_fp8_product_create")
        self._run = _module().fp8_product

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and _lib is not None:
            _lib.compact_fp8_product_destroy(h)
            self._h = None

    @_on_its_stream
    def __call__(self, a: Fp8Matrix, b: Fp8Matrix, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        return self._run(self._h.value, a.data, a.scales, b.data, b.scales, out, _float_code(dtype, "compact_fp8_product_run"))

    def status(self) -> int:
        """ERR_DEVICE_TIMEOUT if a kernel of this handle has given up on a wait since the last call, on any device or in a graph; OK
        otherwise.  Synchronises the devices that the handle has launched on."""
        return int(lib().compact_fp8_product_status(self._h))

    def debug_withhold(self, k_steps: int) -> None:
        """The next product loads only that many k-steps of each tile and gives up waiting for the rest after a few thousand polls (a test hook)."""
        _check(lib().compact_debug_fp8_product_withhold(self._h, k_steps), "compact_debug_fp8_product_withhold")


def set_product_kernel(which: int) -> int:
    """0: automatic, 1: pairs of SMs, 2: clusters that split K.  Returns the previous choice."""
    return lib().compact_fp8_product_set_kernel(which)


class ProductPlan(NamedTuple):
    kernel: int           # of an automatic product: 1 or 2
    width: int            # columns of a tile of the pairs' kernel
    tiles: int
    per_barrier: int      # k-steps
    panels: int           # of column tiles


def debug_product_plan(M: int, N: int, K: int) -> ProductPlan:
    """What (M, K) by (N, K) is divided into (a test hook; nothing is launched)."""
    plan = (C.c_int32 * 5)()
    _check(lib().compact_debug_fp8_product_plan(M, N, K, plan), "compact_debug_fp8_product_plan")
    return ProductPlan(*plan)


# -- RMS norm ---------------------------------------------------------------------------------------
class NormOutput(NamedTuple):
    h: torch.Tensor               # x + residual, what was normed (x itself without a residual)
    y: Optional[torch.Tensor]
    rstd: torch.Tensor            # fp32, one per token: what the backward needs besides h
    q: Optional[Fp8Matrix]


class RMSNorm:
    """y = h * rstd * weight with h = x + residual and rstd = 1 / sqrt(mean(h^2) + eps)."""

    def __init__(self, n: int, eps: float = 1e-6, dtype: torch.dtype = torch.bfloat16):
        self.code = _float_code(dtype, "RMSNorm")
        if not 1 <= n <= RMS_NORM_MAX_N:
            raise CompactError(ERR_SHAPE, "RMSNorm")
        if not (eps >= 0.0 and math.isfinite(C.c_float(eps).value)):      # as the kernel takes it
            raise CompactError(ERR_INVALID_ARG, "RMSNorm")
        self.n, self.eps, self.dtype = n, eps, dtype

    @_on_its_stream
    def forward(self, x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, want_y: bool = True, want_fp8: bool = False,
                fp8_dtype: torch.dtype = torch.float8_e4m3fn, h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                q: Optional[Fp8Matrix] = None) -> NormOutput:
        """want_y: y in the norm's dtype; want_fp8: y in 8 bits with a scale for each 128 columns, from the unrounded y.  With a
        residual, h may be passed as the memory to write x + residual to (x's or the residual's own, for an update in place)."""
        data, scales = (None, None) if q is None else q
        h, y, rstd, data, scales = _module().rms_norm_fwd(self.code, self.n, self.eps, x, weight, residual, h, want_y, y, want_fp8,
                                                          _fp8_code(fp8_dtype, "compact_rms_norm_fwd"), data, scales)
        return NormOutput(h, y, rstd, None if data is None else Fp8Matrix(data, scales))

    @_on_its_stream
    def backward(self, dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, residual_grad: Optional[torch.Tensor] = None,
                 dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, need_dx: bool = True, need_dweight: bool = True,
                 accumulate: bool = False):
        """Returns (dx, dweight): the gradient of x (and of the residual) and, in fp32, of the weight.  residual_grad: the
        gradient that reaches h past the norm.  accumulate adds to the dweight passed in."""
        return _module().rms_norm_bwd(self.code, self.n, dy, h, weight, rstd, residual_grad, need_dx, dx, need_dweight, dweight, accumulate)


# -- rotary positions -------------------------------------------------------------------------------
class Rotary:
    """Turns the first rot_dim elements of every head by position; see include/compact_block.h for the scalings."""

    def __init__(self, head_dim: int, rot_dim: Optional[int] = None, base: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                 factor: float = 1.0, low: float = 1.0, high: float = 4.0, trained_length: float = 8192, attention_factor: float = 1.0):
        if scaling not in _SCALINGS:
            raise CompactError(ERR_INVALID_ARG, "Rotary: unknown scaling")
        self.head_dim, self.rot_dim = head_dim, head_dim if rot_dim is None else rot_dim
        cfg = RotaryConfig(head_dim, self.rot_dim, int(interleaved), _SCALINGS[scaling], base, factor, low, high, trained_length, attention_factor)
        self._h = C.c_void_p()
        _check(lib().compact_rotary_create(C.byref(cfg), C.byref(self._h)), "compact_rotary_create")
        self._turn = _module().rotary_apply

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and _lib is not None:
            _lib.compact_rotary_destroy(h)
            self._h = None

    @_on_its_stream
    def forward(self, q: torch.Tensor, k: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None, first_position: int = 0,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """q (tokens, heads, head_dim) and k (tokens, kv_heads, head_dim), any strides between tokens and heads; positions: one
        integer per token, or token t stands at first_position + t.  Outputs may be the inputs."""
        return self._turn(self._h.value, self.head_dim, q, k, positions, first_position, 0, q_out, k_out)

    @_on_its_stream
    def backward(self, dq: torch.Tensor, dk: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None, first_position: int = 0,
                 dq_out: Optional[torch.Tensor] = None, dk_out: Optional[torch.Tensor] = None):
        """The gradient: the transposed turn, for the same positions."""
        return self._turn(self._h.value, self.head_dim, dq, dk, positions, first_position, 1, dq_out, dk_out)
