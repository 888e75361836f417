"""ctypes binding of the operators around 8-bit projections (include/tn_fp8.h): argument marshalling only.

Root-mean-square norm with the residual's addition, silu(gate) * up, products of 8-bit weights with 8-bit activations, and
the gradients of all three. Tensors are torch CUDA (ROCm) tensors on the current GPU; work goes to its current HIP stream. Nothing
here computes.

    layer = tn.Fp8Linear([w_gate, w_up], max_tokens=8192)        # bf16 or fp32 [M, N] weights, quantised at create
    n = tn.rms_norm(x, weight, residual=res, outputs="fp8")      # n.sum = x + res, n.fp8 = the norm in 8 bits
    h = layer.gated(n.fp8)                                       # silu(gate) * up in 8 bits
    y = down(h)                                                  # bf16
"""
from __future__ import annotations

import ctypes
from typing import List, NamedTuple, Optional, Sequence, Tuple

import torch

from .binding import (TN_DTYPE_BF16, TN_DTYPE_F32, TN_FLAG_TRANSPOSE, TN_QUERY_IN_FEATURES, TN_QUERY_OUT_FEATURES, TNLinearError,
                      load_library)

TN_DTYPE_FP8 = 2
TN_FP8_BLOCK = 128

FP8_EXPORTED_SYMBOLS = (
    "tn_fp8_row_strides",
    "tn_fp8_quantize",
    "tn_rms_norm",
    "tn_rms_norm_gradients",
    "tn_rms_norm_gradients_workspace",
    "tn_silu_gate",
    "tn_silu_gate_gradients",
    "tn_fp8_linear_create",
    "tn_fp8_linear_forward",
    "tn_fp8_linear_gated",
    "tn_fp8_linear_plan_query",
    "tn_fp8_linear_tensor",
    "tn_fp8_linear_query",
    "tn_fp8_linear_destroy",
)

_CODES, _SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu
_DTYPE = {torch.float32: TN_DTYPE_F32, torch.bfloat16: TN_DTYPE_BF16}


class _Desc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("n_tensors", ctypes.c_int32),
        ("out_features", ctypes.c_int64),
        ("in_features", ctypes.c_int64),
        ("tensors", ctypes.POINTER(ctypes.c_void_p)),
        ("scales", ctypes.POINTER(ctypes.c_void_p)),
        ("max_tokens", ctypes.c_int64),
        ("flags", ctypes.c_int32),
        ("stream", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_int64),
    ]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        p, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        args = {
            "tn_fp8_row_strides": [i64, i32, ctypes.POINTER(i64), ctypes.POINTER(i64)],
            "tn_fp8_quantize": [i32, i64, i64, i32, p, i64, p, p, p],
            "tn_rms_norm": [i32, i64, i64, p, i64, p, i64, p, f32, p, i64, p, i64, p, p, p],
            "tn_rms_norm_gradients": [i32, i64, i64, p, i64, p, i64, p, f32, p, i64, p, i64, p, p, i64, p],
            "tn_rms_norm_gradients_workspace": [i64, i64],
            "tn_silu_gate": [i32, i64, i64, p, i64, p, i64, p, p, p],
            "tn_silu_gate_gradients": [i32, i64, i64, p, i64, p, i64, p, i64, p, p, p],
            "tn_fp8_linear_create": [ctypes.POINTER(p), ctypes.POINTER(_Desc)],
            "tn_fp8_linear_forward": [p, p, p, p, i64, i64, p],
            "tn_fp8_linear_gated": [p, p, p, p, p, i64, p],
            "tn_fp8_linear_plan_query": [ctypes.POINTER(_Desc), i64, i32, i32, ctypes.POINTER(i64)],
            "tn_fp8_linear_tensor": [p, i32, p, p, p],
            "tn_fp8_linear_query": [p, i32, ctypes.POINTER(i64)],
            "tn_fp8_linear_destroy": [p],
        }
        for name, types in args.items():
            fn = getattr(lib, name)
            fn.argtypes = types
            fn.restype = i64 if name == "tn_rms_norm_gradients_workspace" else ctypes.c_int
        _lib = lib
    return _lib


def _check(status: int, where: str) -> None:
    if status != 0:
        raise TNLinearError(status, where)


# The binding's own time is most of a small call's. torch.cuda.current_stream() builds an object (2.8 us); this is what it asks (0.1).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_gpu = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(gpu: int) -> int:
    """The current HIP stream of that GPU."""
    if _raw_stream is None:
        return torch.cuda.current_stream(gpu).cuda_stream
    return _raw_stream(gpu)


# Launches go to the current GPU, and nothing maps another one's memory there: every tensor of a call must be on it. (get_device() of a tensor
# in host memory is -1.)
def _here(name: str, gpu: int) -> int:
    if gpu != _current_gpu():
        raise ValueError(f"{name} is on GPU {gpu}, and GPU {_current_gpu()} is the current one")
    return gpu


def _matrix(name: str, t: torch.Tensor, rows: int, cols: int, dtype: torch.dtype, gpu: int) -> int:
    """The row stride of t, a [rows, cols] matrix of dtype on that GPU whose rows are contiguous and apart."""
    if not (t.dtype is dtype and t.shape == (rows, cols) and t.get_device() == gpu):
        raise ValueError(f"{name} must be a [{rows}, {cols}] tensor of {dtype} on GPU {gpu}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
    stride, step = t.stride()
    if rows <= 1:
        stride = cols
    if (step != 1 and cols > 1) or stride < cols:
        raise ValueError(f"{name}: elements of a row must be contiguous and rows must not overlap (strides {t.stride()})")
    return stride


def _input(name: str, t: torch.Tensor) -> Tuple[int, int]:
    """(type code, GPU) of an input matrix that sets the type of a call: on the current GPU."""
    code = _DTYPE.get(t.dtype)
    if code is None or t.dim() != 2 or t.shape[1] < 1 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA [rows, cols] tensor of float32 or bfloat16, not {tuple(t.shape)} of {t.dtype} on {t.device}")
    return code, _here(name, t.get_device())


def _vector(name: str, t: Optional[torch.Tensor], cols: int, dtype: torch.dtype, gpu: int) -> Optional[int]:
    if t is None:
        return None
    if not (t.get_device() == gpu and t.dtype == dtype and t.dim() == 1 and t.shape[0] == cols and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous [{cols}] tensor of {dtype} on GPU {gpu}")
    return t.data_ptr()


class Fp8Rows:
    """Rows in 8 bits: `codes` (float8_e4m3fn [rows, segments * P], P = cols rounded up to 128) and `scales` (float8_e8m0fnu
    [rows, S], one for each block of 128, S rounded up to 4), as include/tn_fp8.h lays them out. `values` and `block_scales`
    are views of a segment without its padding. Padding has to be zero, codes and scale bytes: every function here writes it so, and
    products read it. Whoever makes Fp8Rows of codes of their own clears it (a NaN code there makes its row's products NaN)."""

    __slots__ = ("codes", "scales", "rows", "cols", "segments", "_parts")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int, segments: int = 1):
        width, blocks = -(-cols // TN_FP8_BLOCK) * TN_FP8_BLOCK * segments, -(-cols // TN_FP8_BLOCK) * segments
        rows = codes.shape[0]
        if not (codes.is_cuda and codes.dtype == _CODES and codes.is_contiguous() and tuple(codes.shape) == (rows, width)):
            raise ValueError(f"codes must be a contiguous CUDA [rows, {width}] tensor of float8_e4m3fn")
        if not (scales.get_device() == codes.get_device() and scales.dtype == _SCALES and scales.is_contiguous()
                and tuple(scales.shape) == (rows, -(-blocks // 4) * 4)):
            raise ValueError(f"scales must be a contiguous [{rows}, {-(-blocks // 4) * 4}] tensor of float8_e8m0fnu on the GPU of codes")
        self.codes, self.scales, self.rows, self.cols, self.segments, self._parts = codes, scales, rows, cols, segments, None

    @classmethod
    def empty(cls, rows: int, cols: int, segments: int = 1, device="cuda") -> "Fp8Rows":
        blocks = -(-cols // TN_FP8_BLOCK) * segments
        new = cls.__new__(cls)
        new.codes = torch.empty((rows, blocks * TN_FP8_BLOCK), dtype=_CODES, device=device)
        new.scales = torch.empty((rows, -(-blocks // 4) * 4), dtype=_SCALES, device=device)
        if not new.codes.is_cuda:
            raise ValueError("Fp8Rows live on a GPU")
        new.rows, new.cols, new.segments, new._parts = rows, cols, segments, None
        return new

    def _segment(self, segment: int):
        """(codes, scales) of a segment: views, made once for all segments (a view costs as much as a tenth of a small call)."""
        parts = self._parts
        if parts is None:
            cols, segments, blocks = self.cols, self.segments, -(-self.cols // TN_FP8_BLOCK)
            codes, scales = self.codes, self.scales
            codes = codes.split(blocks * TN_FP8_BLOCK, 1) if segments > 1 else (codes,)
            if cols % TN_FP8_BLOCK:
                codes = [c.narrow(1, 0, cols) for c in codes]
            if scales.shape[1] != blocks * segments:
                scales = scales.narrow(1, 0, blocks * segments)
            scales = scales.split(blocks, 1) if segments > 1 else (scales,)
            parts = self._parts = (codes, scales)
        return parts[0][segment], parts[1][segment]

    def values(self, segment: int = 0) -> torch.Tensor:
        return self._segment(segment)[0]

    def block_scales(self, segment: int = 0) -> torch.Tensor:
        return self._segment(segment)[1]

    def _ready(self, name: str, rows: int, cols: int, segments: int, gpu: int) -> "Fp8Rows":
        if (self.rows, self.cols, self.segments) != (rows, cols, segments):
            raise ValueError(f"{name} holds [{self.rows}, {self.segments} x {self.cols}], not [{rows}, {segments} x {cols}]")
        if self.codes.get_device() != gpu:
            raise ValueError(f"{name} is on {self.codes.device}, not on GPU {gpu}")
        return self


class RowOutput(NamedTuple):
    """What a row operator returns; None for what was not asked for."""
    y: Optional[torch.Tensor]
    fp8: Optional[Fp8Rows]
    sum: Optional[torch.Tensor] = None


_OUTPUTS = {"y": (True, False), "fp8": (False, True), "both": (True, True)}


def _outputs(outputs: str, out: Optional[RowOutput], like: torch.Tensor, rows: int, cols: int, segments: int, gpu: int):
    """(y, its address, its row stride, fp8, the addresses of its codes and scales) of a call: the caller's, or new ones."""
    want = _OUTPUTS.get(outputs)
    if want is None:
        raise ValueError('outputs is "y", "fp8" or "both"')
    y, y_ptr, stride, fp8, codes, scales = None, None, 0, None, None, None
    if want[0]:
        if out is not None and out.y is not None:
            y = out.y
            stride = _matrix("out.y", y, rows, segments * cols, like.dtype, gpu)
        else:
            stride = segments * cols
            y = like.new_empty((rows, stride))
        y_ptr = y.data_ptr()
    if want[1]:
        if out is not None and out.fp8 is not None:
            fp8 = out.fp8._ready("out.fp8", rows, cols, segments, gpu)
        else:
            fp8 = Fp8Rows.empty(rows, cols, segments, like.device)
        codes, scales = fp8.codes.data_ptr(), fp8.scales.data_ptr()
    return y, y_ptr, stride, fp8, codes, scales


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def quantize_fp8(x: torch.Tensor, segments: int = 1, out: Optional[Fp8Rows] = None) -> Fp8Rows:
    """x [rows, segments * cols] in 8 bits, each segment in blocks of its own."""
    code, gpu = _input("x", x)
    rows, width = x.shape
    if segments < 1 or width % segments:
        raise ValueError(f"x has {width} columns: not {segments} equal segments")
    cols = width // segments
    stride = _matrix("x", x, rows, width, x.dtype, gpu)
    out = Fp8Rows.empty(rows, cols, segments, x.device) if out is None else out._ready("out", rows, cols, segments, gpu)
    _check(_library().tn_fp8_quantize(code, rows, cols, segments, x.data_ptr(), stride, out.codes.data_ptr(), out.scales.data_ptr(), _stream(gpu)),
           "tn_fp8_quantize")
    return out


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
             outputs: str = "y", out: Optional[RowOutput] = None) -> RowOutput:
    """s = x + residual (in x's type), y = s / sqrt(mean(s^2) + eps) * weight. `outputs`: "y" (x's type), "fp8" (8 bits) or
    "both". Returns (y, fp8, sum); sum is s where there is a residual, and may be given as out.sum. out.y and out.sum may be x or
    residual themselves, but not the same tensor."""
    code, gpu = _input("x", x)
    rows, cols = x.shape
    x_stride, weight_ptr = _matrix("x", x, rows, cols, x.dtype, gpu), _vector("weight", weight, cols, x.dtype, gpu)
    y, y_ptr, y_stride, fp8, codes, scales = _outputs(outputs, out, x, rows, cols, 1, gpu)
    total, total_ptr, res_ptr, res_stride, sum_stride = None, None, None, 0, 0
    if residual is not None:
        res_stride, res_ptr = _matrix("residual", residual, rows, cols, x.dtype, gpu), residual.data_ptr()
        if out is not None and out.sum is not None:
            total = out.sum
            sum_stride = _matrix("out.sum", total, rows, cols, x.dtype, gpu)
        else:
            total, sum_stride = x.new_empty((rows, cols)), cols
        total_ptr = total.data_ptr()
    _check(_library().tn_rms_norm(code, rows, cols, x.data_ptr(), x_stride, res_ptr, res_stride, weight_ptr, eps, total_ptr, sum_stride, y_ptr,
                                  y_stride, codes, scales, _stream(gpu)), "tn_rms_norm")
    return RowOutput(y, fp8, total)


def rms_norm_gradients(dy: torch.Tensor, s: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                       dsum: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, dweight: bool = True
                       ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dx, dweight) of rms_norm for the gradient dy of its y and, where s is read elsewhere too, the gradient dsum that arrives
    there: dx in s's type, for x and the residual alike; dweight in fp32 (None without a weight, or with dweight=False).
    s is what rms_norm returned as sum (x, if it had no residual)."""
    code, gpu = _input("s", s)
    rows, cols = s.shape
    s_stride, weight_ptr = _matrix("s", s, rows, cols, s.dtype, gpu), _vector("weight", weight, cols, s.dtype, gpu)
    dy_stride = _matrix("dy", dy, rows, cols, s.dtype, gpu)
    ds_stride = 0 if dsum is None else _matrix("dsum", dsum, rows, cols, s.dtype, gpu)
    if dx is None:
        dx, dx_stride = s.new_empty((rows, cols)), cols
    else:
        dx_stride = _matrix("dx", dx, rows, cols, s.dtype, gpu)
    lib = _library()
    dw, space, need = None, None, 0
    if dweight and weight is not None:
        need = lib.tn_rms_norm_gradients_workspace(rows, cols)
        if need < 0:
            _check(int(need), "tn_rms_norm_gradients_workspace")
        dw = s.new_empty((cols,), dtype=torch.float32)
        space = s.new_empty((need,), dtype=torch.uint8)
    _check(lib.tn_rms_norm_gradients(code, rows, cols, dy.data_ptr(), dy_stride, s.data_ptr(), s_stride, weight_ptr, eps, _ptr(dsum), ds_stride,
                                     dx.data_ptr(), dx_stride, _ptr(dw), _ptr(space), need, _stream(gpu)), "tn_rms_norm_gradients")
    return dx, dw


def silu_gate(gate_up: torch.Tensor, outputs: str = "y", out: Optional[RowOutput] = None) -> RowOutput:
    """silu(gate) * up of gate_up = [gate | up], [rows, 2 * cols]; outputs as in rms_norm."""
    code, gpu = _input("gate_up", gate_up)
    rows, cols = gate_up.shape[0], gate_up.shape[1] // 2
    stride = _matrix("gate_up", gate_up, rows, 2 * cols, gate_up.dtype, gpu)
    y, y_ptr, y_stride, fp8, codes, scales = _outputs(outputs, out, gate_up, rows, cols, 1, gpu)
    _check(_library().tn_silu_gate(code, rows, cols, gate_up.data_ptr(), stride, y_ptr, y_stride, codes, scales, _stream(gpu)), "tn_silu_gate")
    return RowOutput(y, fp8)


def silu_gate_gradients(gate_up: torch.Tensor, dh: torch.Tensor, outputs: str = "y", out: Optional[RowOutput] = None) -> RowOutput:
    """[dgate | dup] for the gradient dh of silu(gate) * up; in 8 bits they are two segments."""
    code, gpu = _input("gate_up", gate_up)
    rows, cols = gate_up.shape[0], gate_up.shape[1] // 2
    stride = _matrix("gate_up", gate_up, rows, 2 * cols, gate_up.dtype, gpu)
    dh_stride = _matrix("dh", dh, rows, cols, gate_up.dtype, gpu)
    y, y_ptr, y_stride, fp8, codes, scales = _outputs(outputs, out, gate_up, rows, cols, 2, gpu)
    _check(_library().tn_silu_gate_gradients(code, rows, cols, gate_up.data_ptr(), stride, dh.data_ptr(), dh_stride, y_ptr, y_stride, codes,
                                             scales, _stream(gpu)), "tn_silu_gate_gradients")
    return RowOutput(y, fp8)


TN_FP8_PLAN_TILE_TOKENS, TN_FP8_PLAN_TILE_FEATURES, TN_FP8_PLAN_RANGES, TN_FP8_PLAN_FUSED, TN_FP8_PLAN_STREAM_PIECES = range(5)


def fp8_plan_query(out_features: int, in_features: int, n_tensors: int, tokens: int, gated: bool, what: int, transpose: bool = False,
                   max_tokens: Optional[int] = None) -> int:
    """Host-only: how a call of such a layer would run (TN_FP8_PLAN_*); needs no GPU."""
    desc = _Desc()
    desc.dtype, desc.n_tensors, desc.out_features, desc.in_features = TN_DTYPE_BF16, n_tensors, out_features, in_features
    desc.max_tokens, desc.flags = tokens if max_tokens is None else max_tokens, TN_FLAG_TRANSPOSE if transpose else 0
    value = ctypes.c_int64(0)
    _check(_library().tn_fp8_linear_plan_query(ctypes.byref(desc), tokens, int(gated), what, ctypes.byref(value)), "tn_fp8_linear_plan_query")
    return int(value.value)


class Fp8Linear:
    """One 8-bit weight [M, N], or two that read the same activations (gate and up), living on the GPU that is current when it is made
    and has to be current when it is used.

    tensors  one or two contiguous CUDA tensors of float32 or bfloat16, quantised in blocks of 128 x 128; or, with `scales`,
             float8_e4m3fn codes and their float8_e8m0fnu scales [ceil(M / 128), ceil(N / 128)]
    workspace  a block of CUDA memory that several layers may share (up to 64 MB are of use), instead of one of the layer's own
    transpose=True  the layer maps gradients of the outputs (two segments for two tensors) to that of the inputs
    """

    def __init__(self, tensors: Sequence[torch.Tensor], max_tokens: int, transpose: bool = False,
                 scales: Optional[Sequence[torch.Tensor]] = None, workspace: Optional[torch.Tensor] = None):
        self._handle = None
        if not torch.cuda.is_available():
            raise RuntimeError("Fp8Linear needs a GPU: there is no CPU path")
        tensors = list(tensors)
        if len(tensors) not in (1, 2) or any(t.dim() != 2 or t.shape != tensors[0].shape or t.dtype != tensors[0].dtype for t in tensors):
            raise ValueError("one or two [M, N] tensors of the same size and type")
        first = tensors[0]
        code = TN_DTYPE_FP8 if scales is not None else _DTYPE.get(first.dtype)
        if code is None or (scales is not None and first.dtype != _CODES) or not all(t.is_cuda and t.is_contiguous() for t in tensors):
            raise ValueError("tensors must be contiguous CUDA tensors of float32 or bfloat16, or of float8_e4m3fn together with their scales")
        gpu = _here("tensors", first.get_device())
        if tensors[-1].get_device() != gpu:
            raise ValueError("tensors must be on one GPU")
        m, n = first.shape
        desc = _Desc()
        desc.dtype, desc.n_tensors, desc.out_features, desc.in_features = code, len(tensors), m, n
        ptrs = (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
        desc.tensors = ptrs
        if scales is not None:
            shape = (-(-m // TN_FP8_BLOCK), -(-n // TN_FP8_BLOCK))
            if len(scales) != len(tensors) or any(not (s.get_device() == gpu and s.is_contiguous() and s.dtype == _SCALES and tuple(s.shape) == shape) for s in scales):
                raise ValueError(f"scales: one contiguous {list(shape)} tensor of float8_e8m0fnu for each tensor, on its GPU")
            scale_ptrs = (ctypes.c_void_p * len(tensors))(*[s.data_ptr() for s in scales])
            desc.scales = scale_ptrs
        self._workspace = workspace          # keep the caller's block alive as long as the handle
        if workspace is not None:
            if not (workspace.get_device() == gpu and workspace.is_contiguous() and workspace.numel() > 0):
                raise ValueError("workspace must be a contiguous tensor on the GPU of the tensors")
            desc.workspace, desc.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        desc.max_tokens, desc.flags, desc.stream = int(max_tokens), TN_FLAG_TRANSPOSE if transpose else 0, _stream(gpu)
        h = ctypes.c_void_p(0)
        _check(_library().tn_fp8_linear_create(ctypes.byref(h), ctypes.byref(desc)), "tn_fp8_linear_create")
        self._handle = int(h.value)
        self.shape, self.n_tensors, self.transpose = (m, n), len(tensors), bool(transpose)
        self._device, self._gpu = first.device, gpu
        self.M, self.N = self.query(TN_QUERY_OUT_FEATURES), self.query(TN_QUERY_IN_FEATURES)
        self._segments = len(tensors) if transpose else 1

    def _open(self) -> None:
        if self._handle is None:
            raise RuntimeError("layer was closed")
        _here("the layer", self._gpu)

    def _input(self, x) -> Fp8Rows:
        self._open()
        if not isinstance(x, Fp8Rows):
            if x.dim() != 2 or x.shape[1] != self.N:
                raise ValueError(f"x must be [tokens, {self.N}]")
            x = quantize_fp8(x, self._segments)
        return x._ready("x", x.rows, self.N // self._segments, self._segments, self._gpu)

    def forward(self, x, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """bf16 [tokens, M] for x in 8 bits (Fp8Rows), or a float32 / bfloat16 tensor, which is quantised first; two
        tensors' outputs lie beside each other."""
        x = self._input(x)
        if out is None:
            out, stride = torch.empty((x.rows, self.M), dtype=torch.bfloat16, device=self._device), self.M
        else:
            stride = _matrix("out", out, x.rows, self.M, torch.bfloat16, self._gpu)
        _check(_lib.tn_fp8_linear_forward(self._handle, x.codes.data_ptr(), x.scales.data_ptr(), out.data_ptr(), stride, x.rows, _stream(self._gpu)),
               "tn_fp8_linear_forward")
        return out

    __call__ = forward

    def gated(self, x, out: Optional[Fp8Rows] = None) -> Fp8Rows:
        """silu(x Wg^T) * (x Wu^T) in 8 bits, for a layer of two tensors (Wg, Wu); not in place of x."""
        if self.n_tensors != 2 or self.transpose:
            raise ValueError("gated needs a layer of two tensors that is not transposed")
        x = self._input(x)
        m = self.shape[0]
        out = Fp8Rows.empty(x.rows, m, 1, self._device) if out is None else out._ready("out", x.rows, m, 1, self._gpu)
        _check(_lib.tn_fp8_linear_gated(self._handle, x.codes.data_ptr(), x.scales.data_ptr(), out.codes.data_ptr(), out.scales.data_ptr(),
                                        x.rows, _stream(self._gpu)), "tn_fp8_linear_gated")
        return out

    def quantized_tensor(self, slot: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
        """(codes [M, N], scales [ceil(M / 128), ceil(N / 128)]) of tensor `slot`."""
        self._open()
        m, n = self.shape
        codes = torch.empty((m, n), dtype=_CODES, device=self._device)
        scales = torch.empty((-(-m // TN_FP8_BLOCK), -(-n // TN_FP8_BLOCK)), dtype=_SCALES, device=self._device)
        _check(_lib.tn_fp8_linear_tensor(self._handle, int(slot), codes.data_ptr(), scales.data_ptr(), _stream(self._gpu)), "tn_fp8_linear_tensor")
        return codes, scales

    def query(self, what: int) -> int:
        if self._handle is None:
            raise RuntimeError("layer was closed")
        value = ctypes.c_int64(0)
        _check(_library().tn_fp8_linear_query(self._handle, int(what), ctypes.byref(value)), "tn_fp8_linear_query")
        return int(value.value)

    def close(self) -> None:
        if self._handle is not None:
            handle, self._handle = self._handle, None
            _check(_library().tn_fp8_linear_destroy(handle), "tn_fp8_linear_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
