"""ctypes binding of the projections with frozen 4-bit weights (include/tn_int4.h): argument marshalling only.

Weights are whole numbers of 4 bits under group scales, W[f][k] = (code - zero) * scale, activations bf16. Tensors are torch CUDA (ROCm)
tensors on the current GPU; work goes to its current HIP stream. Nothing here computes.

    gate_up = tn.Int4Linear([w_gate, w_up], max_tokens=8192, group=128)      # bf16 or fp32 [M, N] weights, quantised at create
    down = tn.Int4Linear([codes], 8192, scales=[scales], zeros=[zeros])      # or codes as a checkpoint has them
    y = down(gate_up.gated(x))                                               # silu(gate) * up and its projection, bf16
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

import torch
from torch.autograd.graph import increment_version

from .binding import TN_DTYPE_BF16, TN_FLAG_TRANSPOSE, TN_QUERY_IN_FEATURES, TN_QUERY_OUT_FEATURES, load_library
from .fp8 import _DTYPE, _check, _here, _matrix, _stream

TN_DTYPE_INT4, TN_DTYPE_F16 = 3, 4

INT4_EXPORTED_SYMBOLS = (
    "tn_int4_linear_create",
    "tn_int4_linear_workspace",
    "tn_int4_linear_forward",
    "tn_int4_linear_gated",
    "tn_int4_linear_plan_query",
    "tn_int4_linear_tensor",
    "tn_int4_linear_query",
    "tn_int4_linear_destroy",
)

_SCALE_DTYPE = {torch.bfloat16: TN_DTYPE_BF16, torch.float16: TN_DTYPE_F16}


class _Desc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("n_tensors", ctypes.c_int32),
        ("out_features", ctypes.c_int64),
        ("in_features", ctypes.c_int64),
        ("group", ctypes.c_int32),
        ("scale_dtype", ctypes.c_int32),
        ("tensors", ctypes.POINTER(ctypes.c_void_p)),
        ("scales", ctypes.POINTER(ctypes.c_void_p)),
        ("zeros", ctypes.POINTER(ctypes.c_void_p)),
        ("flags", ctypes.c_int32),
        ("stream", ctypes.c_void_p),
    ]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        args = {
            "tn_int4_linear_create": [ctypes.POINTER(p), ctypes.POINTER(_Desc)],
            "tn_int4_linear_workspace": [p, p, i64, i64, i32],
            "tn_int4_linear_forward": [p, p, i64, p, i64, i64, p, i64, p],
            "tn_int4_linear_gated": [p, p, i64, p, i64, i64, p, i64, p],
            "tn_int4_linear_plan_query": [ctypes.POINTER(_Desc), i64, i32, i32, ctypes.POINTER(i64)],
            "tn_int4_linear_tensor": [p, i32, p, p, p, p],
            "tn_int4_linear_query": [p, i32, ctypes.POINTER(i64)],
            "tn_int4_linear_destroy": [p],
        }
        for name, types in args.items():
            fn = getattr(lib, name)
            fn.argtypes = types
            fn.restype = i64 if name == "tn_int4_linear_workspace" else ctypes.c_int
        _lib = lib
    return _lib


def _pointers(tensors):
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


TN_INT4_PLAN_TILE_TOKENS, TN_INT4_PLAN_RANGES, TN_INT4_PLAN_STREAM_TOKENS, TN_INT4_PLAN_STREAM_PIECES = range(4)


def int4_plan_query(out_features: int, in_features: int, n_tensors: int, tokens: int, gated: bool, what: int, transpose: bool = False,
                    group: int = 128) -> int:
    """Host-only: how a call of such a layer would run (TN_INT4_PLAN_*); needs no GPU."""
    desc = _Desc()
    desc.dtype, desc.n_tensors, desc.out_features, desc.in_features = TN_DTYPE_BF16, n_tensors, out_features, in_features
    desc.group, desc.flags = group, TN_FLAG_TRANSPOSE if transpose else 0
    value = ctypes.c_int64(0)
    _check(_library().tn_int4_linear_plan_query(ctypes.byref(desc), tokens, int(gated), what, ctypes.byref(value)), "tn_int4_linear_plan_query")
    return int(value.value)


class Int4Linear:
    """One 4-bit weight [M, N], or two that read the same activations (gate and up), living on the GPU that is current when it is made
    and has to be current when it is used. Graphs that captured its calls are not replayed after close().

    tensors  one or two contiguous CUDA tensors: [M, N] of float32 or bfloat16, quantised in groups along N; or, with `scales`, uint8 codes
             [M, ceil(N / 2)], two to a byte with the even input in the low half
    max_tokens  the most tokens of a call
    group    inputs to a scale: 32, 64 or 128
    scales   bfloat16 or float16 [M, ceil(N / group)]; zeros  uint8 likewise, 0 to 15 (None: 8)
    in_features  N, where codes have one for a spare half byte too
    transpose=True  the layer maps gradients of the outputs (two tensors': beside each other) to that of the inputs
    """

    def __init__(self, tensors: Sequence[torch.Tensor], max_tokens: int, transpose: bool = False, group: int = 128,
                 scales: Optional[Sequence[torch.Tensor]] = None, zeros: Optional[Sequence[torch.Tensor]] = None, in_features: Optional[int] = None):
        self._handle = None
        if not torch.cuda.is_available():
            raise RuntimeError("Int4Linear needs a GPU: there is no CPU path")
        desc, keep, first, gpu = _description(tensors, max_tokens, transpose, group, scales, zeros, in_features)
        desc.stream = _stream(gpu)
        h = ctypes.c_void_p(0)
        _check(_library().tn_int4_linear_create(ctypes.byref(h), ctypes.byref(desc)), "tn_int4_linear_create")
        del keep
        self._handle = int(h.value)
        self.shape, self.n_tensors, self.transpose, self.group = (desc.out_features, desc.in_features), desc.n_tensors, bool(transpose), desc.group
        self.scale_dtype = torch.float16 if desc.scale_dtype == TN_DTYPE_F16 else torch.bfloat16
        self.max_tokens, self._device, self._gpu = int(max_tokens), first.device, gpu
        self.M, self.N = self.query(TN_QUERY_OUT_FEATURES), self.query(TN_QUERY_IN_FEATURES)

    def _run(self, fn, gated: bool, cols: int, x: torch.Tensor, out: Optional[torch.Tensor], where: str) -> torch.Tensor:
        if self._handle is None:
            raise RuntimeError("layer was closed")
        gpu = _here("the layer", self._gpu)
        if x.dim() != 2:
            raise ValueError(f"x must be [tokens, {self.N}]")
        tokens = x.shape[0]
        if tokens > self.max_tokens:
            raise ValueError(f"x has {tokens} tokens: the layer was made for {self.max_tokens}")
        x_stride = _matrix("x", x, tokens, self.N, torch.bfloat16, gpu)
        given = out is not None
        if not given:
            out, stride = torch.empty((tokens, cols), dtype=torch.bfloat16, device=self._device), cols
        else:
            stride = _matrix("out", out, tokens, cols, torch.bfloat16, gpu)
        x_ptr = x.data_ptr()
        need = _lib.tn_int4_linear_workspace(self._handle, x_ptr, x_stride, tokens, gated)
        if need < 0:
            _check(int(need), "tn_int4_linear_workspace")
        space = torch.empty((need,), dtype=torch.uint8, device=self._device) if need else None
        _check(fn(self._handle, x_ptr, x_stride, out.data_ptr(), stride, tokens, None if space is None else space.data_ptr(), need, _stream(gpu)), where)
        if given:
            increment_version(out)
        return out

    def forward(self, x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """bf16 [tokens, M] for bf16 x [tokens, N] (rows may have a stride); two tensors' outputs lie beside each other. out may not overlap x:
        columns of one buffer beside each other are apart."""
        return self._run(_library().tn_int4_linear_forward, False, self.M, x, out, "tn_int4_linear_forward")

    __call__ = forward

    def gated(self, x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """silu(x Wg^T) * (x Wu^T) in bf16, for a layer of two tensors (Wg, Wu)."""
        if self.n_tensors != 2 or self.transpose:
            raise ValueError("gated needs a layer of two tensors that is not transposed")
        return self._run(_library().tn_int4_linear_gated, True, self.shape[0], x, out, "tn_int4_linear_gated")

    def quantized_tensor(self, slot: int = 0) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(codes uint8 [M, ceil(N / 2)], scales float32 [M, ceil(N / group)], zeros uint8 likewise) of tensor `slot`. Another layer is made of
        them with scales.to(layer.scale_dtype), the type they came in (bfloat16 where they were made here), which holds them exactly."""
        if self._handle is None:
            raise RuntimeError("layer was closed")
        gpu = _here("the layer", self._gpu)
        m, n = self.shape
        groups = -(-n // self.group)
        codes = torch.empty((m, -(-n // 2)), dtype=torch.uint8, device=self._device)
        scales = torch.empty((m, groups), dtype=torch.float32, device=self._device)
        zeros = torch.empty((m, groups), dtype=torch.uint8, device=self._device)
        _check(_lib.tn_int4_linear_tensor(self._handle, int(slot), codes.data_ptr(), scales.data_ptr(), zeros.data_ptr(), _stream(gpu)), "tn_int4_linear_tensor")
        return codes, scales, zeros

    def query(self, what: int) -> int:
        if self._handle is None:
            raise RuntimeError("layer was closed")
        value = ctypes.c_int64(0)
        _check(_library().tn_int4_linear_query(self._handle, int(what), ctypes.byref(value)), "tn_int4_linear_query")
        return int(value.value)

    def close(self) -> None:
        if self._handle is not None:
            handle, self._handle = self._handle, None
            _check(_library().tn_int4_linear_destroy(handle), "tn_int4_linear_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _description(tensors, max_tokens, transpose, group, scales, zeros, in_features):
    """(description, what it points to, first tensor, GPU)"""
    tensors = list(tensors)
    if len(tensors) not in (1, 2) or any(t.dim() != 2 or t.shape != tensors[0].shape or t.dtype != tensors[0].dtype for t in tensors):
        raise ValueError("one or two [M, N] tensors of the same size and type")
    if group not in (32, 64, 128):
        raise ValueError(f"group is 32, 64 or 128, not {group}")
    if int(max_tokens) < 1:
        raise ValueError("max_tokens must be at least 1")
    first = tensors[0]
    code = TN_DTYPE_INT4 if scales is not None else _DTYPE.get(first.dtype)
    if code is None or (scales is not None and first.dtype != torch.uint8) or not all(t.is_cuda and t.is_contiguous() for t in tensors):
        raise ValueError("tensors must be contiguous CUDA tensors of float32 or bfloat16, or of uint8 together with their scales")
    gpu = _here("tensors", first.get_device())
    if any(t.get_device() != gpu for t in tensors):
        raise ValueError("tensors must be on one GPU")
    m, n = first.shape
    if scales is not None:
        n = 2 * n if in_features is None else int(in_features)
        if first.shape[1] != -(-n // 2):
            raise ValueError(f"codes of {n} inputs have {-(-n // 2)} bytes a row, not {first.shape[1]}")
    elif in_features is not None and in_features != n:
        raise ValueError(f"tensors have {n} inputs, not {in_features}")
    elif zeros is not None:
        raise ValueError("zeros go with scales")
    desc = _Desc()
    desc.dtype, desc.n_tensors, desc.out_features, desc.in_features, desc.group = code, len(tensors), m, n, group
    desc.flags = TN_FLAG_TRANSPOSE if transpose else 0
    keep = [_pointers(tensors)]
    desc.tensors = keep[0]
    if scales is not None:
        shape = (m, -(-n // group))
        fits = lambda s, types: s.get_device() == gpu and s.is_contiguous() and s.dtype in types and tuple(s.shape) == shape      # noqa: E731
        scales = list(scales)
        if len(scales) != len(tensors) or not all(fits(s, _SCALE_DTYPE) and s.dtype == scales[0].dtype for s in scales):
            raise ValueError(f"scales: one contiguous {list(shape)} tensor of bfloat16 or float16 for each tensor, on its GPU")
        desc.scale_dtype = _SCALE_DTYPE[scales[0].dtype]
        keep.append(_pointers(scales))
        desc.scales = keep[-1]
        if zeros is not None:
            zeros = list(zeros)
            if len(zeros) != len(tensors) or not all(fits(z, (torch.uint8,)) for z in zeros):
                raise ValueError(f"zeros: one contiguous {list(shape)} tensor of uint8 for each tensor, on its GPU")
            keep.append(_pointers(zeros))
            desc.zeros = keep[-1]
    return desc, keep, first, gpu
