"""ctypes binding of the AdamW step over many tensors (include/tn_adamw.h): argument marshalling only.

    optimizer = tn.AdamW(factors, lr=1e-4, weight_decay=0.01, state_bits=8)
    grads = layer.param_gradients(x, dy)                       # fp32, one for each factor
    norm = optimizer.step(grads, max_norm=1.0)                 # fp32 tensor on the GPU; nothing waits for it

Tensors are torch CUDA (ROCm) tensors on the current GPU; work goes to its current HIP stream. Nothing here computes.
"""
from __future__ import annotations

import ctypes
import math
from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch
from torch.autograd.graph import increment_version

from .binding import TN_DTYPE_BF16, TN_DTYPE_F32, load_library
from .fp8 import _CODES, _DTYPE, _SCALES, _check, _here, _stream

TN_ADAMW_BLOCK = 128

ADAMW_EXPORTED_SYMBOLS = (
    "tn_adamw_state_values",
    "tn_adamw_create",
    "tn_adamw_workspace",
    "tn_adamw_gradient_norm",
    "tn_adamw_step",
    "tn_adamw_reset_master",
    "tn_adamw_destroy",
)


class _Desc(ctypes.Structure):
    _fields_ = [
        ("n_tensors", ctypes.c_int32),
        ("state_bits", ctypes.c_int32),
        ("sizes", ctypes.POINTER(ctypes.c_int64)),
        ("dtypes", ctypes.POINTER(ctypes.c_int32)),
        ("params", ctypes.POINTER(ctypes.c_void_p)),
        ("decays", ctypes.POINTER(ctypes.c_float)),
        ("first", ctypes.c_void_p),
        ("second", ctypes.c_void_p),
        ("first_scales", ctypes.c_void_p),
        ("second_scales", ctypes.c_void_p),
        ("master", ctypes.c_void_p),
        ("count", ctypes.c_void_p),
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("seed", ctypes.c_uint32),
        ("init_master", ctypes.c_int32),
        ("stream", ctypes.c_void_p),
    ]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        p, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
        args = {
            "tn_adamw_state_values": [i32, ctypes.POINTER(i64)],
            "tn_adamw_create": [ctypes.POINTER(p), ctypes.POINTER(_Desc)],
            "tn_adamw_workspace": [p],
            "tn_adamw_gradient_norm": [p, ctypes.POINTER(p), ctypes.POINTER(i32), p, p, i64, p],
            "tn_adamw_step": [p, ctypes.POINTER(p), ctypes.POINTER(i32), f64, p, f64, p, i32, p, i64, p],
            "tn_adamw_reset_master": [p, p],
            "tn_adamw_destroy": [p],
        }
        for name, types in args.items():
            fn = getattr(lib, name)
            fn.argtypes = types
            fn.restype = i64 if name in ("tn_adamw_state_values", "tn_adamw_workspace") else ctypes.c_int
        _lib = lib
    return _lib


def _state_values(sizes: Sequence[int]) -> int:
    values = _library().tn_adamw_state_values(len(sizes), (ctypes.c_int64 * len(sizes))(*sizes))
    if values < 0:
        _check(int(values), "tn_adamw_state_values")
    return int(values)


class AdamW:
    """Updates `params` - contiguous CUDA tensors of float32 or bfloat16, no two of which overlap - in place, all in one launch for up to 256
    of them, and lives on the GPU that is current when it is made and has to be current when it is used.

    weight_decay  one number, or one for each tensor (none for norms' weights, say)
    state_bits    32: m and v in fp32; 8: m and sqrt(v) in e4m3 with a scale for each 128 and rounding at random, 2.02 bytes a value instead of 8,
                  and the step divides by no less than the least sqrt(v) that gradients can leave beside that m
    seed          of that rounding: whoever starts again from a state_dict() with the same seed gets the same results

    A bfloat16 parameter is the rounding of an fp32 master held here, so that whoever sets it from outside calls reset_master(). Steps
    of one optimizer follow each other (on one stream, or on several that wait for each other). Graphs that captured them are not replayed after close().
    """

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.01, state_bits: int = 32, seed: int = 0):
        self._handle = None
        if not torch.cuda.is_available():
            raise RuntimeError("AdamW needs a GPU: there is no CPU path")
        params = list(params)
        gpu = _check_params(params)
        decays = _check_numbers(len(params), lr, betas, eps, weight_decay, state_bits, seed)
        device = params[0].device
        self.params, self.lr, self.betas, self.eps, self.weight_decay = params, float(lr), (float(betas[0]), float(betas[1])), float(eps), decays
        self.state_bits, self.seed, self._gpu, self._device = int(state_bits), int(seed), gpu, device
        self._sizes, self._shapes = [p.numel() for p in params], [p.shape for p in params]
        self._param_pointers = [p.data_ptr() for p in params]
        self._all_f32 = (ctypes.c_int32 * len(params))(*[TN_DTYPE_F32] * len(params))
        values = _state_values(self._sizes)
        kind = torch.float32 if state_bits == 32 else _CODES
        new = lambda n, dtype: torch.zeros((n,), dtype=torch.uint8 if dtype.itemsize == 1 else dtype, device=device).view(dtype)      # noqa: E731
        self._state: Dict[str, torch.Tensor] = {"first": new(values, kind), "second": new(values, kind), "count": torch.zeros((), dtype=torch.int64, device=device)}
        if state_bits == 8:
            self._state["first_scales"], self._state["second_scales"] = new(values // TN_ADAMW_BLOCK, _SCALES), new(values // TN_ADAMW_BLOCK, _SCALES)
        if any(p.dtype == torch.bfloat16 for p in params):
            self._state["master"] = new(values, torch.float32)
        self._make()

    def _make(self) -> None:
        n, s = len(self.params), self._state
        desc = _Desc()
        desc.n_tensors, desc.state_bits = n, self.state_bits
        desc.sizes = (ctypes.c_int64 * n)(*self._sizes)
        desc.dtypes = (ctypes.c_int32 * n)(*[_DTYPE[p.dtype] for p in self.params])
        desc.params = ctypes.cast((ctypes.c_void_p * n)(*[p.data_ptr() for p in self.params]), ctypes.POINTER(ctypes.c_void_p))
        desc.decays = (ctypes.c_float * n)(*self.weight_decay)
        desc.first, desc.second, desc.count = s["first"].data_ptr(), s["second"].data_ptr(), s["count"].data_ptr()
        if self.state_bits == 8:
            desc.first_scales, desc.second_scales = s["first_scales"].data_ptr(), s["second_scales"].data_ptr()
        if "master" in s:
            desc.master = s["master"].data_ptr()
        desc.beta1, desc.beta2, desc.eps, desc.seed, desc.init_master = *self.betas, self.eps, self.seed, 1
        desc.stream = _stream(self._gpu)
        h = ctypes.c_void_p(0)
        _check(_library().tn_adamw_create(ctypes.byref(h), ctypes.byref(desc)), "tn_adamw_create")
        self._handle = int(h.value)
        self._workspace_bytes = int(_lib.tn_adamw_workspace(self._handle))

    def reset_master(self) -> None:
        """Masters from the parameters as they are: one launch on the current stream, in its place among the steps. Captured steps stay
        valid, and read the new masters."""
        self._open()
        self._in_place()
        _check(_lib.tn_adamw_reset_master(self._handle, _stream(self._gpu)), "tn_adamw_reset_master")

    def _open(self) -> None:
        if self._handle is None:
            raise RuntimeError("optimizer was closed")
        _here("the optimizer", self._gpu)

    def _in_place(self) -> None:
        if [p.data_ptr() for p in self.params] != self._param_pointers:
            raise RuntimeError("a parameter's memory is not where it was when the optimizer was made")

    def _gradients(self, grads: Sequence[torch.Tensor]):
        self._open()
        n, gpu, f32, bf16 = len(self._shapes), self._gpu, torch.float32, torch.bfloat16
        grads = list(grads)
        if len(grads) != n:
            raise ValueError(f"{len(grads)} gradients for {n} parameters")
        pointers, halves = [], []
        # (for hundreds of tensors this loop is most of a call's time on the host: as little as it takes)
        for g, shape in zip(grads, self._shapes):
            if not isinstance(g, torch.Tensor) or g.shape != shape or g.get_device() != gpu or not g.is_contiguous():
                raise ValueError(f"gradient {len(pointers)} must be a contiguous {tuple(shape)} tensor of float32 or bfloat16 on GPU {gpu}")
            dtype = g.dtype
            if dtype is not f32:
                if dtype is not bf16:
                    raise ValueError(f"gradient {len(pointers)} must be of float32 or bfloat16, not {dtype}")
                halves.append(len(pointers))
            pointers.append(g.data_ptr())
        codes = self._all_f32
        if halves:
            codes = (ctypes.c_int32 * n)()              # (TN_DTYPE_F32 is 0)
            for i in halves:
                codes[i] = TN_DTYPE_BF16
        return (ctypes.c_void_p * n)(*pointers), codes

    def _space(self) -> torch.Tensor:
        return torch.empty((self._workspace_bytes,), dtype=torch.uint8, device=self._device)

    def gradient_norm(self, grads: Sequence[torch.Tensor], out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """sqrt(sum of the squares of all gradients) as a float32 tensor of one value, summed in 64 bits."""
        pointers, codes = self._gradients(grads)
        given = out is not None
        out = self._scalar("out", out) if given else torch.empty((), dtype=torch.float32, device=self._device)
        space = self._space()
        _check(_lib.tn_adamw_gradient_norm(self._handle, pointers, codes, out.data_ptr(), space.data_ptr(), self._workspace_bytes, _stream(self._gpu)),
               "tn_adamw_gradient_norm")
        if given:
            increment_version(out)
        return out

    def _scalar(self, name: str, t: torch.Tensor) -> torch.Tensor:
        if not (isinstance(t, torch.Tensor) and t.get_device() == self._gpu and t.dtype == torch.float32 and t.numel() == 1):
            raise ValueError(f"{name} must be a float32 tensor of one value on GPU {self._gpu}")
        return t

    def step(self, grads: Sequence[torch.Tensor], lr: Union[float, torch.Tensor, None] = None, max_norm: Optional[float] = None,
             norm: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """One step with one gradient for each parameter (float32 or bfloat16, of its shape). lr: a number instead of the optimizer's, or a
        float32 tensor of one value, which a captured step reads at every replay. max_norm: gradients are scaled down to that norm over
        all of them; norm: that norm where it is known already (gradient_norm's, or one over several ranks). Returns the norm, None without
        max_norm. Where it is not finite nothing changes. Parameters count as modified in place for autograd, as by torch's own optimizers (a replayed
        step cannot say so)."""
        pointers, codes = self._gradients(grads)
        self._in_place()
        rate, rate_ptr = self.lr, None
        if isinstance(lr, torch.Tensor):
            rate_ptr = self._scalar("lr", lr).data_ptr()
        elif lr is not None:
            rate = float(lr)
        if not (0 <= rate < math.inf):
            raise ValueError(f"lr must be a finite number that is not negative, not {rate}")
        space, given = None, norm is not None
        if max_norm is None:
            if given:
                raise ValueError("norm goes with max_norm")
        else:
            if not (0 < max_norm < math.inf):
                raise ValueError(f"max_norm must be a finite number above 0, not {max_norm}")
            if given:
                self._scalar("norm", norm)
            else:
                norm, space = torch.empty((), dtype=torch.float32, device=self._device), self._space()
        _check(_lib.tn_adamw_step(self._handle, pointers, codes, rate, rate_ptr, max_norm or 0.0, None if norm is None else norm.data_ptr(), int(given),
                                  None if space is None else space.data_ptr(), self._workspace_bytes, _stream(self._gpu)), "tn_adamw_step")
        increment_version(self.params)
        return norm

    def state_dict(self) -> Dict[str, torch.Tensor]:
        """The state's own tensors: first and second (over all parameters, each starting at a multiple of 128), count, master where a
        parameter is in bfloat16, first_scales and second_scales where the state is in 8 bits."""
        return dict(self._state)

    def load_state_dict(self, state: Dict[str, torch.Tensor]) -> None:
        """Copies a state of the same parameters and state_bits; parameters are loaded by whoever owns them. In 8 bits a root of v below what these
        betas allow beside its m is taken for a rounding (include/tn_adamw.h), also where the state is one of other betas."""
        if set(state) != set(self._state):
            raise ValueError(f"a state of this optimizer has {sorted(self._state)}, not {sorted(state)}")
        for key, t in self._state.items():
            if state[key].shape != t.shape or state[key].dtype != t.dtype:
                raise ValueError(f"{key} must be a {tuple(t.shape)} tensor of {t.dtype}, not {tuple(state[key].shape)} of {state[key].dtype}")
        for key, t in self._state.items():
            t.copy_(state[key])

    def close(self) -> None:
        if self._handle is not None:
            handle, self._handle = self._handle, None
            _check(_library().tn_adamw_destroy(handle), "tn_adamw_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _check_params(params: List[torch.Tensor]) -> int:
    if not params:
        raise ValueError("no parameters")
    for i, p in enumerate(params):
        if not (isinstance(p, torch.Tensor) and p.is_cuda and p.is_contiguous() and p.dtype in _DTYPE):
            raise ValueError(f"parameter {i} must be a contiguous CUDA tensor of float32 or bfloat16")
    gpu = _here("parameter 0", params[0].get_device())
    if any(p.get_device() != gpu for p in params):
        raise ValueError("parameters must be on one GPU")
    spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size(), i) for i, p in enumerate(params) if p.numel())
    for (_, end, i), (start, _, j) in zip(spans, spans[1:]):
        if start < end:
            raise ValueError(f"parameters {i} and {j} overlap")
    return gpu


def _check_numbers(n, lr, betas, eps, weight_decay, state_bits, seed) -> List[float]:
    if not 0 <= lr < math.inf:
        raise ValueError(f"lr must be a finite number that is not negative, not {lr}")
    if len(betas) != 2 or not all(0 <= b < 1 for b in betas):
        raise ValueError(f"betas must be two numbers from 0 up to 1, not {betas}")
    if not 0 <= eps < math.inf:
        raise ValueError(f"eps must be a finite number that is not negative, not {eps}")
    if state_bits not in (8, 32):
        raise ValueError(f"state_bits is 8 or 32, not {state_bits}")
    if not 0 <= seed < 2 ** 32:
        raise ValueError(f"seed must be a whole number below 2^32, not {seed}")
    decays = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
    if len(decays) != n or not all(0 <= d < math.inf for d in decays):
        raise ValueError("weight_decay must be a number that is not negative, or one for each parameter")
    return decays
