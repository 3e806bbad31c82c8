"""Python binding of the LR-QAT C ABI (include/lrqat.h).

Argument marshalling only: every step of the layer runs in the HIP library
liblrqat.so.  torch provides device memory (tensors) and the current stream.
The functions keep the C names; tensors must be contiguous and on the GPU.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from dataclasses import dataclass
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblrqat.so")

LRQAT_OK, LRQAT_EINVAL, LRQAT_EUNSUPPORTED, LRQAT_EWORKSPACE, LRQAT_EHIP = range(5)
PHI_FIXED_Q8, PHI_INT_PACKED2 = 0, 1
FP32, BF16 = 0, 1
_FMT = {"q8": PHI_FIXED_Q8, "int_packed2": PHI_INT_PACKED2}
_DT = {"fp32": FP32, "bf16": BF16}


class _Layer(ctypes.Structure):
    _fields_ = [("out_features", ctypes.c_int64), ("in_features", ctypes.c_int64),
                ("rank", ctypes.c_int32), ("alpha", ctypes.c_float), ("bits", ctypes.c_int32),
                ("phi_format", ctypes.c_int32), ("group_size", ctypes.c_int64),
                ("act_bits", ctypes.c_int32), ("act_dtype", ctypes.c_int32)]


class _ParamGroup(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p),
                ("exp_avg_sq", ctypes.c_void_p), ("n", ctypes.c_int64), ("lr_max", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]


class _AdamWConfig(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("max_grad_norm", ctypes.c_float), ("total_steps", ctypes.c_int64), ("warmup_steps", ctypes.c_int64)]


class _KVCache(ctypes.Structure):
    _fields_ = [("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("scale_tokens", ctypes.c_int32), ("pages", ctypes.c_int64), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class _KVBatch(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int32), ("table_width", ctypes.c_int32), ("tokens", ctypes.c_int64),
                ("first", ctypes.c_void_p), ("cached", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
                ("max_new", ctypes.c_int32), ("max_cached", ctypes.c_int32)]


class _StructSlot:
    # the C struct of a spec lies in a slot, not among the attributes that vars() and copies see
    __slots__ = ("_struct",)


@dataclass(frozen=True)
class LayerSpec(_StructSlot):
    """Hyper-parameters of one LR-QAT linear (mirrors the C struct lrqat_layer)."""
    out_features: int
    in_features: int
    rank: int
    alpha: float
    bits: int
    phi_format: str = "q8"        # "q8" or "int_packed2"
    group_size: int = 0
    act_bits: int = 0
    act_dtype: str = "bf16"       # "bf16" or "fp32"

    def c_struct(self) -> _Layer:
        return _Layer(self.out_features, self.in_features, self.rank, self.alpha, self.bits,
                      _FMT[self.phi_format], self.group_size, self.act_bits, _DT[self.act_dtype])

    @property
    def _c(self):
        # the fields are frozen, so one struct serves every call (the library only reads it)
        try:
            return self._struct
        except AttributeError:
            object.__setattr__(self, "_struct", self.c_struct())
            return self._struct

    def __getstate__(self):
        return dict(self.__dict__)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.act_dtype == "bf16" else torch.float32

    def scale_shape(self):
        m, k, g = self.out_features, self.in_features, self.group_size
        return (m,) if g == 0 else (m, k // g)

    def phi_shape(self):
        m, k = self.out_features, self.in_features
        return (m, k) if self.phi_format == "q8" else (m, k // 2)

    @property
    def phi_dtype(self):
        return torch.int8 if self.phi_format == "q8" else torch.uint8


class LRQATError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_lib().lrqat_status_string(status).decode()}: {message}")
        self.status = status


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2406_06385_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        P, I64, SZ, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.POINTER(_Layer)
        lib.lrqat_forward_workspace_size.argtypes = [F, I64]
        lib.lrqat_forward_workspace_size.restype = SZ
        lib.lrqat_backward_workspace_size.argtypes = [F, I64]
        lib.lrqat_backward_workspace_size.restype = SZ
        lib.lrqat_init_from_weights.argtypes = [F, P, P, P, P, P]
        lib.lrqat_infer_workspace_size.argtypes = [F, I64]
        lib.lrqat_infer_workspace_size.restype = SZ
        lib.lrqat_infer_forward.argtypes = [F, I64, P, P, P, P, P, P, SZ, P]
        lib.lrqat_forward.argtypes = [F, I64, P, P, P, P, P, P, P, P, SZ, P]
        lib.lrqat_backward.argtypes = [F, I64, P, P, P, P, P, P, P, P, P, P, P, ctypes.c_int, P, SZ, P]
        lib.lrqat_backward_static.argtypes = [F, I64, P, P, P, P, P, P, P, P, P, P, P, ctypes.c_int, P]
        lib.lrqat_backward_static_capacity.argtypes = []
        lib.lrqat_backward_static_capacity.restype = SZ
        lib.lrqat_merge_to_int4.argtypes = [F, P, P, P, P, P]
        for fn in ("lrqat_init_from_weights", "lrqat_forward", "lrqat_backward", "lrqat_backward_static",
                   "lrqat_merge_to_int4", "lrqat_infer_forward"):
            getattr(lib, fn).restype = ctypes.c_int
        lib.lrqat_init_lp.argtypes = [F, P, ctypes.c_float, ctypes.c_int, P, P, P]
        lib.lrqat_init_lp.restype = ctypes.c_int
        lib.lrqat_init_loftq_workspace_size.argtypes = [F]
        lib.lrqat_init_loftq_workspace_size.restype = SZ
        lib.lrqat_init_loftq.argtypes = [F, P, P, ctypes.c_int, P, P, P, P, P, SZ, P]
        lib.lrqat_init_loftq.restype = ctypes.c_int
        PG = ctypes.POINTER(_ParamGroup)
        lib.lrqat_adamw_workspace_size.argtypes = [ctypes.c_int, PG]
        lib.lrqat_adamw_workspace_size.restype = SZ
        lib.lrqat_adamw_step.argtypes = [ctypes.POINTER(_AdamWConfig), I64, ctypes.c_int, PG, P, P, SZ, P]
        lib.lrqat_adamw_step.restype = ctypes.c_int
        FL, I32 = ctypes.c_float, ctypes.c_int32
        lib.lrqat_infer_forward_codes.argtypes = [F, I64, P, P, P, P, P, P, P, P, SZ, P]
        lib.lrqat_infer_forward_codes.restype = ctypes.c_int
        lib.lrqat_rmsnorm_forward.argtypes = [I64, I64, I32, P, P, P, FL, P, P, P, P, P, P]
        lib.lrqat_rmsnorm_forward.restype = ctypes.c_int
        lib.lrqat_rmsnorm_backward_workspace_size.argtypes = [I64, I64]
        lib.lrqat_rmsnorm_backward_workspace_size.restype = SZ
        lib.lrqat_rmsnorm_backward.argtypes = [I64, I64, I32, P, P, FL, P, P, P, P, ctypes.c_int, P, SZ, P]
        lib.lrqat_rmsnorm_backward.restype = ctypes.c_int
        KC, KB = ctypes.POINTER(_KVCache), ctypes.POINTER(_KVBatch)
        for fn in ("lrqat_kv_write", "lrqat_kv_read"):
            getattr(lib, fn).argtypes = [KC, KB, I32, P, I64, P, I64, P]
            getattr(lib, fn).restype = ctypes.c_int
        lib.lrqat_kv_attention_workspace_size.argtypes = [KC, KB, I32]
        lib.lrqat_kv_attention_workspace_size.restype = SZ
        lib.lrqat_kv_attention.argtypes = [KC, KB, I32, I32, P, I64, FL, ctypes.c_int, P, I64, P, SZ, P]
        lib.lrqat_kv_attention.restype = ctypes.c_int
        lib.lrqat_status_string.argtypes = [ctypes.c_int]
        lib.lrqat_status_string.restype = ctypes.c_char_p
        lib.lrqat_last_error.restype = ctypes.c_char_p
        lib.lrqat_timing_enable.argtypes = [ctypes.c_int]
        lib.lrqat_timing_read.argtypes = [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(I64),
                                          ctypes.POINTER(ctypes.c_double), ctypes.c_int]
        lib.lrqat_timing_read.restype = ctypes.c_int
        _LIB = lib
    return _LIB


def load_library() -> str:
    """Load liblrqat.so (raises if it is missing) and return its path."""
    _lib()
    return LIB_PATH


def _check(status: int):
    if status != LRQAT_OK:
        raise LRQATError(status, _lib().lrqat_last_error().decode())


def _ptr(t):
    """Address of a tensor that _expect has passed (None: a null pointer)."""
    return None if t is None else t.data_ptr()


def _checked_ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors passed to the LR-QAT library must be contiguous GPU tensors")
    return t.data_ptr()


# the current stream's handle without a Stream object around it, and the current device without a check that the GPU is
# initialised (calls have tensors on it), where torch offers those
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(_raw_device())
    return torch.cuda.current_stream().cuda_stream


def _torch_stream(stream):
    return torch.cuda.current_stream() if stream is None else stream


def _on(stream):
    """Where a call makes the buffers that it is not given: on its stream.  (Entering the current stream again would
    take 9 us.)"""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


_Tensor = torch.Tensor


def _expect(t, shape, dtype, name, device=None):
    """Reject a tensor whose shape, dtype, layout or device the C ABI would
    misread (the library sees only a pointer)."""
    # one expression for the tensors that pass: a decoding step calls the library every few microseconds
    if (isinstance(t, _Tensor) and t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous()
            and (device is None or t.device == device)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name}: expected {tuple(shape)} {dtype}, got {tuple(t.shape)} {t.dtype}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: must be a contiguous GPU tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")


def _weights(spec: "LayerSpec", phi0, s, A, B, device, z=None):
    m, k, r = spec.out_features, spec.in_features, spec.rank
    _expect(phi0, spec.phi_shape(), spec.phi_dtype, "phi0", device)
    _expect(s, spec.scale_shape(), torch.float32, "s", device)
    if z is not None:
        _expect(z, spec.scale_shape(), torch.int32, "z", device)
    _expect(A, (m, r), torch.float32, "A", device)
    _expect(B, (r, k), torch.float32, "B", device)


def lrqat_forward_workspace_size(spec: LayerSpec, tokens: int) -> int:
    L = spec._c
    n = _lib().lrqat_forward_workspace_size(ctypes.byref(L), tokens)
    if n == 0:
        raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
    return n


def lrqat_backward_workspace_size(spec: LayerSpec, tokens: int) -> int:
    L = spec._c
    n = _lib().lrqat_backward_workspace_size(ctypes.byref(L), tokens)
    if n == 0:
        raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
    return n


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def lrqat_init_from_weights(spec: LayerSpec, W0: torch.Tensor, stream=None, asymmetric=False):
    """-> (s0 float32, Phi0) computed on the GPU from W0 [m][k] float32, or
    (s0, z0 int32, Phi0) with asymmetric=True (Phi0 then carries z0)."""
    _expect(W0, (spec.out_features, spec.in_features), torch.float32, "W0")
    st = _torch_stream(stream)
    with torch.cuda.stream(st):
        s0 = torch.empty(spec.scale_shape(), dtype=torch.float32, device=W0.device)
        z0 = torch.empty(spec.scale_shape(), dtype=torch.int32, device=W0.device) if asymmetric else None
        phi0 = torch.empty(spec.phi_shape(), dtype=spec.phi_dtype, device=W0.device)
    L = spec._c
    _check(_lib().lrqat_init_from_weights(ctypes.byref(L), _ptr(W0), _ptr(s0), _ptr(z0), _ptr(phi0), _stream(st)))
    return (s0, z0, phi0) if asymmetric else (s0, phi0)


def lrqat_init_lp(spec: LayerSpec, W0: torch.Tensor, p: float, n_grid: int = 100, stream=None):
    """-> (s0, Phi0) with s0 from the L^p-norm range search over n_grid clipping ratios."""
    _expect(W0, (spec.out_features, spec.in_features), torch.float32, "W0")
    st = _torch_stream(stream)
    with torch.cuda.stream(st):
        s0 = torch.empty(spec.scale_shape(), dtype=torch.float32, device=W0.device)
        phi0 = torch.empty(spec.phi_shape(), dtype=spec.phi_dtype, device=W0.device)
    L = spec._c
    _check(_lib().lrqat_init_lp(ctypes.byref(L), _ptr(W0), float(p), int(n_grid), _ptr(s0), _ptr(phi0), _stream(st)))
    return s0, phi0


def lrqat_init_loftq(spec: LayerSpec, W0: torch.Tensor, s0: torch.Tensor, n_iter: int = 32, stream=None):
    """-> (Phi0 packed INT-b, A, B, sigma) of the LoftQ (T = 1) initialisation for the given scale."""
    m, k, r = spec.out_features, spec.in_features, spec.rank
    _expect(W0, (m, k), torch.float32, "W0")
    dev = W0.device
    _expect(s0, spec.scale_shape(), torch.float32, "s0", dev)
    L = spec._c
    n = _lib().lrqat_init_loftq_workspace_size(ctypes.byref(L))
    if n == 0:
        raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
    st = _torch_stream(stream)
    with torch.cuda.stream(st):
        phi0 = torch.empty(spec.phi_shape(), dtype=spec.phi_dtype, device=dev)
        A = torch.empty((m, r), dtype=torch.float32, device=dev)
        B = torch.empty((r, k), dtype=torch.float32, device=dev)
        sigma = torch.empty(r, dtype=torch.float32, device=dev)
        ws = workspace(n, dev)
    _check(_lib().lrqat_init_loftq(ctypes.byref(L), _ptr(W0), _ptr(s0), int(n_iter), _ptr(phi0), _ptr(A), _ptr(B),
                                   _ptr(sigma), _ptr(ws), ws.numel(), _stream(st)))
    return phi0, A, B, sigma


def lrqat_forward(spec: LayerSpec, X, phi0, s, A, B, Y=None, ws=None, stream=None, z=None):
    """Y = X_hat W_hat^T.  X [T][k] in the layer's activation dtype; z (int32,
    shaped like s) is the zero offset of asymmetric quantisation."""
    T = X.shape[0] if X.dim() == 2 else -1
    _expect(X, (T, spec.in_features), spec.torch_dtype, "X")
    dev = X.device
    _weights(spec, phi0, s, A, B, dev, z)
    if Y is None or ws is None:
        with torch.cuda.stream(_torch_stream(stream)):  # buffers made here belong to the stream the kernels run on
            if Y is None:
                Y = torch.empty((T, spec.out_features), dtype=spec.torch_dtype, device=dev)
            if ws is None:
                ws = workspace(lrqat_forward_workspace_size(spec, T), dev)
    _expect(Y, (T, spec.out_features), spec.torch_dtype, "Y", dev)
    _expect(ws, (ws.numel(),), torch.uint8, "ws", dev)
    L = spec._c
    _check(_lib().lrqat_forward(ctypes.byref(L), T, _ptr(X), _ptr(phi0), _ptr(s), _ptr(z), _ptr(A), _ptr(B),
                                _ptr(Y), _ptr(ws), ws.numel(), _stream(stream)))
    return Y


def _backward_args(spec, X, phi0, s, A, B, dY, dX, dA, dB, want_dx, ds, want_ds, z, stream):
    T = X.shape[0] if X.dim() == 2 else -1
    m, k, r = spec.out_features, spec.in_features, spec.rank
    _expect(X, (T, k), spec.torch_dtype, "X")
    dev = X.device
    _weights(spec, phi0, s, A, B, dev, z)
    _expect(dY, (T, m), spec.torch_dtype, "dY", dev)
    if dA is None or dB is None or (dX is None and want_dx) or (ds is None and want_ds):
        with torch.cuda.stream(_torch_stream(stream)):  # buffers made here belong to the stream the kernels run on
            if dX is None and want_dx:
                dX = torch.empty((T, k), dtype=spec.torch_dtype, device=dev)
            if dA is None:
                dA = torch.empty((m, r), dtype=torch.float32, device=dev)
            if dB is None:
                dB = torch.empty((r, k), dtype=torch.float32, device=dev)
            if ds is None and want_ds:
                ds = torch.empty(spec.scale_shape(), dtype=torch.float32, device=dev)
    if dX is not None:
        _expect(dX, (T, k), spec.torch_dtype, "dX", dev)
    _expect(dA, (m, r), torch.float32, "dA", dev)
    _expect(dB, (r, k), torch.float32, "dB", dev)
    if ds is not None:
        _expect(ds, spec.scale_shape(), torch.float32, "ds", dev)
    return T, dev, dX, dA, dB, ds


def lrqat_backward(spec: LayerSpec, X, phi0, s, A, B, dY, dX=None, dA=None, dB=None, want_dx=True,
                   accumulate=False, ws=None, stream=None, z=None, ds=None, want_ds=False):
    """-> (dX or None, dA, dB) with the straight-through estimator; W_hat is
    recomputed.  With want_ds (or a ds tensor) -> (dX, dA, dB, ds)."""
    T, dev, dX, dA, dB, ds = _backward_args(spec, X, phi0, s, A, B, dY, dX, dA, dB, want_dx, ds, want_ds, z, stream)
    if ws is None:
        with torch.cuda.stream(_torch_stream(stream)):
            ws = workspace(lrqat_backward_workspace_size(spec, T), dev)
    _expect(ws, (ws.numel(),), torch.uint8, "ws", dev)
    L = spec._c
    _check(_lib().lrqat_backward(ctypes.byref(L), T, _ptr(X), _ptr(phi0), _ptr(s), _ptr(z), _ptr(A), _ptr(B),
                                 _ptr(dY), _ptr(dX), _ptr(dA), _ptr(dB), _ptr(ds), int(bool(accumulate)), _ptr(ws),
                                 ws.numel(), _stream(stream)))
    return (dX, dA, dB, ds) if ds is not None else (dX, dA, dB)


def lrqat_backward_static(spec: LayerSpec, X, phi0, s, A, B, dY, dX, dA, dB, accumulate=False, stream=None,
                          z=None, ds=None):
    """lrqat_backward on the library's device-resident scratch array: every
    output tensor is the caller's, nothing is allocated."""
    T, dev, dX, dA, dB, ds = _backward_args(spec, X, phi0, s, A, B, dY, dX, dA, dB, dX is not None, ds, False, z, stream)
    L = spec._c
    _check(_lib().lrqat_backward_static(ctypes.byref(L), T, _ptr(X), _ptr(phi0), _ptr(s), _ptr(z), _ptr(A),
                                        _ptr(B), _ptr(dY), _ptr(dX), _ptr(dA), _ptr(dB), _ptr(ds),
                                        int(bool(accumulate)), _stream(stream)))
    return (dX, dA, dB, ds) if ds is not None else (dX, dA, dB)


def lrqat_backward_static_capacity() -> int:
    return int(_lib().lrqat_backward_static_capacity())


def lrqat_merge_to_int4(spec: LayerSpec, phi0, A, B, out=None, stream=None):
    """W_Z = clip(round(Phi0 + (alpha/r) A B)) double-packed, uint8 [m][k/2]."""
    m, k, r = spec.out_features, spec.in_features, spec.rank
    dev = A.device
    _expect(phi0, spec.phi_shape(), spec.phi_dtype, "phi0", dev)
    _expect(A, (m, r), torch.float32, "A", dev)
    _expect(B, (r, k), torch.float32, "B", dev)
    if out is None:
        with torch.cuda.stream(_torch_stream(stream)):
            out = torch.empty((m, k // 2), dtype=torch.uint8, device=dev)
    _expect(out, (m, k // 2), torch.uint8, "out", dev)
    L = spec._c
    _check(_lib().lrqat_merge_to_int4(ctypes.byref(L), _ptr(phi0), _ptr(A), _ptr(B), _ptr(out), _stream(stream)))
    return out


def lrqat_infer_workspace_size(spec: LayerSpec, tokens: int) -> int:
    L = spec._c
    n = _lib().lrqat_infer_workspace_size(ctypes.byref(L), tokens)
    if n == 0:
        raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
    return n


def lrqat_infer_forward(spec: LayerSpec, X, W_int4, s, z=None, Y=None, ws=None, stream=None):
    """Y = X_hat (s (W_Z - z))^T on the merged packed int4 weights uint8 [m][k/2]."""
    T = X.shape[0] if X.dim() == 2 else -1
    m, k = spec.out_features, spec.in_features
    _expect(X, (T, k), spec.torch_dtype, "X")
    dev = X.device
    _expect(W_int4, (m, k // 2), torch.uint8, "W_int4", dev)
    _expect(s, spec.scale_shape(), torch.float32, "s", dev)
    if z is not None:
        _expect(z, spec.scale_shape(), torch.int32, "z", dev)
    if Y is None or ws is None:
        with torch.cuda.stream(_torch_stream(stream)):
            if Y is None:
                Y = torch.empty((T, m), dtype=spec.torch_dtype, device=dev)
            if ws is None:
                ws = workspace(lrqat_infer_workspace_size(spec, T), dev)
    _expect(Y, (T, m), spec.torch_dtype, "Y", dev)
    _expect(ws, (ws.numel(),), torch.uint8, "ws", dev)
    L = spec._c
    _check(_lib().lrqat_infer_forward(ctypes.byref(L), T, _ptr(X), _ptr(W_int4), _ptr(s), _ptr(z), _ptr(Y),
                                      _ptr(ws), ws.numel(), _stream(stream)))
    return Y


class Int8Tokens(NamedTuple):
    """Activations as int8 codes: X_hat = sx codes, as the W4A8 projections take them."""
    codes: torch.Tensor            # int8 [T][k rounded up to 256], columns past k are 0
    sx: torch.Tensor               # float32 [T]
    nsum: Optional[torch.Tensor]   # int32 [T], the sum of each token's codes


def int8_tokens(tokens: int, width: int, device="cuda") -> Int8Tokens:
    """Buffers for the codes of [tokens][width] activations."""
    return Int8Tokens(torch.empty((tokens, -(-width // 256) * 256), dtype=torch.int8, device=device),
                      torch.empty(tokens, dtype=torch.float32, device=device),
                      torch.empty(tokens, dtype=torch.int32, device=device))


def _expect_codes(q: Int8Tokens, tokens, width, device):
    _expect(q.codes, (tokens, -(-width // 256) * 256), torch.int8, "codes", device)
    _expect(q.sx, (tokens,), torch.float32, "sx", device)
    if q.nsum is not None:
        _expect(q.nsum, (tokens,), torch.int32, "nsum", device)


def lrqat_infer_forward_codes(spec: LayerSpec, X: Int8Tokens, W_int4, s, z=None, Y=None, ws=None, stream=None):
    """lrqat_infer_forward of a W4A8 layer on activations that are int8 codes already (lrqat_rmsnorm_forward)."""
    T = X.codes.shape[0] if X.codes.dim() == 2 else -1
    m, k = spec.out_features, spec.in_features
    dev = X.codes.device
    _expect_codes(X, T, k, dev)
    _expect(W_int4, (m, k // 2), torch.uint8, "W_int4", dev)
    _expect(s, spec.scale_shape(), torch.float32, "s", dev)
    if z is not None:
        _expect(z, spec.scale_shape(), torch.int32, "z", dev)
    if Y is None or ws is None:
        with _on(stream):
            if Y is None:
                Y = torch.empty((T, m), dtype=spec.torch_dtype, device=dev)
            if ws is None:
                ws = workspace(lrqat_infer_workspace_size(spec, T), dev)
    _expect(Y, (T, m), spec.torch_dtype, "Y", dev)
    _expect(ws, (ws.numel(),), torch.uint8, "ws", dev)
    L = spec._c
    _check(_lib().lrqat_infer_forward_codes(ctypes.byref(L), T, _ptr(X.codes), _ptr(X.sx), _ptr(X.nsum), _ptr(W_int4),
                                            _ptr(s), _ptr(z), _ptr(Y), _ptr(ws), ws.numel(), _stream(stream)))
    return Y


_ACT = {torch.float32: FP32, torch.bfloat16: BF16}


def _act(t, name):
    """lrqat_dtype of a [tokens][width] activation tensor."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dim() != 2 or t.dtype not in _ACT:
        raise ValueError(f"{name}: expected [tokens][width] in bfloat16 or float32, got {tuple(t.shape)} {t.dtype}")
    return _ACT[t.dtype]


def lrqat_rmsnorm_forward(X, gain, eps=1e-5, R=None, H=None, Y=None, codes: Optional[Int8Tokens] = None, stream=None):
    """-> (H, Y, codes): h = X + R and y = gain h / sqrt(mean(h^2) + eps), as H (where there is a residual R or a
    tensor for it), as Y, or as int8 codes (buffers of int8_tokens).  Y is made when neither Y nor codes is given."""
    act = _act(X, "X")
    dev, shape = X.device, X.shape
    _expect(X, shape, X.dtype, "X")
    _expect(gain, (shape[1],), torch.float32, "gain", dev)
    if (H is None and R is not None) or (Y is None and codes is None):
        with _on(stream):
            if H is None and R is not None:
                H = torch.empty_like(X)
            if Y is None and codes is None:
                Y = torch.empty_like(X)
    for t, name in ((R, "R"), (H, "H"), (Y, "Y")):
        if t is not None:
            _expect(t, shape, X.dtype, name, dev)
    q = (None, None, None)
    if codes is not None:
        _expect_codes(codes, shape[0], shape[1], dev)
        q = (codes.codes.data_ptr(), codes.sx.data_ptr(), _ptr(codes.nsum))
    _check(_lib().lrqat_rmsnorm_forward(shape[0], shape[1], act, X.data_ptr(), _ptr(R), gain.data_ptr(), eps, _ptr(H),
                                        _ptr(Y), *q, _stream(stream)))
    return H, Y, codes


def lrqat_rmsnorm_backward_workspace_size(tokens: int, width: int) -> int:
    n = _lib().lrqat_rmsnorm_backward_workspace_size(tokens, width)
    if n == 0:
        raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
    return n


def lrqat_rmsnorm_backward(H, gain, eps, dY, dH=None, dX=None, dgain=None, want_dgain=True, accumulate=False, ws=None,
                           stream=None):
    """-> (dX, dgain or None) at the stream H that the forward stored; dH is the gradient that reaches it past the norm."""
    act = _act(H, "H")
    dev, shape = H.device, H.shape
    _expect(H, shape, H.dtype, "H")
    _expect(gain, (shape[1],), torch.float32, "gain", dev)
    _expect(dY, shape, H.dtype, "dY", dev)
    if dH is not None:
        _expect(dH, shape, H.dtype, "dH", dev)
    if dgain is not None:
        want_dgain = True
    if dX is None or (want_dgain and (dgain is None or ws is None)):
        with _on(stream):
            if dX is None:
                dX = torch.empty_like(H)
            if want_dgain and dgain is None:
                if accumulate:
                    raise ValueError("accumulate needs the dgain to add into")
                dgain = torch.empty_like(gain)
            if want_dgain and ws is None:
                ws = workspace(lrqat_rmsnorm_backward_workspace_size(*shape), dev)
    _expect(dX, shape, H.dtype, "dX", dev)
    if dgain is not None:
        _expect(dgain, (shape[1],), torch.float32, "dgain", dev)
    if ws is not None:
        _expect(ws, (ws.numel(),), torch.uint8, "ws", dev)
    _check(_lib().lrqat_rmsnorm_backward(shape[0], shape[1], act, H.data_ptr(), gain.data_ptr(), eps, dY.data_ptr(),
                                         _ptr(dH), dX.data_ptr(), _ptr(dgain), int(bool(accumulate)), _ptr(ws),
                                         0 if ws is None else ws.numel(), _stream(stream)))
    return dX, dgain


@dataclass(frozen=True)
class KVCacheSpec:
    """Sizes of a paged int8 KV cache (one layer's)."""
    kv_heads: int
    head_dim: int             # a multiple of 16, up to 256
    pages: int
    page_tokens: int = 64     # a power of two, 16 .. 256
    scale_tokens: int = 1     # tokens that share a scale: 1, or a power of two from 16 to page_tokens

    def code_shape(self):
        return (self.pages, self.kv_heads, self.page_tokens, self.head_dim)

    def scale_shape(self):
        return (self.pages, self.kv_heads, self.page_tokens // self.scale_tokens)


@dataclass(frozen=True, eq=False)
class KVCache(_StructSlot):
    """The cache's memory: codes int8 of spec.code_shape(), scales float32 of spec.scale_shape()."""
    spec: KVCacheSpec
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    def __post_init__(self):
        sp = self.spec
        if sp.scale_tokens < 1 or sp.page_tokens < 1:
            raise ValueError("page_tokens and scale_tokens must be at least 1")
        _expect(self.k, sp.code_shape(), torch.int8, "k")
        dev = self.k.device
        _expect(self.v, sp.code_shape(), torch.int8, "v", dev)
        _expect(self.k_scale, sp.scale_shape(), torch.float32, "k_scale", dev)
        _expect(self.v_scale, sp.scale_shape(), torch.float32, "v_scale", dev)

    @property
    def _ref(self):
        """The C struct's address.  The struct is made once, and again where a tensor's memory has been exchanged since
        (by set_(), by .data, by a resize_() that moved it): its sizes may have gone with it, so they are checked too."""
        at = (self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr())
        try:
            ref, was = self._struct
            if was == at:
                return ref
        except AttributeError:
            pass
        self.__post_init__()
        sp = self.spec
        ref = ctypes.byref(_KVCache(sp.kv_heads, sp.head_dim, sp.page_tokens, sp.scale_tokens, sp.pages, *at))
        object.__setattr__(self, "_struct", (ref, at))
        return ref

    def __getstate__(self):
        return dict(self.__dict__)


def lrqat_kv_cache(spec: KVCacheSpec, device="cuda") -> KVCache:
    """A cache of that many pages; its memory needs no start value."""
    code = lambda: torch.empty(spec.code_shape(), dtype=torch.int8, device=device)  # noqa: E731
    scale = lambda: torch.empty(spec.scale_shape(), dtype=torch.float32, device=device)  # noqa: E731
    return KVCache(spec, code(), code(), scale(), scale())


@dataclass(frozen=True, eq=False)
class KVBatch(_StructSlot):
    """The tokens of one step: sequence i has rows first[i] .. first[i + 1] - 1 of the step's tensors, at the positions
    that follow its cached[i] earlier tokens; page_table[i] lists the pages of its positions.  One batch serves every
    layer's calls of a step.  max_new and max_cached bound the sequences' new and cached tokens: new tokens past max_new are
    left out; more cached ones than max_cached are attended, only slower."""
    first: torch.Tensor        # int32 [sequences + 1]
    cached: torch.Tensor       # int32 [sequences]
    page_table: torch.Tensor   # int32 [sequences][width]
    tokens: int
    max_new: int
    max_cached: int

    def __post_init__(self):
        _expect(self.first, (self.first.numel(),), torch.int32, "first")
        dev, n = self.first.device, self.first.numel() - 1
        if n < 0:
            raise ValueError("first: expected sequences + 1 entries")
        _expect(self.cached, (n,), torch.int32, "cached", dev)
        _expect(self.page_table, (n, self.page_table.shape[-1] if self.page_table.dim() else 0), torch.int32, "page_table",
                dev)

    @property
    def _ref(self):
        """As a cache's."""
        at = (self.first.data_ptr(), self.cached.data_ptr(), self.page_table.data_ptr())
        try:
            ref, was = self._struct
            if was == at:
                return ref
        except AttributeError:
            pass
        self.__post_init__()
        ref = ctypes.byref(_KVBatch(self.cached.numel(), self.page_table.shape[1], self.tokens, *at, self.max_new,
                                    self.max_cached))
        object.__setattr__(self, "_struct", (ref, at))
        return ref

    def __getstate__(self):
        return dict(self.__dict__)


def _rows(t, tokens, heads, d, dtypes, name, device):
    """[tokens][heads][d] with dense heads and any distance between tokens (columns of a fused projection) -> that
    distance in elements."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.shape != (tokens, heads, d) or t.dtype not in dtypes:
        raise ValueError(f"{name}: expected {(tokens, heads, d)} in {' or '.join(str(x) for x in dtypes)}, got "
                         f"{tuple(t.shape)} {t.dtype}")
    s = t.stride()
    if (s[2] != 1 or (heads > 1 and s[1] != d)) and t.numel():
        raise ValueError(f"{name}: the heads of a token must be dense (strides {s})")
    if t.device != device:  # (the cache's, which is a GPU)
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    return s[0] if tokens > 1 else heads * d


def _kv_pair(cache, batch, K, V):
    sp, dev = cache.spec, cache.k.device
    if batch.first.device != dev:
        raise ValueError(f"batch: on {batch.first.device}, expected {dev}")
    ks = _rows(K, batch.tokens, sp.kv_heads, sp.head_dim, _ACT, "K", dev)
    vs = _rows(V, batch.tokens, sp.kv_heads, sp.head_dim, (K.dtype,), "V", dev)
    return K.data_ptr(), ks, V.data_ptr(), vs


def lrqat_kv_write(cache: KVCache, batch: KVBatch, K, V, stream=None):
    """Quantise the batch's K and V [tokens][kv_heads][head_dim] into the cache.  Tokens may lie any multiple of 16
    bytes apart (columns of a fused projection)."""
    pair = _kv_pair(cache, batch, K, V)
    _check(_lib().lrqat_kv_write(cache._ref, batch._ref, _ACT[K.dtype], *pair,
                                 _stream(stream)))


def lrqat_kv_read(cache: KVCache, batch: KVBatch, K=None, V=None, dtype=torch.bfloat16, stream=None):
    """-> (K, V) [tokens][kv_heads][head_dim] of the batch's positions, as the cache holds them."""
    if K is None or V is None:
        shape = (batch.tokens, cache.spec.kv_heads, cache.spec.head_dim)
        like = K if K is not None else V
        dt = dtype if like is None else like.dtype
        with _on(stream):
            K = torch.empty(shape, dtype=dt, device=cache.k.device) if K is None else K
            V = torch.empty(shape, dtype=dt, device=cache.k.device) if V is None else V
    pair = _kv_pair(cache, batch, K, V)
    _check(_lib().lrqat_kv_read(cache._ref, batch._ref, _ACT[K.dtype], *pair, _stream(stream)))
    return K, V


def lrqat_kv_attention_workspace_size(cache: KVCache, batch: KVBatch, q_heads: int) -> int:
    n = _lib().lrqat_kv_attention_workspace_size(cache._ref, batch._ref, q_heads)
    if n == 0:
        raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
    return n


def lrqat_kv_attention(cache: KVCache, batch: KVBatch, Q, scale=None, causal=True, O=None, ws=None, stream=None):
    """O [tokens][q_heads][head_dim] (bfloat16) of the batch's queries over the cache, which holds their own keys and
    values already.  Q's tokens may lie any multiple of 16 bytes apart.  scale: head_dim ** -0.5 by default."""
    sp, dev = cache.spec, cache.k.device
    if batch.first.device != dev:
        raise ValueError(f"batch: on {batch.first.device}, expected {dev}")
    heads = Q.shape[1] if isinstance(Q, _Tensor) and Q.dim() == 3 else 0
    qs = _rows(Q, batch.tokens, heads, sp.head_dim, (torch.bfloat16,), "Q", dev)
    if O is None or ws is None:
        with _on(stream):
            if O is None:
                O = torch.empty(Q.shape, dtype=Q.dtype, device=dev)
            if ws is None:
                ws = workspace(lrqat_kv_attention_workspace_size(cache, batch, heads), dev)
    os_ = _rows(O, batch.tokens, heads, sp.head_dim, (torch.bfloat16,), "O", dev)
    _expect(ws, (ws.numel(),), torch.uint8, "ws", dev)
    _check(_lib().lrqat_kv_attention(cache._ref, batch._ref, heads, BF16, Q.data_ptr(), qs,
                                     sp.head_dim ** -0.5 if scale is None else scale, int(bool(causal)), O.data_ptr(),
                                     os_, ws.data_ptr(), ws.numel(), _stream(stream)))
    return O


def _groups(groups):
    arr = (_ParamGroup * max(1, len(groups)))()
    dev = None
    for i, g in enumerate(groups):
        p = g["param"]
        dev = dev or p.device
        n = p.numel()
        for key in ("param", "grad", "exp_avg", "exp_avg_sq"):
            _expect(g[key], tuple(p.shape), torch.float32, key, dev)
        arr[i] = _ParamGroup(g["param"].data_ptr(), g["grad"].data_ptr(), g["exp_avg"].data_ptr(),
                             g["exp_avg_sq"].data_ptr(), n, float(g["lr_max"]), float(g.get("weight_decay", 0.0)))
    return arr, dev


def lrqat_adamw_step(groups, step, total_steps, warmup_steps, beta1=0.9, beta2=0.95, eps=1e-8, max_grad_norm=1.0,
                     grad_norm=None, ws=None, stream=None):
    """AdamW with global L2 clipping and the linear warm-up/decay schedule, in place.
    groups: list of dicts with float32 tensors param, grad, exp_avg, exp_avg_sq (same
    shape) and floats lr_max, weight_decay.  grad_norm: optional float32 [1] tensor
    receiving the norm before clipping."""
    arr, dev = _groups(groups)
    cfg = _AdamWConfig(beta1, beta2, eps, max_grad_norm, int(total_steps), int(warmup_steps))
    if ws is None:
        n = _lib().lrqat_adamw_workspace_size(len(groups), arr)
        if n == 0:
            raise LRQATError(LRQAT_EINVAL, _lib().lrqat_last_error().decode())
        with torch.cuda.stream(_torch_stream(stream)):
            ws = workspace(n, dev or "cuda")
    if grad_norm is not None:
        _expect(grad_norm, (1,), torch.float32, "grad_norm", dev)
    _check(_lib().lrqat_adamw_step(ctypes.byref(cfg), int(step), len(groups), arr, _ptr(grad_norm), _checked_ptr(ws),
                                   ws.numel(), _stream(stream)))


def lrqat_timing_enable(on: bool = True):
    _lib().lrqat_timing_enable(int(bool(on)))


def lrqat_timing_reset():
    _lib().lrqat_timing_reset()


def lrqat_timing_read() -> dict:
    """{kernel name: (launches, total milliseconds)} since the last reset."""
    n = 32
    names = (ctypes.c_char_p * n)()
    launches = (ctypes.c_int64 * n)()
    ms = (ctypes.c_double * n)()
    cnt = _lib().lrqat_timing_read(names, launches, ms, n)
    if cnt < 0:
        raise LRQATError(LRQAT_EHIP, "timing read failed")
    return {names[i].decode(): (int(launches[i]), float(ms[i])) for i in range(cnt)}
