"""ctypes binding of the learner-side operators of libscalecom.so: argument marshalling only.

Every method mirrors the C entry point of the same name in include/scalecom_operators.h; torch is used for device memory
and streams, nothing is computed here.  Outputs are written into tensors that the caller provides.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import binding
from .binding import OK, ScaleComError

F32, F16, BF16 = 0, 1, 2
ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2, 3
OPS_MAX_DIM = 1 << 26
ACTIVATIONS = {"silu": ACT_SILU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "relu": ACT_RELU}
TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}

EXPORTS = (
    "scalecom_ops_create", "scalecom_ops_destroy", "scalecom_ops_set_stream", "scalecom_ops_reserve", "scalecom_ops_workspace",
    "scalecom_ops_status", "scalecom_ops_reset", "scalecom_layer_norm", "scalecom_layer_norm_backward", "scalecom_gated_ffn",
    "scalecom_gated_ffn_backward", "scalecom_orthogonalise",
)

_lib = None


def lib() -> ctypes.CDLL:
    """The compiled library with these entry points declared.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        declare = {
            "scalecom_ops_create": [ctypes.POINTER(vp)],
            "scalecom_ops_set_stream": [vp, vp],
            "scalecom_ops_reserve": [vp, i64],
            "scalecom_ops_workspace": [vp, ctypes.POINTER(i64)],
            "scalecom_ops_status": [vp],
            "scalecom_ops_reset": [vp],
            "scalecom_layer_norm": [vp, i32, i64, i64, vp, i64, vp, vp, f32, vp, i64, vp, vp],
            "scalecom_layer_norm_backward": [vp, i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp],
            "scalecom_gated_ffn": [vp, i32, i32, i64, i64, i64, vp, i64, vp, vp, vp, vp, i64, vp],
            "scalecom_gated_ffn_backward": [vp, i32, i32, i32, i64, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp],
            "scalecom_orthogonalise": [vp, i64, i64, i64, i32, vp, i64, i64, i32, vp, i64, i64, i32, vp, i32, f32, f32],
        }
        for name, args in declare.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = ctypes.c_int, args
        L.scalecom_ops_destroy.restype, L.scalecom_ops_destroy.argtypes = None, [vp]
        _lib = L
    return _lib


def _check(rc: int, where: str) -> None:
    if rc != OK:
        raise ScaleComError(rc, where)


# dev: the index of the handle's device. A kernel reads what it is given from there, so a tensor of another device (or of the host)
# is refused here; get_device() is -1 for the host's.
def _type(dev: int, t: torch.Tensor, name: str) -> int:
    kind = TYPES.get(t.dtype)
    if kind is None or t.get_device() != dev:
        raise TypeError("%s must be a tensor of float32, float16 or bfloat16 on the handle's device cuda:%s" % (name, dev))
    return kind


def _matrix(dev: int, t: torch.Tensor, kind: torch.dtype, shape: torch.Size, name: str) -> int:
    """Row distance of a matrix whose rows are contiguous (a slice of longer rows is fine)."""
    if t.dtype is not kind or t.get_device() != dev:
        raise TypeError("%s must be a tensor of %s on the handle's device cuda:%s" % (name, kind, dev))
    if t.shape != shape or len(shape) != 2:
        raise ValueError("%s must be of shape %s" % (name, tuple(shape)))
    s0, s1 = t.stride()
    rows, cols = shape
    if (s1 != 1 and cols > 1) or (s0 < cols and rows > 1):
        raise ValueError("%s must have contiguous rows" % name)
    return s0 if s0 >= cols else cols


def _vector(dev: int, t: Optional[torch.Tensor], n: int, name: str) -> Optional[int]:
    if t is None:
        return None
    if not (t.get_device() == dev and t.dtype is torch.float32 and t.numel() == n and t.is_contiguous()):
        raise TypeError("%s must be a contiguous float32 tensor of %d elements on the handle's device cuda:%s" % (name, n, dev))
    return t.data_ptr()


def _whole(dev: int, t: Optional[torch.Tensor], kinds: Sequence[torch.dtype], shape, name: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype not in kinds or t.get_device() != dev or not t.is_contiguous():
        raise TypeError("%s must be a contiguous tensor of %s on the handle's device cuda:%s" % (name, " or ".join(map(str, kinds)), dev))
    if t.shape != shape:
        raise ValueError("%s must be of shape %s" % (name, shape))
    return t.data_ptr()


class Operators:
    """One operator handle on the current device: a stream binding and scratch.  Inputs and outputs belong to the caller.

    Tensors have to be on the handle's device.  Calls run on the stream that the handle is bound to -- by default the legacy default
    stream, which is also torch's default one -- and not on the stream that is current where they are made: inside
    `with torch.cuda.stream(s)` bind the handle to s, or order the two streams with events."""

    _device: Optional[int] = None

    def __init__(self, stream: Optional[torch.cuda.Stream] = None):
        h, L = ctypes.c_void_p(), lib()
        _check(L.scalecom_ops_create(ctypes.byref(h)), "scalecom_ops_create")
        self._h = h.value
        self._device = torch.cuda.current_device()
        # looked up once: a small call's time is its way through here
        self._layer_norm, self._layer_norm_backward = L.scalecom_layer_norm, L.scalecom_layer_norm_backward
        self._gated_ffn, self._gated_ffn_backward = L.scalecom_gated_ffn, L.scalecom_gated_ffn_backward
        self._orthogonalise = L.scalecom_orthogonalise
        if stream is not None:
            self.set_stream(stream)

    def close(self) -> None:
        if getattr(self, "_h", None):
            h, self._h = self._h, None
            if _lib is not None:                 # at interpreter exit the module globals may already be gone
                _lib.scalecom_ops_destroy(h)

    __del__ = close

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def set_stream(self, stream: Optional[torch.cuda.Stream]) -> None:
        _check(lib().scalecom_ops_set_stream(self._h, stream.cuda_stream if stream is not None else None), "scalecom_ops_set_stream")

    def reserve(self, nbytes: int) -> None:
        """Make the scratch at least so large now, so that no later call has to wait and allocate."""
        _check(lib().scalecom_ops_reserve(self._h, int(nbytes)), "scalecom_ops_reserve")

    def workspace(self) -> int:
        out = ctypes.c_int64()
        _check(lib().scalecom_ops_workspace(self._h, ctypes.byref(out)), "scalecom_ops_workspace")
        return out.value

    def status(self) -> int:
        return lib().scalecom_ops_status(self._h)

    def reset(self) -> None:
        _check(lib().scalecom_ops_reset(self._h), "scalecom_ops_reset")

    def layer_norm(self, x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], eps: float, y: torch.Tensor,
                   mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None) -> None:
        """y = (x - mean) * rstd * gamma + beta over the last dimension of the matrix x."""
        dev, kind, shape = self._device, x.dtype, x.shape
        code = _type(dev, x, "x")
        rows, width = shape
        _check(self._layer_norm(self._h, code, rows, width, x.data_ptr(), _matrix(dev, x, kind, shape, "x"),
                                         _vector(dev, gamma, width, "gamma"), _vector(dev, beta, width, "beta"), eps,
                                         y.data_ptr(), _matrix(dev, y, kind, shape, "y"),
                                         _vector(dev, mean, rows, "mean"), _vector(dev, rstd, rows, "rstd")), "scalecom_layer_norm")

    def layer_norm_backward(self, dy: torch.Tensor, x: torch.Tensor, gamma: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                            dx: Optional[torch.Tensor] = None, dgamma: Optional[torch.Tensor] = None,
                            dbeta: Optional[torch.Tensor] = None) -> None:
        """dx, and the gradients of gamma and beta (written, not added to)."""
        dev, kind, shape = self._device, x.dtype, x.shape
        code = _type(dev, x, "x")
        rows, width = shape
        _check(self._layer_norm_backward(
            self._h, code, rows, width, dy.data_ptr(), _matrix(dev, dy, kind, shape, "dy"),
            x.data_ptr(), _matrix(dev, x, kind, shape, "x"), _vector(dev, gamma, width, "gamma"),
            _vector(dev, mean, rows, "mean"), _vector(dev, rstd, rows, "rstd"),
            None if dx is None else dx.data_ptr(), width if dx is None else _matrix(dev, dx, kind, shape, "dx"),
            _vector(dev, dgamma, width, "dgamma"), _vector(dev, dbeta, width, "dbeta")), "scalecom_layer_norm_backward")

    def gated_ffn(self, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, y: torch.Tensor,
                  saved: Optional[torch.Tensor] = None, activation: str = "silu") -> None:
        """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; saved [2, tokens, hidden] keeps what the backward pass needs."""
        dev, kind, shape = self._device, x.dtype, x.shape
        code = _type(dev, x, "x")
        (tokens, width), hidden, k = shape, w_gate.shape[0], (kind,)
        _check(self._gated_ffn(
            self._h, code, ACTIVATIONS[activation], tokens, width, hidden, x.data_ptr(), _matrix(dev, x, kind, shape, "x"),
            _whole(dev, w_gate, k, (hidden, width), "w_gate"), _whole(dev, w_up, k, (hidden, width), "w_up"),
            _whole(dev, w_down, k, (width, hidden), "w_down"), y.data_ptr(), _matrix(dev, y, kind, shape, "y"),
            _whole(dev, saved, k, (2, tokens, hidden), "saved")), "scalecom_gated_ffn")

    def gated_ffn_backward(self, dy: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                           saved: torch.Tensor, dx: Optional[torch.Tensor] = None, dw_gate: Optional[torch.Tensor] = None,
                           dw_up: Optional[torch.Tensor] = None, dw_down: Optional[torch.Tensor] = None,
                           activation: str = "silu") -> None:
        """Gradients of the block (written, not added to); the weights' may be float32 whatever the type of x."""
        dev, kind, shape = self._device, x.dtype, x.shape
        code = _type(dev, x, "x")
        (tokens, width), hidden, k = shape, w_gate.shape[0], (kind,)
        grads = [g for g in (dw_gate, dw_up, dw_down) if g is not None]
        gk = (grads[0].dtype if grads else kind,)
        if gk[0] not in (kind, torch.float32):
            raise TypeError("weight gradients must be of x's type or float32")
        _check(self._gated_ffn_backward(
            self._h, code, TYPES[gk[0]], ACTIVATIONS[activation], tokens, width, hidden,
            dy.data_ptr(), _matrix(dev, dy, kind, shape, "dy"), x.data_ptr(), _matrix(dev, x, kind, shape, "x"),
            _whole(dev, w_gate, k, (hidden, width), "w_gate"), _whole(dev, w_up, k, (hidden, width), "w_up"),
            _whole(dev, w_down, k, (width, hidden), "w_down"), _whole(dev, saved, k, (2, tokens, hidden), "saved"),
            None if dx is None else dx.data_ptr(), width if dx is None else _matrix(dev, dx, kind, shape, "dx"),
            _whole(dev, dw_gate, gk, (hidden, width), "dw_gate"), _whole(dev, dw_up, gk, (hidden, width), "dw_up"),
            _whole(dev, dw_down, gk, (width, hidden), "dw_down")), "scalecom_gated_ffn_backward")

    def orthogonalise(self, update: torch.Tensor, out: torch.Tensor, steps: int = 5,
                      coefficients: Sequence = (3.4445, -4.7750, 2.0315), eps: float = 1e-7, scale: float = 1.0) -> None:
        """out = scale * (`steps` Newton-Schulz steps on update / (|update|_F + eps)), for a matrix or a batch of matrices.
        coefficients: (a, b, c), or one such triple for each step."""
        if update.dim() not in (2, 3) or out.shape != update.shape:
            raise ValueError("update and out must be matrices, or batches of matrices, of one shape")
        dev = self._device
        kin, kout = _type(dev, update, "update"), _type(dev, out, "out")
        a, b = (update, out) if update.dim() == 3 else (update.unsqueeze(0), out.unsqueeze(0))
        batch, rows, cols = a.shape
        ld, stride = [], []
        for t, name in ((a, "update"), (b, "out")):
            s0, s1, s2 = t.stride()
            if (cols > 1 and s2 != 1) or (rows > 1 and s1 < cols):
                raise ValueError("%s must have contiguous rows" % name)
            ld.append(s1 if rows > 1 else max(s1, cols))
            stride.append(s0 if batch > 1 else 0)
        flat = [float(v) for c in coefficients for v in c] if hasattr(coefficients[0], "__len__") else [float(v) for v in coefficients]
        if len(flat) not in (3, 3 * steps):
            raise ValueError("coefficients must be one triple, or one for each step")
        co = (ctypes.c_float * len(flat))(*flat)
        _check(self._orthogonalise(self._h, batch, rows, cols, kin, update.data_ptr(), ld[0], stride[0], kout, out.data_ptr(),
                                            ld[1], stride[1], int(steps), ctypes.cast(co, ctypes.c_void_p), len(flat) // 3, eps, scale),
               "scalecom_orthogonalise")
