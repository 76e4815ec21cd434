"""Matrices in microscaled 4-bit floating point: 32 elements of a row share a power of two and are held as one of
0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign, 17 bytes where binary16 takes 64.

    W4 = mx4.quantize(W)                 # W [n, k] fp32, binary16 or bfloat16, made once
    Y = mx4.product(X, W4)               # X [t, k] binary16 or bfloat16: the weight alone is in 4 bits
    Y = mx4.product(mx4.quantize(X), W4, torch.bfloat16)    # both are: the matrix units multiply the codes
    mx4.dequantize(W4, torch.float32)    # the values

All of it runs in kernels of the library (``rsh_mx4_*``) on the current stream; sums are fp32, rounded once.  Serving
forms: nothing here records a gradient, and operands that want one are refused while gradients are recorded; operands with a
forward-mode tangent are refused.
"""
from __future__ import annotations

import contextlib

import torch
from torch.autograd import forward_ad

from . import binding

BLOCK = 32
_TYPES = {torch.float32: binding.RSH_F32, torch.float16: binding.RSH_F16, torch.bfloat16: binding.RSH_BF16}
_NOTHING = contextlib.nullcontext()
_WHAT = "products and conversions in 4 bits, and layers as they are served, have"


def _on(index: int):
    """Launches go to the current device: make the operands' device that."""
    return _NOTHING if index == torch._C._cuda_getDevice() else torch.cuda.device(index)


def _matrix(X, name: str, types, most: int):
    """X as (matrix whose rows are contiguous, elements from row to row)."""
    if not isinstance(X, torch.Tensor) or X.dtype not in types:
        raise TypeError(f"{name}: expected a tensor of {' or '.join(str(t) for t in types)}, got {getattr(X, 'dtype', type(X))}")
    if X.dim() != 2:
        raise ValueError(f"{name}: expected a matrix, got shape {tuple(X.shape)}")
    if not X.is_cuda:
        raise ValueError(f"{name}: expected a tensor on the GPU, got {X.device}")
    return _rows(X, most)


def _rows(X, most: int = binding.RSH_FFN_MAX_WIDTH):
    """The same for a matrix that is known to be one.  Rows further apart than `most` elements, which the library refuses, are copied
    like columns with a stride."""
    k = X.shape[1]
    if X.is_contiguous():
        return X, k
    if (k > 1 and X.stride(1) != 1) or (X.shape[0] > 1 and not k <= X.stride(0) <= most):
        return X.contiguous(), k
    return X, X.stride(0) if X.shape[0] > 1 else k


def _tangent(*tensors) -> bool:
    """Whether one of them carries a tangent (forward-mode derivatives, which torch.no_grad() does not stop)."""
    if forward_ad._current_level < 0:      # no such derivative is being formed anywhere
        return False
    for t in tensors:
        if forward_ad.unpack_dual(t).tangent is not None:
            return True
    return False


def _no_gradient(*tensors) -> None:
    if any(t.requires_grad for t in tensors) and torch.is_grad_enabled():
        raise ValueError(f"{_WHAT} no gradient: call them under torch.no_grad() or on detached operands")
    if _tangent(*tensors):
        raise ValueError(f"{_WHAT} no forward-mode derivative: call them on detached operands")


class Mx4:
    """A matrix [rows, k]: codes uint8 [rows, 16 B] and scales uint8 [rows, B], B = ceil(k / 32), as
    ``include/rsh_spmm.h`` describes them (cells past k are zero)."""

    __slots__ = ("codes", "scales", "shape")

    def __init__(self, codes, scales, k: int):
        k, blocks = int(k), -(-int(k) // BLOCK)
        for t, name, width in ((codes, "codes", 16 * blocks), (scales, "scales", blocks)):
            if t.dtype != torch.uint8 or t.dim() != 2 or not t.is_contiguous() or t.shape[1] != width:
                raise ValueError(f"{name}: expected contiguous uint8 [rows, {width}] for k = {k}, got {t.dtype} {tuple(t.shape)}")
        if codes.shape[0] != scales.shape[0] or codes.device != scales.device or codes.device.type != "cuda":
            raise ValueError(f"codes and scales: {tuple(codes.shape)} on {codes.device} against {tuple(scales.shape)} on {scales.device}")
        if codes.data_ptr() % 16 or scales.data_ptr() % 4:
            raise ValueError("codes and scales: expected alignment to 16 and 4 bytes")
        self.codes, self.scales, self.shape = codes, scales, (codes.shape[0], k)

    @classmethod
    def _of(cls, codes, scales, k: int):
        """Of arrays that the library has just made."""
        Q = cls.__new__(cls)
        Q.codes, Q.scales, Q.shape = codes, scales, (codes.shape[0], k)
        return Q

    @property
    def device(self):
        return self.codes.device

    def dequantize(self, dtype=torch.bfloat16):
        return dequantize(self, dtype)

    def __repr__(self):
        return f"Mx4(shape={self.shape}, device={self.device})"


def quantize(X) -> Mx4:
    """X [rows, k] (fp32, binary16 or bfloat16; rows with a stride are read in place) in 4 bits."""
    X, ld = _matrix(X, "X", _TYPES, (1 << 31) - 1)
    _no_gradient(X)
    rows, k = X.shape
    if rows == 0 or k == 0:
        blocks = -(-k // BLOCK)
        return Mx4._of(*(torch.empty((rows, w), dtype=torch.uint8, device=X.device) for w in (16 * blocks, blocks)), k)
    with _on(X.get_device()):
        return Mx4._of(*binding.mx4_quantize(X, _TYPES[X.dtype], ld), k)


def dequantize(Q: Mx4, dtype=torch.bfloat16):
    """The values of Q; fp32 and bfloat16 hold each of them exactly."""
    if dtype not in _TYPES:
        raise TypeError(f"dtype: expected one of {list(_TYPES)}, got {dtype}")
    Y = torch.empty(Q.shape, dtype=dtype, device=Q.device)
    if Y.numel():
        with _on(Q.codes.get_device()):
            binding.mx4_dequantize(Q.codes, Q.scales, Y, _TYPES[dtype])
    return Y


HALVES = {t: c for t, c in _TYPES.items() if t != torch.float32}


def product(X, W: Mx4, dtype=None):
    """X W^T: X [t, k] binary16 or bfloat16 (the result's type too), or in 4 bits with the result's type given."""
    if not isinstance(W, Mx4):
        raise TypeError(f"W: expected Mx4, got {type(W)}")
    if isinstance(X, Mx4):
        if dtype not in HALVES:
            raise TypeError(f"dtype: expected one of {list(HALVES)} beside activations in 4 bits, got {dtype}")
        data, x_scales, x_type, ld = X.codes, X.scales, binding.RSH_MX4, 0
    else:
        data, ld = _matrix(X, "X", HALVES, binding.RSH_FFN_MAX_WIDTH)
        _no_gradient(data)
        if dtype not in (None, data.dtype):
            raise TypeError(f"dtype: the result has the activations' type {data.dtype}, asked for {dtype}")
        dtype, x_scales, x_type = data.dtype, None, HALVES[data.dtype]
    (t, k), n = X.shape, W.shape[0]
    if k != W.shape[1]:
        raise ValueError(f"X {tuple(X.shape)} and W {W.shape}: the last sizes differ")
    if data.get_device() != W.codes.get_device():
        raise ValueError(f"X is on {data.device}, W on {W.device}")
    if t == 0 or n == 0 or k == 0:
        return torch.zeros((t, n), dtype=dtype, device=W.device)
    Y = torch.empty((t, n), dtype=dtype, device=W.device)
    with _on(W.codes.get_device()):
        binding.mx4_product(data, x_scales, x_type, ld, W.codes, W.scales, Y, HALVES[dtype], k)
    return Y
