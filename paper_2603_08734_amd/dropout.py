"""Dropout whose random numbers are a function of a seed, an offset and an element's place, so that no mask is stored.

    drop = dropout.Drop(0.1, seed, offset)       # offset: what tells apart the layers and steps of a program, say
    Y = dropout.dropout(X, drop)                 # fp32, binary16 or bfloat16, [..., d] with d up to 2^21; autograd-aware, derivatives of any order
    S = residual.join(X, B, drop=drop)           # the same numbers inside the join after a block

An element is dropped (becomes zero, whatever it was) with probability p, rounded to a multiple of 2^-16, and multiplied by
1 / (1 - p) otherwise, in the join too and for the gradients.  ``include/rsh_spmm.h`` says which random number an element has: rows are the last
dimension, counted over the others.
"""
from __future__ import annotations

import torch

from . import binding
from .mx4 import _TYPES, _on, _rows, _tangent

_FORWARD_MODE = "dropout and joins have no forward-mode derivative: call them on detached operands"
MOST = binding.RSH_ROWS_MAX_STRIDE       # elements from row to row; rows further apart are copied


NOTHING = binding.rsh_drop_t()      # no dropout, as part of other structures


class Drop:
    """p: share that is dropped, 0 .. 1.  seed: an integer, or an int64 tensor of one element on the operands' GPU, read when the kernels
    run (a captured graph draws new numbers when the program changes it between replays; changing it between a forward pass and its
    backward pass is an error).  offset: an integer; both are taken modulo 2^64.  It does not change afterwards."""

    __slots__ = ("share", "seed", "offset")

    def __init__(self, p: float, seed, offset: int = 0):
        if not 0 <= p <= 1:
            raise ValueError(f"p: expected a number from 0 to 1, got {p}")
        if isinstance(seed, torch.Tensor):
            if seed.dtype != torch.int64 or seed.numel() != 1 or not seed.is_cuda:
                raise ValueError(f"seed: expected an integer or one int64 on the GPU, got {seed.dtype} {tuple(seed.shape)} on {seed.device}")
        else:
            seed = int(seed) % (1 << 64)
        for name, v in zip(self.__slots__, (round(p * 65536), seed, int(offset) % (1 << 64))):
            object.__setattr__(self, name, v)

    def __setattr__(self, name, value):
        # a backward pass draws the forward pass's numbers again
        raise AttributeError(f"{name}: a Drop does not change; make another")

    def __reduce__(self):
        return Drop, (self.share / 65536, self.seed, self.offset)

    @property
    def tensor(self):
        """The seed where it is a tensor, else None."""
        return self.seed if isinstance(self.seed, torch.Tensor) else None


def _struct(drop, device: int):
    """The library's description; no dropout where there is none."""
    if drop is None:
        return NOTHING
    seed = drop.tensor
    if seed is None:
        return binding.rsh_drop_t(drop.seed, drop.offset, None, drop.share)
    if seed.get_device() != device:
        raise ValueError(f"seed is on {seed.device}, the operands on cuda:{device}")
    return binding.rsh_drop_t(0, drop.offset, seed.data_ptr(), drop.share)


def _apply(X, drop):
    x, ld = _rows(X, MOST)
    with _on(x.get_device()):
        return binding.dropout(x, _TYPES[x.dtype], ld, _struct(drop, x.get_device()))


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, drop):
        ctx.drop = drop
        if drop.tensor is not None:
            ctx.save_for_backward(drop.tensor)
        return _apply(X, drop)

    @staticmethod
    def backward(ctx, dY):
        ctx.saved_tensors       # a seed that has changed is an error
        return dropout(dY, ctx.drop), None


def dropout(X, drop: Drop):
    """X with the share of its elements dropped that ``drop`` says."""
    if not isinstance(drop, Drop):
        raise TypeError(f"drop: expected Drop, got {type(drop)}")
    if not isinstance(X, torch.Tensor) or X.dtype not in _TYPES:
        raise TypeError(f"X: expected a tensor of {list(_TYPES)}, got {getattr(X, 'dtype', type(X))}")
    if not X.is_cuda:
        raise ValueError(f"X: expected a tensor on the GPU, got {X.device}")
    if _tangent(X):
        raise ValueError(_FORWARD_MODE)
    if X.numel() == 0:
        return X * 1
    rows = X if X.dim() == 2 else X.reshape(-1, X.shape[-1]) if X.dim() else X.reshape(1, 1)
    Y = _Dropout.apply(rows, drop) if X.requires_grad and torch.is_grad_enabled() else _apply(rows, drop)
    return Y if X.dim() == 2 else Y.reshape(X.shape)
