"""The gated feed-forward block H = act(X Wg^T) * (X Wu^T), forward and backward, in kernels of the library.

    H = ffn.gated(X, W_gate, W_up, "silu")     # binary16 or bfloat16, X [..., d], weights [f, d]; autograd-aware
    H = ffn.gated(X, Wg4, Wu4, "silu")         # the weights in 4 bits (mx4.quantize), for serving

Both projections, the activation and the product run as one kernel (``rsh_gated_forward``): sums are fp32 until H is rounded.
A forward pass that will be differentiated keeps both projections in the inputs' type; the backward pass
(``rsh_gated_backward``) forms their gradients in one pass over them, rounds those to the same type, and multiplies.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding
from .mx4 import HALVES, Mx4, _matrix, _no_gradient, _on

ACTIVATIONS = {"silu": binding.RSH_ACT_SILU, "gelu": binding.RSH_ACT_GELU, "relu": binding.RSH_ACT_RELU}


def _weights(Wg, Wu):
    """Both weights as matrices with one row stride, and that."""
    Wg, ld = _matrix(Wg, "W_gate", HALVES)
    Wu, ld_u = _matrix(Wu, "W_up", HALVES)
    return (Wg, Wu, ld) if ld == ld_u else (Wg.contiguous(), Wu.contiguous(), Wg.shape[1])


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, Wg, Wu, act, keep):
        x, ld_x = _matrix(X, "X", HALVES)
        wg, wu, ld_w = _weights(Wg, Wu)
        ctx.act = act
        if x.numel() == 0 or wg.numel() == 0:
            ctx.save_for_backward(X, Wg, Wu, None, None)
            return X.new_zeros((X.shape[0], Wg.shape[0]))
        with _on(x.device):
            H, G, U = binding.gated_forward(x, HALVES[x.dtype], ld_x, wg, wu, ld_w, None, None, act, wg.shape[0], keep)
        ctx.save_for_backward(X, Wg, Wu, G, U)
        return H

    @staticmethod
    @once_differentiable
    def backward(ctx, dH):
        X, Wg, Wu, G, U = ctx.saved_tensors
        want = ctx.needs_input_grad[:3]
        if G is None:
            return (*(torch.zeros_like(t) if w else None for t, w in zip((X, Wg, Wu), want)), None, None)
        x, ld_x = _matrix(X, "X", HALVES)
        wg, wu, ld_w = _weights(Wg, Wu)
        dH, ld_h = _matrix(dH.to(X.dtype), "dH", HALVES)
        with _on(x.device):
            grads = binding.gated_backward(x, HALVES[x.dtype], ld_x, wg, wu, ld_w, G, U, dH, ld_h, ctx.act, want)
        return (*grads, None, None)


def gated(X, W_gate, W_up, activation: str = "silu"):
    """act(X W_gate^T) * (X W_up^T): X [..., d], weights [f, d] of X's type or in 4 bits, result [..., f]."""
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation: expected one of {list(ACTIVATIONS)}, got {activation!r}")
    if not isinstance(X, torch.Tensor) or X.dim() < 1:
        raise TypeError(f"X: expected a tensor [..., d], got {type(X)}")
    four = isinstance(W_gate, Mx4)
    if four != isinstance(W_up, Mx4):
        raise TypeError("W_gate and W_up: either both in 4 bits or neither")
    if tuple(W_gate.shape) != tuple(W_up.shape) or len(W_gate.shape) != 2 or W_gate.shape[1] != X.shape[-1]:
        raise ValueError(f"X {tuple(X.shape)}, W_gate {tuple(W_gate.shape)} and W_up {tuple(W_up.shape)} do not fit")
    if X.dtype not in HALVES or (not four and (W_gate.dtype != X.dtype or W_up.dtype != X.dtype)):
        raise TypeError(f"expected one type for X and 16-bit weights, one of {list(HALVES)}; X is {X.dtype}")
    if X.device.type != "cuda" or W_gate.device != X.device or W_up.device != X.device:
        raise ValueError(f"X is on {X.device}, W_gate on {W_gate.device}, W_up on {W_up.device}; expected one GPU")
    act, (f, d) = ACTIVATIONS[activation], W_gate.shape
    rows = X if X.dim() == 2 else X.reshape(-1, d) if d else X.reshape(X.shape[:-1].numel(), 0)
    if four:
        _no_gradient(X)
        if rows.numel() == 0 or f == 0:
            H = X.new_zeros((rows.shape[0], f))
        else:
            x, ld_x = _matrix(rows, "X", HALVES)
            with _on(X.device):
                H, _, _ = binding.gated_forward(x, HALVES[X.dtype], ld_x, W_gate.codes, W_up.codes, 0, W_gate.scales, W_up.scales, act, f, False)
    else:
        keep = torch.is_grad_enabled() and (X.requires_grad or W_gate.requires_grad or W_up.requires_grad)
        H = _Gated.apply(rows, W_gate, W_up, act, keep)
    return H if X.dim() == 2 else H.reshape(*X.shape[:-1], f)
