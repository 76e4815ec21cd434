"""The edges of a block: the norm before it, and the join after it with its gate, residual scale and dropout.

    Y = residual.norm(X, residual.Norm("rms", weight))            # before a block; fp32, binary16 or bfloat16, X [..., d]
    S = residual.join(X, B, gate=gate, scale=0.5, drop=drop)      # X + 0.5 gate drop(B)
    S, Y = residual.join(X, B, after=N1, gate=gate, before=N2)    # S = X + gate N1(B), Y = N2(S): the next block's input at once

All of a row's steps run in one kernel (``rsh_join_forward``) in fp32; S and Y are each rounded once, Y being the norm of the sum as it was
before its rounding.  Autograd-aware (reverse mode, first derivatives) in X, B, the gate and the norms' parameters; one pass over the
rows (two beyond 8192 columns, ``rsh_join_backward``) forms all gradients, from X, B and two numbers a row and norm: S is added up again,
since the rounded one would bring its error into them.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding
from .dropout import _FORWARD_MODE, MOST, NOTHING, Drop, _struct
from .mx4 import _TYPES, _on, _rows, _tangent

_DROPS = (type(None), Drop)
KINDS = {"rms": binding.RSH_NORM_RMS, "layer": binding.RSH_NORM_LAYER}


class Norm:
    """x r weight + bias with r = 1 / sqrt(mean of x^2 + eps) ("rms"), or the same of x - mean of x ("layer").  weight, bias: [d] in
    fp32 or in the rows' type, None for ones and zeros."""

    __slots__ = ("kind", "weight", "bias", "eps")

    def __init__(self, kind: str = "rms", weight=None, bias=None, eps: float = 1e-6):
        if kind not in KINDS:
            raise ValueError(f"kind: expected one of {list(KINDS)}, got {kind!r}")
        if not 2.0 ** -126 <= eps < float("inf"):
            raise ValueError(f"eps: expected a positive normal number of fp32, got {eps}")
        self.kind, self.weight, self.bias, self.eps = kind, weight, bias, eps


_NORMS = (type(None), Norm)


_NO_NORM = binding.rsh_norm_t()


def _norm_struct(kind: int, eps: float, weight, bias, stats):
    """Of a norm whose parameters are contiguous or None."""
    return binding.rsh_norm_t(None if weight is None else weight.data_ptr(), None if bias is None else bias.data_ptr(), stats,
                              0 if weight is None else _TYPES[weight.dtype], 0 if bias is None else _TYPES[bias.dtype], kind, eps)


class _Plan:
    """What of a join is no tensor: kinds and eps of both norms, the residual scale, dropout."""

    __slots__ = ("after", "after_eps", "before", "before_eps", "scale", "drop")

    def __init__(self, after, before, scale, drop):
        self.after, self.after_eps = (KINDS[after.kind], after.eps) if after else (0, 0.0)
        self.before, self.before_eps = (KINDS[before.kind], before.eps) if before else (0, 0.0)
        self.scale, self.drop = scale, drop


def _describe(plan, X, B, gate, aw, ab, bw, bb, S, Y, stats, t, d, device):
    """The library's structure, and what has to live until the launch.  X may be None in a backward pass."""
    x = b = g = first = second = at_x = at_b = at_g = None
    ld_x = ld_b = ld_g = g_type = 0
    if X is not None:
        x, ld_x = _rows(X, MOST)
        at_x = x.data_ptr()
    if B is not None:
        b, ld_b = _rows(B, MOST)
        at_b = b.data_ptr()
    if gate is not None:
        g, ld_g = (gate, 0) if gate.dim() == 1 else _rows(gate, MOST)
        at_g, g_type = g.data_ptr(), _TYPES[g.dtype]
    if stats is not None:
        first = stats.data_ptr()
        second = first + 8 * t if plan.after and plan.before else first
    join = binding.rsh_join_t(at_x, at_b, at_g, None if S is None else S.data_ptr(), None if Y is None else Y.data_ptr(), t, d, ld_x, ld_b, ld_g,
                              _norm_struct(plan.after, plan.after_eps, aw, ab, first) if plan.after else _NO_NORM,
                              _norm_struct(plan.before, plan.before_eps, bw, bb, second) if plan.before else _NO_NORM,
                              NOTHING if plan.drop is None else _struct(plan.drop, device), _TYPES[(X if B is None else B).dtype], g_type, plan.scale)
    return join, (x, b, g)


def _forward(plan, X, B, gate, aw, ab, bw, bb, keep):
    t, d = X.shape
    device = X.get_device()
    S = None if B is None else X.new_empty((t, d))
    Y = X.new_empty((t, d)) if plan.before else None
    stats = None
    if keep and (plan.after or plan.before):
        stats = X.new_empty((bool(plan.after) + bool(plan.before), t, 2), dtype=torch.float32)
    with _on(device):
        join, alive = _describe(plan, X, B, gate, aw, ab, bw, bb, S, Y, stats, t, d, device)
        binding.join_forward(join)
    return S, Y, stats


def _backward(ctx, *grads):
    plan, want = ctx.plan, ctx.needs_input_grad
    X, B, gate, aw, ab, bw, bb, stats, seed = ctx.saved_tensors
    dS = grads[0] if B is not None else None
    dY = grads[-1] if plan.before else None
    like = dY if dS is None else dS
    if like is None:
        return (None,) * 9
    if _tangent(*(g for g in (dS, dY) if g is not None)):
        raise ValueError(_FORWARD_MODE)
    t, d = like.shape
    dX = like.new_empty((t, d)) if want[1] else None
    dB = like.new_empty((t, d)) if want[2] else None
    dgate = torch.empty(gate.shape, dtype=gate.dtype, device=gate.device) if want[3] else None
    daw = torch.empty_like(aw) if want[4] else None
    dab = torch.empty_like(ab) if want[5] else None
    dbw = torch.empty_like(bw) if want[6] and dY is not None else None
    dbb = torch.empty_like(bb) if want[7] and dY is not None else None
    vectors = (daw is not None) + (dab is not None) + (dbw is not None) + (dbb is not None) + (dgate is not None and gate.dim() == 1)
    out = (None, dX, dB, dgate, daw, dab, dbw, dbb, None)
    if not vectors and dX is None and dB is None and dgate is None:
        return out
    ds, ld_ds = _rows(dS, MOST) if dS is not None else (None, 0)
    dy, ld_dy = _rows(dY, MOST) if dY is not None else (None, 0)
    at, device = binding._address, like.get_device()
    with _on(device):
        join, alive = _describe(plan, X, B, gate, aw, ab, bw, bb, None, None, stats, t, d, device)
        gradients = binding.rsh_join_gradients_t(at(ds), at(dy), at(dX), at(dB), at(dgate), at(daw), at(dab), at(dbw), at(dbb), None, ld_ds, ld_dy)
        binding.join_backward(join, gradients, vectors, like)
    return out


_backward_once = once_differentiable(_backward)


class _Join(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, X, B, gate, aw, ab, bw, bb, seed):
        ctx.set_materialize_grads(False)
        S, Y, stats = _forward(plan, X, B, gate, aw, ab, bw, bb, True)
        ctx.plan = plan
        ctx.save_for_backward(X if plan.before else None, B, gate, aw, ab, bw, bb, stats, seed)
        return Y if S is None else S if Y is None else (S, Y)

    @staticmethod
    def backward(ctx, *grads):
        # where the gradients' own graph is wanted, it ends here with an error
        return _backward_once(ctx, *grads) if torch.is_grad_enabled() else _backward(ctx, *grads)


def _refuse(X, B, after, gate, drop, before):
    """Say what does not fit."""
    for name, n in (("after", after), ("before", before)):
        if n is not None and not isinstance(n, Norm):
            raise TypeError(f"{name}: expected Norm or None, got {type(n)}")
    if drop is not None and not isinstance(drop, Drop):
        raise TypeError(f"drop: expected Drop or None, got {type(drop)}")
    if not isinstance(X, torch.Tensor) or X.dtype not in _TYPES or X.dim() < 1:
        raise TypeError(f"X: expected a tensor [..., d] of {list(_TYPES)}, got {getattr(X, 'dtype', type(X))} {tuple(getattr(X, 'shape', ()))}")
    if not X.is_cuda:
        raise ValueError(f"X: expected a tensor on the GPU, got {X.device}")
    d = X.shape[-1]
    if B is not None and (not isinstance(B, torch.Tensor) or B.dtype != X.dtype or B.shape != X.shape or B.device != X.device):
        raise ValueError(f"B: expected {X.dtype} {tuple(X.shape)} on {X.device}, got "
                         f"{getattr(B, 'dtype', type(B))} {tuple(getattr(B, 'shape', ()))} on {getattr(B, 'device', None)}")
    for name, v, shapes in (("gate", gate, (X.shape, (d,))), ("after.weight", after and after.weight, ((d,),)), ("after.bias", after and after.bias, ((d,),)),
                            ("before.weight", before and before.weight, ((d,),)), ("before.bias", before and before.bias, ((d,),))):
        if v is not None and (not isinstance(v, torch.Tensor) or v.dtype not in (X.dtype, torch.float32) or v.device != X.device or tuple(v.shape) not in map(tuple, shapes)):
            raise ValueError(f"{name}: expected {' or '.join(str(tuple(s)) for s in shapes)} of {X.dtype} or fp32 on {X.device}, got "
                             f"{getattr(v, 'dtype', type(v))} {tuple(getattr(v, 'shape', ()))} on {getattr(v, 'device', None)}")


def _fits(X, B, gate, params) -> bool:
    """The ordinary case of what is refused otherwise: matrices, vectors as parameters."""
    if X.dim() != 2 or not X.is_cuda or X.dtype not in _TYPES:
        return False
    dtype, shape, device = X.dtype, X.shape, X.get_device()
    if B is not None and (type(B) is not torch.Tensor or B.dtype != dtype or B.shape != shape or B.get_device() != device):
        return False
    d = shape[1:]
    for v in params:
        if v is not None and (v.dtype not in (dtype, torch.float32) or v.shape != d or v.get_device() != device):
            return False
    return gate is None or (gate.dtype in (dtype, torch.float32) and (gate.shape == d or gate.shape == shape) and gate.get_device() == device)


def _run(X, B, after, gate, scale, drop, before):
    """S, Y or both, in X's shape."""
    if not (type(X) is torch.Tensor and type(after) in _NORMS and type(before) in _NORMS and type(drop) in _DROPS):
        _refuse(X, B, after, gate, drop, before)
    aw, ab = (after.weight, after.bias) if after is not None else (None, None)
    bw, bb = (before.weight, before.bias) if before is not None else (None, None)
    params = (aw, ab, bw, bb)
    tensors = [v for v in (X, B, gate, *params) if v is not None]
    if not (all(isinstance(v, torch.Tensor) for v in tensors) and _fits(X, B, gate, params)):
        _refuse(X, B, after, gate, drop, before)
    d = X.shape[-1]
    if _tangent(*tensors):
        raise ValueError(_FORWARD_MODE)
    if X.numel() == 0:
        # nothing to norm or add: empty results, whose gradients are zeros
        S = X if B is None else X + B
        S = S + sum(v.sum() for v in tensors[1:] if v.requires_grad).to(X.dtype) * 0 if any(v.requires_grad for v in tensors[1:]) else S * 1
        return (S, S * 1) if B is not None and before else S
    flat = X.dim() == 2
    rows = [v if v is None or flat else v.reshape(-1, d) for v in (X, B)]
    if gate is not None:
        gate = gate.contiguous() if gate.dim() == 1 else gate if flat else gate.reshape(-1, d)
    params = [v if v is None or v.is_contiguous() else v.contiguous() for v in params]
    plan = _Plan(after, before, scale, drop)
    if torch.is_grad_enabled() and any(v.requires_grad for v in tensors):
        out = _Join.apply(plan, *rows, gate, *params, drop.tensor if drop else None)
        if flat:
            return out
        return tuple(o.reshape(X.shape) for o in out) if isinstance(out, tuple) else out.reshape(X.shape)
    S, Y, _ = _forward(plan, *rows, gate, *params, False)
    if not flat:
        S, Y = (v if v is None else v.reshape(X.shape) for v in (S, Y))
    return Y if S is None else S if Y is None else (S, Y)


def norm(X, norm: Norm):
    """N(X) of every row of X [..., d]."""
    if not isinstance(norm, Norm):
        raise TypeError(f"norm: expected Norm, got {type(norm)}")
    return _run(X, None, None, None, 1.0, None, norm)


def join(X, B, after: Norm | None = None, gate=None, scale: float = 1.0, drop: Drop | None = None, before: Norm | None = None):
    """S = X + scale * gate * drop(after(B)), and with ``before`` the pair (S, before(S)).  X, B [..., d] of one type; gate: [d] or of X's
    shape, in fp32 or X's type; scale: a number, finite in fp32 also when divided by 1 - p of drop."""
    if B is None:
        raise TypeError("B: expected a tensor; the norm alone is residual.norm")
    if not abs(scale) < 2.0 ** 127:
        raise ValueError(f"scale: expected a finite number of fp32, got {scale}")
    if isinstance(drop, Drop) and 0 < drop.share < 65536 and not abs(scale) * 65536 / (65536 - drop.share) < 2.0 ** 128:
        raise ValueError(f"scale: {scale} / (1 - {drop.share / 65536}) is beyond fp32")
    return _run(X, B, after, gate, float(scale), drop, before)
