"""A residual block from training to serving many requests, each with an adapter of its own.

Trains a block X + scale gate drop(ffn(norm(X))) towards a fixed one's outputs, freezes its weights in 4 bits, trains low-rank adapters of a few
requests beside its projection back, and serves all requests in one batch:

    python examples/residual_block.py [--d 256] [--f 704] [--tokens 256] [--steps 20] [--requests 3]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_08734_amd import adapters, dropout, ffn, mx4, residual     # noqa: E402

EPS = 1e-5


def block(x, w, drop=None, following=None):
    """The block in its training form; w: norm, gate, W_gate, W_up and W_down."""
    h = ffn.gated(residual.norm(x, residual.Norm("rms", w["norm"], eps=EPS)), w["wg"], w["wu"])
    return residual.join(x, h @ w["wd"].t(), gate=w["gate"], drop=drop, before=following)


def descend(loss_of, weights, steps: int, rate: float, scale: float = 1024.0):
    """Gradient descent with steps of the gradient's own size on fp32 copies of the weights; the losses, and the weights in their types."""
    master = {n: w.float().clone() for n, w in weights.items()}
    losses = []
    for step in range(steps):
        now = {n: master[n].to(w.dtype, copy=True).requires_grad_() for n, w in weights.items()}
        loss = loss_of(now, step)
        for (n, m), g in zip(master.items(), torch.autograd.grad(loss * scale, list(now.values()))):
            m -= rate * m.norm() * g.float() / (g.float().norm() + 1e-30)
        losses.append(loss.item())
    return {n: m.to(weights[n].dtype) for n, m in master.items()}, losses


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("d", 256), ("f", 704), ("tokens", 256), ("steps", 20), ("requests", 3), ("rank", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    args = ap.parse_args(argv)
    d, f, t, n = args.d, args.f, args.tokens, args.requests
    g = torch.Generator(device="cuda").manual_seed(0)

    def weight(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda") * scale

    x = weight(t, d).half()
    fixed = dict(norm=torch.ones(d, device="cuda"), gate=torch.ones(d, device="cuda"), wg=weight(f, d, scale=d ** -0.5).half(),
                 wu=weight(f, d, scale=d ** -0.5).half(), wd=weight(d, f, scale=f ** -0.5).half())
    target = block(x, fixed).float()
    start = {name: (w + 0.3 * weight(*w.shape, scale=w.float().std().item() if w.dim() > 1 else 1.0)).to(w.dtype) for name, w in fixed.items()}
    trained, losses = descend(lambda w, step: (block(x, w, dropout.Drop(0.05, 1, step)).float() - target).square().mean(), start, args.steps, 0.02)
    out = {"first_loss": losses[0], "last_loss": losses[-1]}
    print(f"block: loss {losses[0]:.5f} -> {losses[-1]:.5f} in {args.steps} steps")

    # The frozen block, and adapters towards a target of every request's own.
    four = [mx4.quantize(trained[name]) for name in ("wg", "wu", "wd")]
    norm = residual.Norm("rms", trained["norm"], eps=EPS)
    with torch.no_grad():
        hidden = ffn.gated(residual.norm(x, norm), four[0], four[1])
        shared = mx4.product(hidden, four[2])
    index = torch.arange(t, device="cuda", dtype=torch.int32) % (n + 1)       # the last has none
    wanted = shared.float() + 0.1 * weight(n + 1, 1, d)[index.long()].squeeze(1)
    pair = dict(a=weight(n, args.rank, f, scale=f ** -0.5).half(), b=weight(n, args.rank, d, scale=0.02).half())
    pair, losses = descend(lambda w, step: (adapters.add(shared, hidden, w["a"], w["b"], index).float() - wanted)[index < n].square().mean(), pair,
                           args.steps, 0.05)
    out.update(first_adapter_loss=losses[0], last_adapter_loss=losses[-1])
    print(f"adapters: loss {losses[0]:.5f} -> {losses[-1]:.5f}")

    with torch.no_grad():
        served = ffn.Block(ffn.FeedForward(*four, adapters=(pair["a"], pair["b"], None)), norm, gate=trained["gate"])
        S, Y = served(x, index, following=norm)
        token = torch.cat([served(x[i:i + 1], index[i:i + 1]) for i in range(4)])
    out.update(S=S, Y=Y, token=token, x=x, index=index, four=four, pair=pair, norm=norm, gate=trained["gate"])
    print(f"served {t} tokens of {n + 1} kinds of requests; single tokens differ from the batch by {(token - S[:4]).abs().max().item():.4f}")
    return out


if __name__ == "__main__":
    main()
