"""The edges of a block in 64 bits: norms, the join after a block, dropout's random numbers, low-rank adapters.

Values are torch tensors of float64 on the CPU; gradients come from torch's automatic differentiation of the formulas, which
``tests/test_oracle_edges.py`` pins by central differences.
"""
import numpy as np
import torch

MASK = 0xFFFFFFFF


def philox(counter, key, rounds: int = 10):
    """Philox4x32 (Salmon et al., 2011) of one counter of four words and a key of two."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & MASK, (p >> 32) ^ c[3] ^ k[1], p & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def bits(t: int, d: int, seed: int, offset: int):
    """The 16 random bits of every element of a [t, d] matrix, uint16."""
    blocks = -(-d // 8)
    row, place = np.meshgrid(np.arange(t, dtype=np.uint64), np.arange(blocks, dtype=np.uint64), indexing="ij")
    full = lambda v: np.full_like(row, v)       # noqa: E731
    c = [place, row, full(offset & MASK), full(offset >> 32 & MASK)]
    k0, k1 = seed & MASK, seed >> 32 & MASK
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        low, high = np.uint64(MASK), np.uint64(32)
        c = [(q >> high) ^ c[1] ^ np.uint64(k0), q & low, (p >> high) ^ c[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & MASK, (k1 + 0xBB67AE85) & MASK
    words = np.stack(c, axis=2)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=3)
    return halves.reshape(t, blocks * 8)[:, :d].astype(np.uint16)


def kept(t: int, d: int, p: float, seed: int, offset: int):
    """(mask of what dropout keeps, what it is multiplied by)."""
    share = round(p * 65536)
    return torch.from_numpy(bits(t, d, seed, offset).astype(np.int32) >= share), 65536 / max(65536 - share, 1)


def norm(x, kind, weight, bias, eps):
    """(N(x), x without mean and size, 1 / size) of rows."""
    c = x - x.mean(dim=-1, keepdim=True) if kind == "layer" else x
    r = (c.square().mean(dim=-1, keepdim=True) + eps).rsqrt()
    y = c * r
    y = y if weight is None else y * weight
    return (y if bias is None else y + bias), c * r, r


def join(x, b, after, gate, scale, drop, before):
    """{"S", "Y", ...}: after and before are (kind, weight, bias, eps) or None, drop (mask, factor) or None."""
    out = {}
    n = b
    if after:
        n, out["bh"], out["br"] = norm(b, *after)
    out["n"] = n
    if drop:
        n = torch.where(drop[0], n * drop[1], 0.0)
    out["D"] = n
    out["S"] = x + scale * (n if gate is None else gate * n)
    if before:
        out["Y"], out["Sh"], out["Sr"] = norm(out["S"], *before)
    return out


def adapt(y, x, a, b, index, scales):
    """y + scales[i] (x a[i]^T) b[i], and every token's x a[i]^T."""
    out, h = y, x.new_zeros((x.shape[0], a.shape[1]))
    for i in range(a.shape[0]):
        mine = (index == i).unsqueeze(1)
        hi = x @ a[i].t()
        h = torch.where(mine, hi, h)
        out = torch.where(mine, out + (1.0 if scales is None else scales[i]) * (hi @ b[i]), out)
    return out, h
