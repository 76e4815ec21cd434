"""The 64-bit reference of norms, joins, dropout and adapters, pinned by published vectors, central differences and special cases."""
import numpy as np
import pytest
import torch

from oracle import edges


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_generator_gives_the_published_numbers(counter, key, want):
    assert tuple(edges.philox(counter, key)) == want


def test_an_elements_bits_depend_on_its_place_alone():
    seed, offset = 0x0123456789ABCDEF, 0xFEDCBA9876543210
    whole = edges.bits(5, 21, seed, offset)
    assert np.array_equal(edges.bits(3, 13, seed, offset), whole[:3, :13])
    for row, col in ((0, 0), (2, 7), (4, 8), (3, 20)):
        word = edges.philox((col // 8, row, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))[col % 8 // 2]
        assert whole[row, col] == (word >> 16 if col % 2 else word & 0xFFFF)


def test_share_and_independence():
    b = edges.bits(256, 512, 7, 0).astype(np.float64)
    n = b.size
    for p in (0.1, 0.5):
        # a binomial's standard deviation, five times
        assert abs((b < p * 65536).mean() - p) < 5 * (p * (1 - p) / n) ** 0.5
    for other in (edges.bits(256, 512, 8, 0), edges.bits(256, 512, 7, 1)):
        assert abs(np.corrcoef(b.ravel(), other.ravel())[0, 1]) < 5 / n ** 0.5


def _difference(f, leaves, grads, step=1e-6):
    for x, g in zip(leaves, grads):
        flat = x.detach().reshape(-1)
        for i in torch.randperm(flat.numel())[:6].tolist():
            old = flat[i].item()
            flat[i] = old + step
            up = f().item()
            flat[i] = old - step
            down = f().item()
            flat[i] = old
            assert abs((up - down) / (2 * step) - g.reshape(-1)[i].item()) < 1e-6 * (1 + g.abs().max().item())


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_of_a_join(kind):
    torch.manual_seed(0)
    t, d = 3, 11
    x, b, cs, cy = (torch.randn(t, d, dtype=torch.float64) for _ in range(4))
    gate, w1, b1, w2, b2 = (torch.randn(d, dtype=torch.float64) for _ in range(5))
    leaves = [v.requires_grad_() for v in (x, b, gate, w1, b1, w2, b2)]
    drop = edges.kept(t, d, 0.3, 5, 6)

    def f():
        r = edges.join(x, b, (kind, w1, b1, 1e-3), gate, 0.7, drop, (kind, w2, b2, 1e-3))
        return (r["S"] * cs).sum() + (r["Y"] * cy).sum()
    _difference(lambda: f().detach(), leaves, torch.autograd.grad(f(), leaves))


def test_norms_of_plain_rows():
    x = torch.tensor([[3.0, -4.0], [0.0, 0.0]], dtype=torch.float64)
    y, _, r = edges.norm(x, "rms", None, None, 0.5)
    assert torch.allclose(y[0], x[0] / 13 ** 0.5, atol=1e-15) and torch.equal(y[1], x[1]) and abs(r[1].item() - 2 ** 0.5) < 1e-15
    y, _, _ = edges.norm(x, "layer", torch.tensor([2.0, 2.0]).double(), torch.tensor([1.0, 0.0]).double(), 0.75)
    assert torch.allclose(y[0], torch.tensor([2 * 3.5 / 13 ** 0.5 + 1, -2 * 3.5 / 13 ** 0.5]).double(), atol=1e-15)


def test_gradients_of_adapters():
    torch.manual_seed(1)
    t, k, m, n, r = 5, 7, 6, 3, 2
    y, x, c = torch.randn(t, m).double(), torch.randn(t, k).double(), torch.randn(t, m).double()
    a, b = torch.randn(n, r, k).double(), torch.randn(n, r, m).double()
    index, scales = torch.tensor([2, -1, 0, 2, 7]), torch.tensor([0.5, 1.0, 2.0]).double()
    leaves = [v.requires_grad_() for v in (y, x, a, b)]

    def f():
        return (edges.adapt(y, x, a, b, index, scales)[0] * c).sum()
    grads = torch.autograd.grad(f(), leaves)
    _difference(lambda: f().detach(), leaves, grads)
    out, _ = edges.adapt(y, x, a, b, index, scales)
    assert torch.equal(out[[1, 4]], y[[1, 4]]) and not grads[2][1].any()
    assert torch.allclose(out[0], y[0] + 2 * (b[2].t() @ (a[2] @ x[0])))
