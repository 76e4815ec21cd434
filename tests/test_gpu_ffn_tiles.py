"""The feed-forward products in each of their tiles, exactly: 256 x 256, 128 x 128 and 64 x 128, sums whole and in parts, operands straight into LDS
and through registers, at sizes whose rows, columns and k end inside a tile.

Operands are small integers, so every sum is an integer below 2^24 and exact in fp32 in any order; what is rounded inside the gradients
(dG and dU) stays below 256, which bfloat16 has exactly.  So a result is the 64-bit one rounded once, and a missing or
doubled element shows."""
import pytest

pytestmark = pytest.mark.gpu
DTYPES = ["float16", "bfloat16"]


def _sparse(g, rows, cols, share, kind):
    """-1, 0 and 1, `share` of them not zero."""
    import torch
    m = torch.randint(0, 2, (rows, cols), generator=g, device="cuda") * 2 - 1
    return (m * (torch.rand((rows, cols), generator=g, device="cuda") < share)).to(kind)


def _tile(which, aligned, *sizes):
    from paper_2603_08734_amd import binding
    return binding.ffn_tiles(getattr(binding, "RSH_TILES_" + which), aligned, *sizes)


def _equal(got, ref, what):
    import torch
    want = ref.to(got.dtype)
    assert got.shape == want.shape
    wrong = (got != want).nonzero()
    assert torch.equal(got, want), f"{what}: {len(wrong)} of {got.numel()} differ, first at {wrong[0].tolist()}, last at {wrong[-1].tolist()}"


PRODUCTS = [      # which, aligned, t, n, k, tile
    ("PRODUCT", True, 257, 8200, 72, (128, 128, 1)), ("PRODUCT", True, 515, 515, 4104, (128, 128, 7)),
    ("PRODUCT", True, 2570, 3100, 520, (256, 256, 1)), ("PRODUCT", True, 1290, 3100, 4104, (256, 256, 3)),
    ("PRODUCT", False, 2100, 3100, 71, (128, 128, 1)), ("PRODUCT", False, 2100, 136, 4103, (128, 128, 11)),
    ("PRODUCT", False, 2570, 3100, 263, (256, 256, 1)), ("PRODUCT", False, 130, 8200, 4103, (256, 256, 6)),
    ("PRODUCT", False, 130, 131, 519, (64, 128, 5)),
    ("PRODUCT4", True, 257, 8200, 71, (128, 128, 1)), ("PRODUCT4", True, 2570, 3100, 1051, (256, 256, 1)),
    ("PRODUCT4", True, 130, 72, 4101, (64, 128, 11))]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which,aligned,t,n,k,tile", PRODUCTS)
def test_products(which, aligned, t, n, k, tile, dtype):
    import torch
    from paper_2603_08734_amd import mx4
    print(f"case tiles {which} {dtype} t={t} n={n} k={k} {tile}", flush=True)
    assert _tile(which, aligned, t, n, k) == tile
    g = torch.Generator(device="cuda").manual_seed(t + n + k)
    kind, share, blocks = getattr(torch, dtype), min(1.0, (20 / k) ** 0.5), -(-k // 32)
    x = _sparse(g, t, k, share, kind)
    cells = torch.randint(0, 16, (n, blocks * 32), generator=g, device="cuda") * (torch.rand((n, blocks * 32), generator=g, device="cuda") < share)
    cells[:, k:] = 0
    codes = (cells[:, 0::2] | cells[:, 1::2] << 4).to(torch.uint8)
    scales = torch.randint(127, 129, (n, blocks), generator=g, device="cuda").to(torch.uint8)
    W = mx4.Mx4(codes, scales, k)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda", dtype=torch.float64)
    w = (grid[cells].view(n, blocks, 32) * (scales.double() - 126).unsqueeze(2)).view(n, -1)[:, :k]      # 1 or 2 times the value
    got = mx4.product(mx4.quantize(x), W, kind) if which == "PRODUCT4" else mx4.product(x, W)
    _equal(got, x.double() @ w.t(), "Y")


GATED = [         # which, aligned, t, d, f, tile
    ("GATED", True, 700, 72, 1500, (128, 64, 1)), ("GATED", True, 257, 4104, 515, (128, 64, 8)),
    ("GATED", True, 2100, 136, 3100, (256, 128, 1)), ("GATED", True, 130, 4104, 8200, (256, 128, 3)),
    ("GATED", True, 130, 1056, 72, (64, 64, 11)),
    ("GATED", False, 2100, 71, 1500, (128, 64, 1)), ("GATED", False, 2100, 4103, 72, (128, 64, 15)),
    ("GATED", False, 2100, 71, 3100, (256, 128, 1)), ("GATED", False, 130, 4103, 4104, (256, 128, 6)),
    ("GATED", False, 130, 519, 71, (64, 64, 9)),
    ("GATED4", True, 700, 72, 1500, (128, 64, 1)), ("GATED4", True, 257, 4104, 515, (128, 64, 7)),
    ("GATED4", True, 2100, 136, 3100, (256, 128, 1)), ("GATED4", True, 130, 4104, 8200, (256, 128, 3)),
    ("GATED4", False, 2100, 71, 1500, (128, 64, 1)), ("GATED4", False, 2100, 4103, 72, (128, 64, 11)),
    ("GATED4", False, 2100, 71, 3100, (256, 128, 1)), ("GATED4", False, 130, 4103, 4104, (256, 128, 6))]


def _block(g, t, d, f, kind):
    share = min(1.0, (64 / d) ** 0.5)
    return _sparse(g, t, d, share, kind), _sparse(g, f, d, share, kind), _sparse(g, f, d, share, kind)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which,aligned,t,d,f,tile", GATED)
def test_gated_blocks(which, aligned, t, d, f, tile, dtype):
    """The forward pass; with 16-bit weights, the one that keeps G and U too, whose gradients the next test has."""
    import torch
    from paper_2603_08734_amd import ffn, mx4
    print(f"case tiles {which} {dtype} t={t} d={d} f={f} {tile}", flush=True)
    assert _tile(which, aligned, t, d, f) == tile
    x, wg, wu = _block(torch.Generator(device="cuda").manual_seed(t + d + f), t, d, f, getattr(torch, dtype))
    ref = torch.relu(x.double() @ wg.double().t()) * (x.double() @ wu.double().t())
    if which == "GATED4":
        _equal(ffn.gated(x, mx4.quantize(wg), mx4.quantize(wu), "relu"), ref, "H")
        return
    _equal(ffn.gated(x, wg, wu, "relu"), ref, "H")
    _equal(ffn.gated(x.clone().requires_grad_(), wg, wu, "relu").detach(), ref, "H beside kept G and U")


STEPS = [         # which, aligned, t, d, f, tile
    ("DX", True, 515, 4104, 72, (128, 128, 1)), ("DX", True, 700, 136, 3104, (128, 128, 15)),
    ("DX", True, 2100, 4104, 520, (256, 256, 1)), ("DX", True, 130, 4104, 8200, (256, 256, 12)),
    ("DX", False, 1030, 4103, 135, (128, 128, 1)), ("DX", False, 2100, 135, 2071, (128, 128, 15)),
    ("DX", False, 2100, 4103, 135, (256, 256, 1)), ("DX", False, 130, 4103, 3099, (256, 256, 15)),
    ("DW", True, 130, 136, 4104, (128, 128, 1)), ("DW", True, 2100, 72, 3104, (128, 128, 4)),
    ("DW", True, 130, 2056, 3104, (256, 256, 1)), ("DW", True, 2100, 136, 8200, (256, 256, 3)),
    ("DW", False, 130, 263, 8199, (128, 128, 1)), ("DW", False, 2570, 135, 1499, (128, 128, 8)),
    ("DW", False, 130, 4103, 1499, (256, 256, 1)), ("DW", False, 1290, 135, 8199, (256, 256, 3)),
    ("DW_ONE", True, 130, 136, 8200, (128, 128, 1)), ("DW_ONE", True, 2570, 136, 2072, (128, 128, 6)),
    ("DW_ONE", True, 130, 4104, 3104, (256, 256, 1)), ("DW_ONE", True, 2570, 2056, 2072, (256, 256, 3)),
    ("DW_ONE", False, 130, 4103, 1499, (128, 128, 1)), ("DW_ONE", False, 2570, 135, 3099, (128, 128, 8)),
    ("DW_ONE", False, 130, 4103, 3099, (256, 256, 1)), ("DW_ONE", False, 2570, 263, 8199, (256, 256, 3))]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which,aligned,t,d,f,tile", STEPS + [
    ("GATED", a, t, d, f, tile) for which, a, t, d, f, tile in GATED if which == "GATED"])
def test_gradients(which, aligned, t, d, f, tile, dtype):
    """All gradients of a step, sized for one product's tiles; one weight's at a time where that is the product."""
    import torch
    from paper_2603_08734_amd import ffn
    print(f"case tiles {which} {dtype} t={t} d={d} f={f} {tile}", flush=True)
    assert _tile(which, aligned, t, d, f) == tile
    g = torch.Generator(device="cuda").manual_seed(t + d + f)
    x, wg, wu = _block(g, t, d, f, getattr(torch, dtype))
    dh = _sparse(g, t, f, 0.5, x.dtype)
    x64, wg64, wu64 = x.double(), wg.double(), wu.double()
    G, U = x64 @ wg64.t(), x64 @ wu64.t()
    dG, dU = dh.double() * U * (G > 0), dh.double() * torch.relu(G)
    assert max(dG.abs().max(), dU.abs().max()) <= 256
    refs = {"dX": lambda: dG @ wg64 + dU @ wu64, "dWg": lambda: dG.t() @ x64, "dWu": lambda: dU.t() @ x64}
    for want in ((1, 2) if which == "DW_ONE" else (None,)):
        leaves = [m.detach().requires_grad_(want in (None, i)) for i, m in enumerate((x, wg, wu))]
        H = ffn.gated(*leaves, "relu")
        names = [n for n, leaf in zip(refs, leaves) if leaf.requires_grad]
        for name, got in zip(names, torch.autograd.grad(H, [leaf for leaf in leaves if leaf.requires_grad], dh)):
            _equal(got, refs[name](), name)


def test_the_tiles_that_are_asked_for():
    """Refusals, and that few rows have no tiles."""
    import ctypes
    from paper_2603_08734_amd import binding as b
    assert b.ffn_tiles(b.RSH_TILES_PRODUCT, True, 16, 512, 512) == (0, 0, 0) and b.ffn_tiles(b.RSH_TILES_DX, True, 16, 512, 512) != (0, 0, 0)
    tile = (ctypes.c_int32 * 3)()
    assert b.lib().rsh_ffn_tiles(7, 1, 64, 64, 64, tile) == b.RSH_ERR_BAD_OPTION and b.lib().rsh_ffn_tiles(-1, 1, 64, 64, 64, tile) == b.RSH_ERR_BAD_OPTION
    assert b.lib().rsh_ffn_tiles(0, 1, 64, 0, 64, tile) == b.RSH_ERR_BAD_OPTION and b.lib().rsh_ffn_tiles(0, 1, 64, 64, 64, None) == b.RSH_ERR_NULL
