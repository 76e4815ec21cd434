"""The dense feed-forward work that programs give this library: matrices held in microscaled 4-bit floating point,
products with them, and the gated block of a feed-forward layer with its gradients.

A case is a dict of plain values:

  op     "round_trip"  quantise a matrix [rows, k] to 4 bits and read its values back
         "product"     Y = X W^T with W [n, k] held in 4 bits; x4: the activations [t, k] are quantised to 4 bits too
         "gated"       H = act(X Wg^T) * (X Wu^T), X [t, d], Wg and Wu [f, d]; w4: the weights are held in 4 bits
         "gated_train" the same with the gradients of X, Wg and Wu for a given gradient of H
  dtype  "fp32", "fp16" or "bf16": inputs, results and gradients
  act    "silu", "gelu" (with the error function) or "relu"

Weights in 4 bits are made in ``prepare``: a program quantises a weight once and multiplies with it many times.
Activations are quantised inside the pass.
"""
import torch

own = False     # True: the calls that a user makes of the library; False: the same in elementary operations

DTYPE = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32      # elements that share a scale


def listed():
    return [
        # one token's activations before a product in 4 bits: the smallest call, where latency and launches count
        dict(name="round_trip_token", op="round_trip", rows=1, k=8192, dtype="bf16"),
        # a whole weight at load time
        dict(name="round_trip_weight", op="round_trip", rows=28672, k=8192, dtype="bf16"),
        # activations of a ragged batch, rows that end inside a block, in full precision
        dict(name="round_trip_ragged", op="round_trip", rows=1999, k=4999, dtype="fp32"),
        # one token through a projection, as decoding multiplies it: the weight is read once
        dict(name="product_token", op="product", t=1, n=28672, k=8192, x4=False, dtype="bf16"),
        # 128 tokens of a serving batch through the projection back, long rows and few of them
        dict(name="product_batch", op="product", t=128, n=8192, k=28672, x4=False, dtype="fp16"),
        # a prompt with weights and activations in 4 bits
        dict(name="product_prompt_x4", op="product", t=4096, n=28672, k=8192, x4=True, dtype="bf16"),
        # odd sizes throughout, a few tokens of several requests, both sides in 4 bits
        dict(name="product_odd_x4", op="product", t=77, n=1003, k=4100, x4=True, dtype="fp16"),
        # one token through the gated block
        dict(name="gated_token", op="gated", t=1, d=8192, f=28672, act="silu", w4=False, dtype="bf16"),
        # a few requests decoding together on 4-bit weights
        dict(name="gated_batch_w4", op="gated", t=16, d=4096, f=16384, act="silu", w4=True, dtype="bf16"),
        # a prompt through the gated block
        dict(name="gated_prompt", op="gated", t=2048, d=8192, f=28672, act="silu", w4=False, dtype="bf16"),
        # a training step of a small model on a ragged batch, odd widths
        dict(name="train_odd", op="gated_train", t=1001, d=500, f=1333, act="gelu", dtype="fp16"),
        # a training step of a large block
        dict(name="train_large", op="gated_train", t=4096, d=4096, f=16384, act="silu", dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def _size(rng, lo, hi):
    """Half of the widths are what comes out, the others the multiple of 64 below, as models choose them."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.5 or n < 64 else n // 64 * 64


def draw(rng):
    kind = rng.choice(["round_trip", "product", "product", "gated", "gated", "gated_train"])
    half = rng.choice(["fp16", "bf16"])
    if kind == "round_trip":
        k = _size(rng, 32, 28672)
        return dict(op=kind, rows=_log_int(rng, 1, 28672 * 8192 // k), k=k, dtype=rng.choice(["fp32", "fp16", "bf16"]))
    t = _log_int(rng, 1, 4096)
    if kind == "product":
        return dict(op=kind, t=t, n=_size(rng, 64, 28672), k=_size(rng, 64, 28672 if t <= 1024 else 8192), x4=rng.random() < 0.5, dtype=half)
    d, f = _size(rng, 64, 8192 if t <= 2048 else 4096), _size(rng, 64, 28672 if kind == "gated" or t <= 1024 else 16384)
    act = rng.choice(["silu", "silu", "gelu", "relu"])
    if kind == "gated":
        return dict(op=kind, t=t, d=d, f=f, act=act, w4=rng.random() < 0.5, dtype=half)
    return dict(op=kind, t=t, d=d, f=f, act=act, dtype=half)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(g, rows, cols, scale):
    return torch.randn((rows, cols), generator=g, device="cuda") * scale


def _activations(g, rows, cols, dtype):
    """Unit normal with one feature in 64 twenty times as large, as the outlier features of real activations are."""
    x = _normal(g, rows, cols, 1.0)
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 64, 20.0, 1.0)
    return x.to(DTYPE[dtype])


def _weight_4bit(g, n, k):
    """Codes and scales of a random weight whose blocks differ in size: codes as they occur, scales near 1 / (4 sqrt(k))."""
    blocks = -(-k // BLOCK)
    codes = torch.randint(0, 256, (n, blocks * BLOCK // 2), generator=g, device="cuda", dtype=torch.uint8)
    if k % BLOCK:       # cells past the end of a row are zero
        codes[:, (k + 1) // 2:] = 0
        if k % 2:
            codes[:, k // 2] &= 15
    centre = 127 - 2 - round(0.5 * (k - 1).bit_length())
    scales = (centre + torch.randint(-2, 2, (n, blocks), generator=g, device="cuda")).to(torch.uint8)
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op, dtype = case["op"], case["dtype"]
    if op == "round_trip":
        s["x"] = _activations(g, case["rows"], case["k"], dtype)
    elif op == "product":
        s["x"] = _activations(g, case["t"], case["k"], dtype)
        s["w"] = _weight_4bit(g, case["n"], case["k"])
    else:
        t, d, f = case["t"], case["d"], case["f"]
        s["x"] = _normal(g, t, d, 1.0).to(DTYPE[dtype])
        if case.get("w4"):
            s["wg"], s["wu"] = _weight_4bit(g, f, d), _weight_4bit(g, f, d)
        else:
            s["wg"], s["wu"] = (_normal(g, f, d, d ** -0.5).to(DTYPE[dtype]) for _ in range(2))
        if op == "gated_train":
            s["dh"] = _normal(g, t, f, 0.05).to(DTYPE[dtype])
    if own:
        from paper_2603_08734_amd import mx4
        for name in ("w", "wg", "wu"):
            if isinstance(s.get(name), tuple):
                s[name] = mx4.Mx4(*s[name], case["k"] if op == "product" else case["d"])
        if op == "gated_train":
            for name in ("x", "wg", "wu"):
                s[name].requires_grad_()
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _quantised(x):
    """The values (fp32) that the 4-bit form of x stands for."""
    rows, k = x.shape
    blocks = -(-k // BLOCK)
    v = torch.zeros((rows, blocks * BLOCK), dtype=torch.float32, device=x.device)
    v[:, :k] = x.float()
    v = v.view(rows, blocks, BLOCK)
    e = torch.frexp(v.abs().amax(dim=2, keepdim=True))[1] - 3     # frexp's fraction is below 1: floor(log2) is its exponent - 1
    e = e.clamp(-127, 127)
    m = torch.ldexp(v.abs(), -e)
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    m = (torch.round(m / step) * step).clamp(max=6)
    return torch.ldexp(torch.copysign(m, v), e).view(rows, blocks * BLOCK)[:, :k]


def _values(w, k):
    codes, scales = w
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device=codes.device)
    q = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], dim=2).view(codes.shape[0], -1, BLOCK)
    return torch.ldexp(q, scales.int().unsqueeze(2) - 127).view(codes.shape[0], -1)[:, :k]


def _act(g, act):
    """act(g) and its derivative."""
    if act == "relu":
        return g * (g > 0), (g > 0).float()
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    c = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (2 * torch.pi) ** -0.5


def _plain(s):
    op, dtype = s["op"], DTYPE[s["dtype"]]
    if op == "round_trip":
        return _quantised(s["x"]).to(dtype)
    if op == "product":
        x = _quantised(s["x"]) if s["x4"] else s["x"].float()
        return (x @ _values(s["w"], s["k"]).t()).to(dtype)
    x = s["x"].float()
    wg, wu = ((_values(s[n], s["d"]) if s.get("w4") else s[n].float()) for n in ("wg", "wu"))
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(g, s["act"])
    if op == "gated":
        return (a * u).to(dtype)
    dh = s["dh"].float()
    dg, du = dh * u * da, dh * a
    return [(a * u).to(dtype), (dg @ wg + du @ wu).to(dtype), (dg.t() @ x).to(dtype), (du.t() @ x).to(dtype)]


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2603_08734_amd import ffn, mx4
    if s["op"] == "round_trip":
        return mx4.dequantize(mx4.quantize(s["x"]), s["x"].dtype)
    if s["op"] == "product":
        return mx4.product(mx4.quantize(s["x"]) if s["x4"] else s["x"], s["w"], s["x"].dtype)
    h = ffn.gated(s["x"], s["wg"], s["wu"], s["act"])
    if s["op"] == "gated":
        return h
    return [h.detach(), *torch.autograd.grad(h, (s["x"], s["wg"], s["wu"]), s["dh"])]


# ---------------------------------------------------------------------------
# bounds and the definition in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "round_trip":
        cells = case["rows"] * case["k"]
        # values in, codes and scales, values out
        return {"bytes": 2 * size * cells + case["rows"] * -(-case["k"] // BLOCK) * 17, "flops": 4 * cells}
    if case["op"] == "product":
        t, n, k = case["t"], case["n"], case["k"]
        return {"bytes": size * t * (k + n) + n * -(-k // BLOCK) * 17, "flops": 2 * t * n * k}
    t, d, f = case["t"], case["d"], case["f"]
    if case["op"] == "gated":
        weights = 2 * f * (-(-d // BLOCK) * 17 if case["w4"] else size * d)
        return {"bytes": size * t * (d + f) + weights, "flops": 4 * t * d * f}
    # X, dH and both weights in; H, dX and both gradients out
    return {"bytes": size * (2 * t * d + 2 * t * f + 4 * f * d), "flops": 12 * t * d * f}


def _exact_quantised(x):
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    rows, k = x.shape
    out = torch.empty((rows, k), dtype=torch.float64, device=x.device)
    slab = max(1, (1 << 25) // k)
    for a in range(0, rows, slab):
        v = torch.nn.functional.pad(x[a:a + slab].double(), (0, -k % BLOCK)).unflatten(1, (-1, BLOCK))
        top = v.abs().amax(dim=2, keepdim=True)
        scale = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2)
        # log2 of a number just below a power of two may round up to it
        scale = torch.where(top < 4 * scale, scale / 2, scale)
        scale = torch.where(top >= 8 * scale, scale * 2, scale).clamp(2.0 ** -127, 2.0 ** 127)
        m = (v.abs() / scale).contiguous()
        down, up = torch.bucketize(m, middle), torch.bucketize(m, middle, right=True)   # they differ at a tie
        code = torch.where(down % 2 == 0, down, up)
        out[a:a + slab] = (torch.sign(v) * grid[code] * scale).flatten(1)[:, :k]
    return out


def _exact_values(codes, scales, k):
    c = torch.stack([codes % 16, codes // 16], dim=2).flatten(1).to(torch.int16)
    low, field = c % 2, c // 2 % 4
    m = torch.where(field == 0, 0.5 * low, (1 + 0.5 * low) * torch.exp2(field.double() - 1))
    m = torch.where(c >= 8, -m, m).double()
    return (m.unflatten(1, (-1, BLOCK)) * torch.exp2(scales.double() - 127).unsqueeze(2)).flatten(1)[:, :k]


def exact(case, seed):
    global own
    mode, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mode
    x = s["x"]
    if case["op"] == "round_trip":
        return _exact_quantised(x)
    if case["op"] == "product":
        return (_exact_quantised(x) if case["x4"] else x.double()) @ _exact_values(*s["w"], case["k"]).t()
    x = x.double()
    wg, wu = (_exact_values(*s[n], case["d"]) if case.get("w4") else s[n].double() for n in ("wg", "wu"))
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.nn.functional.relu}[case["act"]]
    if case["op"] == "gated":
        return act(x @ wg.t()) * (x @ wu.t())
    for t in (x, wg, wu):
        t.requires_grad_()
    h = act(x @ wg.t()) * (x @ wu.t())
    return [h.detach(), *torch.autograd.grad(h, (x, wg, wu), s["dh"].double())]
