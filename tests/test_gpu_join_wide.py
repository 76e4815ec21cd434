"""Norms and joins of wide rows in every form of their kernels: without biases (the form of a large training step, whose sums and next rows lie
elsewhere), rows that do not fit registers, gradients of one result only, and more rows than workgroups.  Values and bounds as in test_gpu_join.
"""
import pytest
import torch

from oracle import edges
from test_gpu_join import EPS, LEAVES, TYPES, build, check, close, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [1025, 2049, 4100, 8192])
@pytest.mark.parametrize("dtype,params", [("fp16", "fp32"), ("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
def test_without_biases(d, dtype, params, kind, gate):
    check(5, d, kind, dtype, params=params, gate=gate, p=0.2, bias=False)
    check(3, d, kind, dtype, params=params, gate=gate, bias=False)


@pytest.mark.parametrize("d,t", [(1100, 2600), (4100, 700), (8192, 1300)])
@pytest.mark.parametrize("dtype,gate", [("bf16", "vector"), ("fp16", "full")])
@pytest.mark.parametrize("bias", [False, True])
def test_more_rows_than_workgroups(d, t, dtype, gate, bias):
    check(t, d, "rms" if gate == "vector" else "layer", dtype, gate=gate, p=0.1, bias=bias)


@pytest.mark.parametrize("d", [2049, 8200, 16400, 40001])
@pytest.mark.parametrize("after,before", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_every_form_of_long_rows(d, after, before, gate, p):
    for bias in (False, True):
        kind = "layer" if bias else "rms"
        check(3, d, kind, "bf16", params="bf16", after=after, before=before, gate=gate, p=p, bias=bias)
        check(2, d, kind, "fp32", after=after, before=before, gate=gate, p=p, bias=not bias)


def test_more_long_rows_than_workgroups():
    check(700, 8200, "rms", "bf16", gate="full", p=0.1, bias=False)
    check(150, 20000, "layer", "fp16", gate="vector", p=0.1)


@pytest.mark.parametrize("d", [50, 2049, 8192, 8200, 20000])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("result", ["S", "Y"])
@pytest.mark.parametrize("bias", [False, True])
def test_gradients_of_one_result(d, dtype, result, bias):
    """The other result's gradient is not given: as zeros, and none for what it does not depend on."""
    from paper_2603_08734_amd import dropout, residual
    T, kind, seed = TYPES[dtype], "layer" if bias else "rms", 5 + d
    m = build(4, d, kind, T, torch.float32, True, True, "vector", 0.2, bias=bias)
    m["dy" if result == "S" else "ds"].zero_()
    want = reference(m, kind, True, True, 0.75, edges.kept(4, d, 0.2, seed, 9), T)
    v = {n: x.cuda() for n, x in m.items()}
    names = [n for n in LEAVES if n in v]
    for n in names:
        v[n].requires_grad_()
    S, Y = residual.join(v["x"], v["b"], after=residual.Norm(kind, v["w_after"], v.get("b_after"), EPS), gate=v["gate"], scale=0.75,
                         drop=dropout.Drop(0.2, seed, 9), before=residual.Norm(kind, v["w_before"], v.get("b_before"), EPS))
    out, given = (S, v["ds"]) if result == "S" else (Y, v["dy"])
    for name, g in zip(names, torch.autograd.grad(out, [v[n] for n in names], given, allow_unused=True)):
        if g is None:
            assert result == "S" and name in ("w_before", "b_before")
            continue
        value, bound = want["d" + name]
        close(g, value, bound, T if name in ("x", "b") else torch.float32, f"d{name} of {result} {dtype}")
