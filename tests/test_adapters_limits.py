"""Low-rank adapters: more tokens than a launch takes are refused before anything runs, so no GPU is needed."""
import ctypes

import pytest

from paper_2603_08734_amd import binding as b
from test_edge_refusals import P, _adapters

MOST = b.RSH_ADAPTERS_MAX_TOKENS


@pytest.mark.parametrize("t", [MOST + 1, 1 << 29, (1 << 31) - 1])
def test_too_many_tokens(t):
    L, n = b.lib(), ctypes.c_int64(-1)
    a = _adapters(t=t)
    assert L.rsh_adapters_forward(ctypes.byref(a), P, None) == b.RSH_ERR_TOO_LARGE
    assert L.rsh_adapters_backward(ctypes.byref(a), P, 32, P, P, P, P, None) == b.RSH_ERR_TOO_LARGE
    assert L.rsh_adapters_kept(t, 3, 8, ctypes.byref(n)) == b.RSH_ERR_TOO_LARGE and n.value == 0
    assert L.rsh_adapters_forward_work(t, 64, 32, 3, 8, 1, ctypes.byref(n)) == b.RSH_ERR_TOO_LARGE and n.value == 0
    assert L.rsh_adapters_backward_work(t, 64, 32, 3, 8, ctypes.byref(n)) == b.RSH_ERR_TOO_LARGE and n.value == 0


def test_the_most_tokens():
    """Sizes are reported for them; the grids of their launches: a tile has 64 tokens and up to 512 threads, and every adapter may end one."""
    n = ctypes.c_int64(-1)
    assert b.lib().rsh_adapters_kept(MOST, b.RSH_ADAPTERS_MAX, 8, ctypes.byref(n)) == 0 and n.value >= 4 * 16 * MOST
    assert (MOST // 64 + b.RSH_ADAPTERS_MAX + 1) * 512 < 1 << 32
