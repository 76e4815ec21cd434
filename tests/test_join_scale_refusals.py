"""A join's scale with dropout, at the C boundary: refused before anything is launched, so no GPU is needed."""
import ctypes

import pytest

from paper_2603_08734_amd import binding as b
from test_edge_refusals import P, _drop, _gradients, _join


@pytest.mark.parametrize("scale,share", [(2.0 ** 127, 32768), (-(2.0 ** 126), 50000), (2.0 ** 112, 65535)])
def test_scale_that_leaves_the_range_with_dropout(scale, share):
    join = _join(scale=scale, drop=_drop(share))
    assert b.lib().rsh_join_forward(ctypes.byref(join), None) == b.RSH_ERR_BAD_OPTION
    assert b.lib().rsh_join_backward(ctypes.byref(join), ctypes.byref(_gradients()), None) == b.RSH_ERR_BAD_OPTION


@pytest.mark.parametrize("scale,share", [(2.0 ** 127, 0), (2.0 ** 126, 32767), (2.0 ** 111, 65535), (2.0 ** 127, 65536)])
def test_scales_that_do_not(scale, share):
    """What is missing next is what is refused."""
    join = _join(scale=scale, drop=_drop(share), before=b.rsh_norm_t(P, None, None, b.RSH_F32, b.RSH_F32, b.RSH_NORM_RMS, 1e-5))
    assert b.lib().rsh_join_backward(ctypes.byref(join), ctypes.byref(_gradients()), None) == b.RSH_ERR_NULL
