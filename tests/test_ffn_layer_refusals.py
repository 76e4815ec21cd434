"""Argument checks of the served feed-forward layer, made before anything runs.  No GPU: plans are made without upload, and weights and tokens
lie in host memory."""
import numpy as np
import pytest


def _plan(rows, cols, tokens):
    from paper_2603_08734_amd import Plan
    row_ptr = np.arange(rows + 1, dtype=np.int64)
    return Plan(row_ptr, (np.arange(rows) % cols).astype(np.int32), np.ones(rows, dtype=np.float16), cols, tokens, upload=0)


def test_a_projection_back_of_another_kind_is_refused():
    import torch
    from paper_2603_08734_amd import ffn
    w = torch.zeros((64, 48), dtype=torch.float16)
    for down in (w.t(), None, "codes"):
        with pytest.raises(TypeError, match="W_down"):
            ffn.FeedForward(w, w, down)


def test_a_plan_of_another_width_is_refused():
    import torch
    from paper_2603_08734_amd import ffn
    w = torch.zeros((64, 48), dtype=torch.float16)
    for cols in (63, 65, 48):
        with pytest.raises(ValueError, match="W_down"):
            ffn.FeedForward(w, w, _plan(48, cols, 16))
    with pytest.raises(ValueError, match="W_down"):
        ffn.FeedForward(w[0], w[0], _plan(48, 64, 16))


def test_tokens_are_checked_before_the_block_runs():
    import torch
    from paper_2603_08734_amd import ffn
    w = torch.zeros((64, 48), dtype=torch.float16)
    layer = ffn.FeedForward(w, w, _plan(48, 64, 16))
    for x in (torch.zeros((15, 48), dtype=torch.float16), torch.zeros((16, 48), dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="16 tokens"):
            layer(x)
    for x in (torch.zeros((16, 2, 48), dtype=torch.float16), torch.zeros(48, dtype=torch.float16), 3.0):
        with pytest.raises(ValueError, match="matrix"):
            layer(x)
    with pytest.raises(ValueError, match="X is on cpu"):
        layer(torch.zeros((16, 48), dtype=torch.float16))
