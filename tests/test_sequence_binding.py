"""The Python binding of the window, convolution and scan calls on the host (no GPU needed: the tensors are the CPU's, so every call ends at their
check)."""
import pytest
import torch

import paper_2606_09862_amd as bla
from test_window_abi import lib  # noqa: F401


def test_plans_are_kept_per_shape(lib):  # noqa: F811
    """A decode loop that passes t0 instead of pos, and the pieces of a prompt: one plan for all positions."""
    q, k, ring = torch.zeros(2, 4, 32), torch.zeros(2, 2, 32), torch.zeros(2, 2, 50, 32)
    x, y = torch.zeros(2, 4, 7, 32), torch.zeros(2, 2, 7, 32)
    before = bla._window_plan.cache_info()
    for t0 in range(100):
        with pytest.raises(ValueError, match="on cuda:0"):
            bla.window_step(q, k, k, 47, 3, ring, ring, t0=t0)
        with pytest.raises(ValueError, match="on cuda:0"):
            bla.window_forward(x, y, y, 47, 3, t0=7 * t0)
    after = bla._window_plan.cache_info()
    assert after.misses - before.misses <= 2 and after.currsize - before.currsize <= 2
