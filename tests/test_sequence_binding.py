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


def wide(*shape):
    """A tensor of any shape without its memory."""
    return torch.zeros(1, dtype=torch.bfloat16).expand(*shape)


FAR = (1 << 32) + 8  # 8 in 32 bits


@pytest.mark.parametrize("call", [
    lambda x: bla.window_forward(x, x, x, FAR),
    lambda x: bla.window_forward(x, x, x, 8, FAR),
    lambda x: bla.window_forward(x, x, x, 8, t0=1 << 64),
    lambda x: bla.window_backward(x, x, x, x, x, x, FAR),
    lambda x: bla.window_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], FAR, 0, x, x),
    lambda x: bla.window_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], 8, 0, x, x, t0=(1 << 64) + 3),
    lambda x: bla.window_forward(*[wide(1, 2, FAR, 32)] * 3, 8),
    lambda x: bla.conv_forward(wide(1, 2, FAR, 32), torch.zeros(2, 32, 4)),
    lambda x: bla.conv_forward(x, torch.zeros(2, 32, 4), silu=1 << 32),
    lambda x: bla.conv_step(wide(FAR, 2, 32), torch.zeros(2, 32, 4), x),
    lambda x: bla.ssm_forward(wide(1, 2, FAR, 32), x, x, wide(1, 1, FAR, 16), wide(1, 1, FAR, 16)),
    lambda x: bla.ssm_step(wide(FAR, 2, 32), x, x, wide(FAR, 1, 16), wide(FAR, 1, 16), x),
])
def test_values_past_their_fields(lib, call):  # noqa: F811
    """Sizes and positions that the parameter block cannot hold are refused; they are not taken by their lower bits."""
    with pytest.raises(bla.BlaError):
        call(torch.zeros(1, 2, 8, 32, dtype=torch.bfloat16))
