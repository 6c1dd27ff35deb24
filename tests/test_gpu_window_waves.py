"""Window attention on batches with enough blocks for 128 queries to a workgroup: every width, with rings and without."""
import pytest
import torch

from test_gpu_window import check_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_prompts(dtype, d):
    check_forward(9, 16, 4, 500, d, 70, 5, dtype, lengths=[500, 0, 1, 128, 129, 499, 77, 500, 300])
    check_forward(33, 16, 16, 100, d, 33, 0, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_prompts_from_rings(dtype, d):
    check_forward(9, 16, 4, 400, d, 90, 4, dtype, pos=[0, 3, 93, 94, 500, -1, 1 << 40, 17, 91], cached=True,
                  lengths=[400, 400, 399, 0, 127, 400, 257, 1, 400])
    check_forward(9, 16, 8, 400, d, 700, 9, dtype, pos=[0, 5, 708, 709, 710, 3000, 200, 1, 9], cached=True)
