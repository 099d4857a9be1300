"""The norm's sum of squares where each addition of a long chain is rounded the same way: 256 columns of 1, others whose
square is a little more than half a unit in the last place of 1. rstd within the 32 u of test_gpu_norm.py."""
import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests.test_gpu_norm import check_forward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ones", [32, 64, 128, 256])
@pytest.mark.parametrize("h", [1999, 2048, 4099, 8192, 12289, 16119, 16379, 16384])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_squares_that_are_rounded_one_way(dtype, h, ones):
    x = torch.full((3, h), 2.0 ** -12 * (1 + (2.0 ** -12 if dtype is torch.float32 else 2.0 ** -7)))
    x[:, :ones] = 1.0
    c = {"x": x.to(dtype).cuda(), "residual": None, "weight": torch.ones(h, device="cuda")}
    check_forward(c, forward(c, 0.0), 0.0)
