"""The sum of squares of a batch whose additions are rounded the same way: a 1, and elements whose square is a little more
than half a unit in the last place of 1. Within the 5 u of the norm of test_gpu_grads.py."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests.test_gpu_grads import U, close, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("every", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_squares_that_are_rounded_one_way(dtype, every):
    """A 32 KB chunk: eight vectors a thread, 256 threads side by side. The first one full, one element of the others; or all of them full."""
    per = 16 // dtype.itemsize
    v = 2.0 ** -12 * (1 + (2.0 ** -12 if dtype is torch.float32 else 2.0 ** -7))
    g = torch.zeros(8, 256, per)
    g[0], g[[1, 2, 4, 6], :, 0] = v, v
    if every:
        g[:] = v
    g[0, :, 0] = 1.0
    g = [g.flatten().to(dtype).cuda()]
    out = [torch.empty_like(g[0])]
    close(g, 3.0, run(g, 3.0, out), out)
