"""Rows whose squares are below the range of fp32, with an eps that does not hide them: the bounds of test_gpu_norm.py, to the
least rows whose rstd is an fp32 number."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests.test_gpu_norm import _case, backward, check_backward, check_forward, forward

pytestmark = pytest.mark.gpu

SIZES = [(40, 1000), (41, 20), (700, 33), (39, 1001), (38, 4099), (5, 12289), (1500, 2048), (6, 16384)]


def _small(N, h, dtype, least):
    c = _case(N, h, dtype, residual=False, seed=N + h)
    c["x"] *= torch.exp2(torch.linspace(least, -50, N, device="cuda").round())[:, None]  # (bf16 has the range of fp32)
    c["dsum"].zero_()
    return c


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -130, 2.0 ** -101, 2.0 ** -99])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,h", SIZES)
def test_rows_whose_squares_vanish(N, h, dtype, eps):
    c = _small(N, h, dtype, -110)
    c["x"][0] *= 2.0 ** 110  # ordinary rows among them
    o = forward(c, eps)
    check_forward(c, o, eps)
    check_backward(c, o, *backward(c, o, dw=False), eps=eps)


@pytest.mark.parametrize("scaling", ["row", "block", "mx"])
@pytest.mark.parametrize("N,h", [(40, 1000), (41, 20), (38, 4099)])
def test_eight_bits_of_such_rows(N, h, scaling):
    c = _small(N, h, "f32", -125)
    check_forward(c, forward(c, 0.0, scaling=scaling), 0.0, scaling)


@pytest.mark.parametrize("h", [20, 99, 512, 4099])
def test_rows_past_the_range_of_rstd(h):
    """An rstd past the range of fp32 reads +inf; rows beside it are as ever."""
    c = _small(9, h, "f32", -110)
    clean = forward(c, 0.0)
    c["x"][4] = 0.0
    c["x"][4, 1] = 2.0 ** -149
    o = forward(c, 0.0)
    assert o["rstd"][4].item() == math.inf
    others = [i for i in range(9) if i != 4]
    assert torch.equal(o["y"][others], clean["y"][others]) and torch.equal(o["rstd"][others], clean["rstd"][others])
