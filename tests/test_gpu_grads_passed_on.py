"""Gradients that are passed on as they are keep their bits, a NaN's sign and payload among them, wherever they lie: in a
vector, in a tensor's last elements, in a tensor off 16 bytes."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests.test_gpu_grads import _grads, run

pytestmark = pytest.mark.gpu

NANS = {torch.float32: [0x7FC12345, 0x7F812345, -0x543211], torch.bfloat16: [0x7FC1, 0x7F81, -0x55]}  # (quiet, signalling, negative)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("n", [3, 4097, 8195])
def test_bits_of_a_nan(n, offset, dtype):
    grads = _grads([(n, dtype), (64, dtype)], seed=n, offset=offset)
    words = grads[0].view(torch.int32 if dtype is torch.float32 else torch.int16)
    for i, w in enumerate(NANS[dtype]):
        words[-1 - i] = w
        words[i * 16 % n] = w
    out = [torch.zeros(t.numel() + offset, dtype=dtype, device="cuda")[offset:] for t in grads]
    _, norm, coef = run(grads, 1.0, out)
    assert math.isnan(norm) and math.isnan(coef)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(grads, out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bits_where_nothing_is_clipped(dtype):
    grads = _grads([(1003, dtype), (7, dtype)], seed=2, offset=1)
    grads[0][:3] = torch.tensor([-0.0, 2.0 ** -130, -(2.0 ** -133)])
    out = [torch.zeros(t.numel() + 1, dtype=dtype, device="cuda")[1:] for t in grads]
    assert run(grads, 1e6, out)[2] == 1.0
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(grads, out))
