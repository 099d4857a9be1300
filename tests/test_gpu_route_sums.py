"""Softmax weights that are not renormalised, and their gradients, where a sum of the row's exponentials is rounded the
same way at each addition: one logit is 0 and the others -16.625, whose exponential is a little more than half a unit
in the last place of 1.

Bounds with u = 2^-24: the differences are exact, so an exponential is off by 2 u (1 unit in the last place), the chosen
one and those of the sum alike; a chain of at most 40 additions by 40 u; the quotient, its product and the scale by 3 u: 50 u of a
weight. A gradient has one more sum of k terms and two more products: 70 u of its terms' absolute values."""
import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests import _route as R
from tests.test_gpu_route import backward, forward

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("replay", [False, True])
@pytest.mark.parametrize("first", [0, 60])
@pytest.mark.parametrize("N,E,k,groups,kept", [(160003, 128, 8, 1, 1), (160003, 100, 3, 1, 1), (9001, 32, 8, 1, 1),
                                               (2503, 512, 8, 1, 1), (2503, 512, 8, 2, 1), (300, 512, 8, 1, 1),
                                               (100, 1024, 32, 1, 1), (100, 1020, 9, 17, 3), (100, 1017, 9, 9, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_score_and_many_small_ones(dtype, N, E, k, groups, kept, first, replay):
    x = torch.full((N, E), -16.625, dtype=dtype, device="cuda")
    x[:, min(first, E - 1)] = 0
    given = torch.arange(k, dtype=torch.int32, device="cuda").repeat(N, 1) * (E // k) if replay else None
    ids, w = forward(x, k, groups=groups, kept=kept, renorm=False, given=given)
    on = torch.ones(N, dtype=torch.bool, device="cuda")
    if not replay:
        assert torch.equal(ids, R.choose(x, k, "softmax", None, groups, kept))
    want = R.weights(x, ids, "softmax", False, 2.5, on)
    assert ((w.double() - want).abs() <= 50 * U * want).all(), float(((w.double() - want).abs() / want).max() / U)
    grad = torch.randn(N, k, generator=torch.Generator().manual_seed(k)).cuda()
    want, size = R.gradient(x, ids, want, grad, "softmax", False, 2.5, on)
    dx = backward(x, ids, w, grad, renorm=False)
    assert ((dx.double() - want).abs() <= 70 * U * size + torch.finfo(dtype).eps / 2 * want.abs()).all()
