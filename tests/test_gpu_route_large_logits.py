"""Softmax scores of fp32 logits that are large next to their differences: rows whose logits share their leading bits have
the scores of their differences, whichever of them is the largest. Choices equal, weights within the bounds of
test_gpu_route.py (the differences are whole numbers, up to 120)."""
import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests.test_gpu_route import check

pytestmark = pytest.mark.gpu


def _rows(N, E, base, seed):
    return (torch.randint(0, 121, (N, E), generator=torch.Generator().manual_seed(seed)).float() + base).cuda()


@pytest.mark.parametrize("base", [0.0, 2.0 ** 20, 2.0 ** 23, -(2.0 ** 23)])
@pytest.mark.parametrize("N", [300, 2503])
def test_scores_of_large_logits(N, base):
    for E, k in ((96, 8), (256, 8), (257, 3), (512, 5)):
        x = _rows(N, E, base, E)
        for renorm in (False, True):
            check(x, k, "softmax", renorm=renorm, train=False)


@pytest.mark.parametrize("base", [0.0, 2.0 ** 20, 2.0 ** 23, -(2.0 ** 23)])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("N", [300, 2503])
def test_groups_of_large_logits(N, two, base):
    for E, groups, kept, k in ((128, 8, 3, 8), (256, 4, 1, 4), (512, 2, 1, 8)):
        x = _rows(N, E, base, E + groups)
        for renorm in (False, True):
            check(x, k, "softmax", groups=groups, kept=kept, two=two, renorm=renorm, train=False)
