"""Groups kept by the sum of their two best experts, where a group's second and third best are nearly equal: the sum is
of the larger one, however few bits they differ in. Choices are compared with fp64, weights within the bounds of
test_gpu_route.py.

Sums of a softmax are told apart by fp64 wherever the logits differ; sigmoids are 1 to all digits for logits past 36 or so,
so those rows lie about 0 and 8, where a step of a logit moves a score by 5e-8 and 3e-10."""
import pytest
import torch

from paper_2607_07508_gb300 import sao  # noqa: F401
from tests.test_gpu_route import check

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -22  # of a logit about 2
N = 2503           # eight lanes to a row from 16 tokens for each SM on


def _raised(x, by):
    """x, moved up by whole steps of its own."""
    return (x.view(torch.int32) + by.int()).view(torch.float32)


@pytest.mark.parametrize("score,other", [("softmax", 100), ("sigmoid", 200)])
def test_the_larger_of_two_near_logits_counts(score, other):
    """Group 0 has the better two, the second of them behind a smaller one that shares its leading bits."""
    x = torch.full((N, 256), -3.0)
    x[:, 0], x[:, 1], x[:, 2], x[:, 32], x[:, 33] = 2.5, 2.0, 2 + 250 * STEP, 2.5, 2 + other * STEP
    ids, _ = check(x.cuda(), 4, score, groups=8, kept=1, two=True, train=False)
    assert ids[0].tolist() == [0, 2, 1, 3]


@pytest.mark.parametrize("score,offset", [("softmax", 0), ("softmax", 30), ("softmax", 100), ("sigmoid", 0), ("sigmoid", 8)])
@pytest.mark.parametrize("E,groups,kept,k", [(128, 8, 3, 8), (128, 2, 1, 5), (256, 8, 4, 8), (256, 4, 1, 3), (512, 8, 1, 8),
                                             (512, 2, 1, 1), (64, 8, 7, 4), (128, 4, 3, 8)])
def test_second_and_third_best_of_near_logits(E, groups, kept, k, score, offset):
    """Every group: one best logit, the same for all of them, a second and a third 1 to 511 steps above another common one."""
    g = torch.Generator().manual_seed(E + groups + offset)
    size = E // groups
    x = torch.randn(N, groups, size, generator=g).clamp(max=1.5) + offset
    places = torch.rand(N, groups, size, generator=g).argsort(2)[:, :, :3]
    common = 2.0 + torch.rand(N, 1, 1, generator=g) + offset
    steps = torch.randint(1, 512, (N, groups, 2), generator=g)
    steps[::3, :, 1] = steps[::3, :, :1].squeeze(2) + torch.randint(-1, 2, steps[::3, :, 0].shape, generator=g)
    near = _raised(common.expand(N, groups, 2).contiguous(), steps)
    x.scatter_(2, places, torch.cat([torch.full((N, groups, 1), offset + 3.5), near], 2))
    check(x.view(N, E).cuda(), k, score, groups=groups, kept=kept, two=True, train=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,kept", [(128, 2, 1), (256, 4, 3), (512, 8, 2)])
def test_more_near_logits_than_a_list_holds(E, groups, kept, score):
    """All of a group's logits within 511 steps of one another, or all but its best."""
    g = torch.Generator().manual_seed(E)
    x = _raised(torch.full((N, E), 2.0), torch.randint(0, 512, (N, E), generator=g))
    best = torch.arange(N) % 2 == 0
    x[best] = x[best].view(-1, groups, E // groups).index_fill(2, torch.tensor([E // groups - 1]), 2.5).view(-1, E)
    check(x.cuda(), 8, score, groups=groups, kept=kept, two=True, train=False)
