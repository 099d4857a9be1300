"""The distillation oracle where a teacher's probabilities do not add up to 1: its gradient
against a differentiated restatement of the loss, and against differences of its own loss."""
import numpy as np
import pytest
import torch

from oracle import sao_oracle as O
from tests._teacher import bf16_teacher, distill_autograd


@pytest.mark.parametrize("T", [1.0, 2.0])
def test_bf16_logits_against_the_exact_log_sum_exp(T):
    ids, a, lse = bf16_teacher(60, 300, 20, T, seed=1)
    p = np.exp(a.double().numpy() / T - lse[:, None]).sum(1)
    assert (p > 1.001).sum() >= 3 and (p < 0.999).sum() >= 3  # both sides of 1
    r = np.random.Generator(np.random.PCG64(2))
    H, W, G = r.normal(size=(60, 12)), r.normal(size=(300, 12)), r.normal(size=60)
    got = O.distill_loss(H, W, ids, a, T, teacher_lse=lse, grad=G)
    loss, dH, dW = distill_autograd(H, W, ids, a, T, lse, G)
    np.testing.assert_allclose(got["loss"], loss, rtol=1e-10)
    np.testing.assert_allclose(got["dH"], dH, rtol=1e-9, atol=1e-12)
    np.testing.assert_allclose(got["dW"], dW, rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("off", [-0.05, 0.03])
def test_the_whole_vocabulary_with_another_log_sum_exp(off):
    r = np.random.Generator(np.random.PCG64(3))
    N, V = 6, 9
    H, W, G, a = r.normal(size=(N, 4)), r.normal(size=(V, 4)), r.normal(size=N), r.normal(size=(N, V))
    ids = np.stack([r.permutation(V) for _ in range(N)]).astype(np.int32)
    lse = np.log(np.exp(a).sum(1)) + off
    f = lambda h_, w_: (G * O.distill_loss(h_, w_, ids, a, 1.0, teacher_lse=lse)["loss"]).sum()
    got = O.distill_loss(H, W, ids, a, 1.0, teacher_lse=lse, grad=G)
    eps = 1e-5
    for X, d, which in ((H, got["dH"], 0), (W, got["dW"], 1)):
        for i in np.ndindex(*X.shape):
            up, down = X.copy(), X.copy()
            up[i] += eps
            down[i] -= eps
            diff = (f(up, W) - f(down, W)) if which == 0 else (f(H, up) - f(H, down))
            assert diff / (2 * eps) == pytest.approx(d[i], rel=1e-6, abs=1e-8)


def test_the_best_student_has_no_gradient():
    """Probabilities in proportion to the teacher's entries, whatever those add up to."""
    V, K = 40, 5
    r = np.random.Generator(np.random.PCG64(4))
    ids = r.permutation(V)[:K].astype(np.int32)[None]
    a = r.normal(size=(1, K))
    for mass in (1.0, 1.07, 1.5):
        lse = np.log(np.exp(a).sum(1) / mass)
        H = np.full((1, V), -60.0)
        H[0, ids[0]] = a[0]
        got = O.distill_loss(H, np.eye(V), ids, a, 1.0, teacher_lse=lse, grad=np.ones(1))
        assert np.abs(got["dH"]).max() < 1e-14
