"""Facts that pin the oracle's auxiliary losses without the code that it checks:
distillation against the log-probs, brute force, divergences' own properties and
differences; balance against its extremes, brute force and differences."""
import numpy as np
import pytest

from oracle import sao_oracle as O


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _distill_case(seed, N=7, h=5, V=23, K=4):
    r = _rng(seed)
    H, W = r.normal(size=(N, h)), r.normal(size=(V, h))
    ids = np.stack([r.permutation(V)[:K] for _ in range(N)]).astype(np.int32)
    return r, H, W, ids, r.normal(size=(N, K)) * 2


def test_one_entry_renormalised_is_cross_entropy():
    r, H, W, ids, a = _distill_case(0, K=1)
    logp, lse = O.token_logprobs(H, W, ids[:, 0])
    G = r.normal(size=len(H))
    got = O.distill_loss(H, W, ids, a, 1.0, grad=G)
    np.testing.assert_allclose(got["loss"], -logp, rtol=1e-12)
    np.testing.assert_allclose(got["lse"], lse, rtol=1e-12)
    dH, dW = O.token_logprobs_bwd(H, W, ids[:, 0], lse, -G)
    np.testing.assert_allclose(got["dH"], dH, rtol=1e-10, atol=1e-13)
    np.testing.assert_allclose(got["dW"], dW, rtol=1e-10, atol=1e-13)


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_entries_that_are_the_whole_vocabulary_give_the_plain_divergence(T):
    r, H, W, ids, a = _distill_case(1, V=6, K=6)
    z = H @ W.T / T
    q = np.exp(z - z.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)
    e = np.exp(a / T)
    p = e / e.sum(1, keepdims=True)
    want = [(p[t] * np.log(p[t] / q[t][ids[t]])).sum() for t in range(len(H))]
    full = np.log(e.sum(1))
    for lse in (None, full):
        got = O.distill_loss(H, W, ids, a, T, teacher_lse=lse)
        np.testing.assert_allclose(got["loss"], want, rtol=1e-10)
        assert (got["lse_rest"] == -np.inf).all()


def test_a_student_that_is_the_teacher_has_no_loss_and_no_gradient():
    r, H, W, ids, _ = _distill_case(2)
    z = H @ W.T
    lse = np.log(np.exp(z).sum(1))
    a = np.take_along_axis(z, ids, 1)
    got = O.distill_loss(H, W, ids, a, 1.0, teacher_lse=lse, grad=np.ones(len(H)))
    np.testing.assert_allclose(got["loss"], 0.0, atol=1e-12)
    np.testing.assert_allclose(got["dH"], 0.0, atol=1e-11)
    np.testing.assert_allclose(got["dW"], 0.0, atol=1e-11)


def test_the_rest_is_one_outcome():
    """Brute force over K + 1 outcomes; the divergence is never negative and at most that of finer outcomes."""
    r, H, W, ids, a = _distill_case(3)
    lse = np.log(np.exp(a).sum(1)) + 0.3
    got = O.distill_loss(H, W, ids, a, 1.0, teacher_lse=lse)
    q = np.exp(H @ W.T)
    q /= q.sum(1, keepdims=True)
    for t in range(len(H)):
        p = np.exp(a[t] - lse[t])
        P, Q = np.append(p, 1 - p.sum()), np.append(q[t][ids[t]], 1 - q[t][ids[t]].sum())
        assert got["loss"][t] == pytest.approx((P * np.log(P / Q)).sum(), rel=1e-10)
        assert got["loss"][t] >= 0
        coarse = O.distill_loss(H[t:t + 1], W, ids[t:t + 1, :2], a[t:t + 1, :2], 1.0, teacher_lse=lse[t:t + 1])
        assert coarse["loss"][0] <= got["loss"][t] + 1e-12


@pytest.mark.parametrize("rest", [False, True])
def test_distill_gradient_against_differences(rest):
    r, H, W, ids, a = _distill_case(4, N=3)
    ids[1, 2] = -1
    lse = np.array([np.log(np.exp(a[t][ids[t] >= 0] / 1.7).sum()) for t in range(3)]) + 0.4 if rest else None
    G = r.normal(size=3)
    f = lambda h_, w_: (G * O.distill_loss(h_, w_, ids, a, 1.7, teacher_lse=lse)["loss"]).sum()
    got = O.distill_loss(H, W, ids, a, 1.7, teacher_lse=lse, grad=G)
    eps = 1e-5
    for X, d, which in ((H, got["dH"], 0), (W, got["dW"], 1)):
        for i in np.ndindex(*X.shape):
            up, down = X.copy(), X.copy()
            up[i] += eps
            down[i] -= eps
            diff = (f(up, W) - f(down, W)) if which == 0 else (f(H, up) - f(H, down))
            assert diff / (2 * eps) == pytest.approx(d[i], rel=1e-6, abs=1e-8)


def test_rows_that_say_nothing_or_are_wrong():
    r, H, W, ids, a = _distill_case(5, N=6)
    ids[0] = -1                       # no entry
    a[1] = -np.inf                    # none of a finite logit
    ids[2, 0] = ids[2, 1]             # twice
    ids[3, 1] = len(W)                # out of range
    mask = np.array([1, 1, 1, 1, 0, 1])
    got = O.distill_loss(H, W, ids, a, 1.0, row_mask=mask, grad=np.ones(6))
    assert got["loss"][0] == 0 and got["loss"][1] == 0 and got["loss"][4] == 0 and got["lse"][4] == 0
    assert np.isnan(got["loss"][[2, 3]]).all() and got["loss"][5] > 0
    assert (got["dH"][:5] == 0).all() and (got["dH"][5] != 0).all()
    # with the teacher's total known, a row without an entry has all its mass outside: the student's, too
    got = O.distill_loss(H[:1], W, ids[:1], a[:1], 1.0, teacher_lse=np.zeros(1), grad=np.ones(1))
    assert got["loss"][0] == pytest.approx(0, abs=1e-14) and np.abs(got["dH"]).max() < 1e-14


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_balance_extremes(score):
    E, N = 4, 8
    even = np.arange(N * 2).reshape(N, 2) % E
    assert O.balance_loss(np.zeros((N, E)), even, score)["loss"] == pytest.approx(1.0)
    x = np.full((N, E), -40.0)
    x[:, 1] = 40.0
    one = O.balance_loss(x, np.full((N, 1), 1), score)
    assert one["loss"] == pytest.approx(E) and one["counts"].tolist() == [[0, N, 0, 0]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_balance_against_loops_and_differences(score):
    r = _rng(6)
    N, E, k = 11, 5, 2
    x = r.normal(size=(N, E))
    ids = r.integers(-1, E, size=(N, k))
    mask = (r.random(N) < 0.7).astype(np.uint8)
    cu = [0, 3, 3, 10, 11]
    mask[0], mask[10] = 1, 0  # of four trajectories one is empty and one masked
    got = O.balance_loss(x, ids, score, mask, cu)
    total, used = 0.0, 0
    for b in range(4):
        on = [t for t in range(cu[b], cu[b + 1]) if mask[t]]
        if not on:
            continue
        used += 1
        for e in range(E):
            f = sum(int(ids[t][j] == e) for t in on for j in range(k)) * E / (k * len(on))
            e_x = np.exp(x) if score == "softmax" else 1 / (1 + np.exp(-x))
            P = sum(e_x[t][e] / e_x[t].sum() for t in on) / len(on)
            total += f * P
    assert used == 2 and got["loss"] == pytest.approx(total / used, rel=1e-12)
    assert got["rows"].tolist() == [int(mask[cu[b]:cu[b + 1]].sum()) for b in range(4)]
    for i in np.ndindex(N, E):
        up, down = x.copy(), x.copy()
        up[i] += 1e-5
        down[i] -= 1e-5
        diff = (O.balance_loss(up, ids, score, mask, cu)["loss"] - O.balance_loss(down, ids, score, mask, cu)["loss"]) / 2e-5
        assert diff == pytest.approx(got["dlogits"][i], rel=1e-6, abs=1e-9)


def test_balance_without_rows_or_scores():
    x = np.zeros((3, 4))
    got = O.balance_loss(x, np.zeros((3, 2), int), "softmax", np.zeros(3))
    assert got["loss"] == 0 and got["rows"].tolist() == [0] and (got["dlogits"] == 0).all()
    x[1] = -np.inf
    got = O.balance_loss(x, np.zeros((3, 2), int), "softmax")
    assert got["sums"][0].tolist() == [0.5] * 4 and got["rows"].tolist() == [3] and (got["dlogits"][1] == 0).all()
