"""Distillation where a teacher's probabilities do not add up to 1 (bf16 logits against the exact log-sum-exp; the
whole vocabulary against another one), against the differentiated definition in fp64.

Bounds: dz = m q - p, so an error of e of q or p is one of e (m q + p) of dz. For a student that is far from its
teacher, of gradients as in test_gpu_distill.py (2^-7 with a bf16 head, dZ and the outputs rounded; 1e-5 fp32). At the
best student dz is 0 and what is left is e (m q + p) = 2 e p: exponents of up to 25 off by 2^-24 of themselves,
exponentials and log-sum-exps by as much, sums of 20, 64 u in all."""
import numpy as np
import pytest
import torch

from paper_2607_07508_gb300 import sao
from tests._teacher import bf16_teacher, distill_autograd

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def run(H, W, ids, a, T, lse, G):
    H, W, a = H.cuda(), W.cuda(), a.cuda().contiguous()
    ids, lse, G = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (ids, lse, G))
    N, h = H.shape
    V, K = W.shape[0], ids.shape[1]
    o = {k: torch.empty(N, device="cuda") for k in ("loss", "lse", "lse_rest")}
    z_top, dH, dW = torch.empty(N, K, device="cuda"), torch.empty_like(H), torch.empty(V, h, device="cuda")
    ws = sao.distill_workspace(N, h, V, K, H.dtype)
    sao.sao_distill_loss_fwd(H, W, ids, a, T, o["loss"], o["lse"], o["lse_rest"], z_top, ws, teacher_lse=lse)
    sao.sao_distill_loss_bwd(H, W, ids, a, T, o["lse"], o["lse_rest"], z_top, G, dH, dW, ws, teacher_lse=lse)
    torch.cuda.synchronize()
    return o["loss"].double().cpu().numpy(), dH.double().cpu().numpy(), dW.double().cpu().numpy()


def near(got, want, tol):
    assert np.linalg.norm(got - want) <= tol * np.linalg.norm(want)


@pytest.mark.parametrize("dtype,N", [("bf16", 1), ("bf16", 3), ("bf16", 64), ("bf16", 70), ("bf16", 400), ("f32", 1),
                                     ("f32", 5), ("f32", 20), ("f32", 300)])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_bf16_logits_against_the_exact_log_sum_exp(dtype, N, T):
    V, K, h = 300, 20, 64
    ids, a, lse = bf16_teacher(400, V, K, T, seed=1)
    p = np.exp(a.double().numpy() / T - lse[:, None].astype(np.float64)).sum(1)
    order = np.argsort(-p)  # the rows with most mass, and the one with least
    pick = np.append(order[:N - 1], order[-1]) if N > 1 else order[:1]
    ids, a, lse = ids[pick], a[torch.from_numpy(pick)], lse[pick]
    g = torch.Generator().manual_seed(N)
    H, W = torch.randn(N, h, generator=g).to(DT[dtype]), (torch.randn(V, h, generator=g) * 0.1).to(DT[dtype])
    G = (1 + np.arange(N) % 3).astype(np.float32)
    loss, dH, dW = distill_autograd(H, W, ids, a, T, lse, G)
    got = run(H, W, ids, a, T, lse, G)
    tol = 2.0 ** -7 if dtype == "bf16" else 1e-5
    near(got[1], dH, tol)
    near(got[2], dW, tol)


@pytest.mark.parametrize("dtype,N", [("bf16", 2), ("bf16", 40), ("bf16", 130), ("f32", 4), ("f32", 100)])
@pytest.mark.parametrize("off", [-0.05, 0.03])
def test_the_whole_vocabulary_with_another_log_sum_exp(dtype, N, off):
    V, h = 257, 48
    g = torch.Generator().manual_seed(N)
    H, W = torch.randn(N, h, generator=g).to(DT[dtype]), (torch.randn(V, h, generator=g) * 0.1).to(DT[dtype])
    a = torch.randn(N, V, generator=g)
    r = np.random.Generator(np.random.PCG64(N))
    ids = np.stack([r.permutation(V) for _ in range(N)]).astype(np.int32)
    lse = (torch.logsumexp(a.double(), 1).numpy() + off).astype(np.float32)
    G = (1 + np.arange(N) % 3).astype(np.float32)
    loss, dH, dW = distill_autograd(H, W, ids, a, 1.0, lse, G)
    got = run(H, W, ids, a, 1.0, lse, G)
    tol = 2.0 ** -7 if dtype == "bf16" else 1e-5
    near(got[1], dH, tol)
    near(got[2], dW, tol)


@pytest.mark.parametrize("N", [1, 4, 8, 9, 200])
@pytest.mark.parametrize("mass", [1.0, 1.001, 1.07, 1.5])
def test_the_best_student_has_no_gradient(N, mass):
    """W is the unit matrix: a student's logits are its H, its dZ its dH."""
    V, K = 300, 20
    g = torch.Generator().manual_seed(N)
    r = np.random.Generator(np.random.PCG64(N))
    ids = np.stack([r.permutation(V)[:K] for _ in range(N)]).astype(np.int32)
    a = torch.randn(N, K, generator=g) * 2
    H = torch.full((N, V), -25.0).scatter_(1, torch.from_numpy(ids).long(), a)
    lse = torch.logsumexp(H.double(), 1)
    p = torch.exp(a.double() - lse[:, None])
    lse = (lse - np.log(mass)).float().numpy() if mass > 1 else lse.float().numpy()
    _, dH, dW = run(H, torch.eye(V), ids, a, 1.0, lse, np.ones(N, np.float32))
    rest = np.ones((N, V), bool)
    np.put_along_axis(rest, ids, False, 1)
    # outside the entries the teacher's mass (sum p > 1: none) is met by e^-25 of the student's
    assert np.abs(dH[rest]).max() <= mass * (np.exp(-25.0) * V + 64 * U)
    got = np.take_along_axis(dH, ids, 1)
    assert (np.abs(got) <= 64 * U * 2 * mass * p.numpy() + mass * np.exp(-25.0) * V).all()
