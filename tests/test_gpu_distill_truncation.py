"""How far the fp32 dW of up to 64 rows of a bf16 head is off where a student has large logits outside the entries.

dZ = g e^(z - lse_rest) (m q_rest - rho) is stored to 2^-16 of itself. The backward's z come from one accumulator over
all of h: h / 16 truncated additions, each by up to 2u of a partial sum that is half of S = sum |H W| on average
(u = 2^-24), so (h / 16) u S; lse_rest has the forward's (32 + h / 256) u S (see test_gpu_distill.py); exponentials, the
row's factor, and sums over at most 128 rows of products another 64 u (1 + |z|). In the 2-norm the errors of the
elements bound that of dW, which is the sum of at most one large dZ row by a row of H."""
import pytest
import torch

from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("h", [512, 2048, 6144])
@pytest.mark.parametrize("N", [3, 16, 64])
@pytest.mark.parametrize("z0", [0.0, 12.0, 24.0])
def test_dW_of_few_rows(N, h, z0):
    V, K = 3000, 8
    g = torch.Generator(device="cuda").manual_seed(N + h)
    W = (torch.randn(V, h, generator=g, device="cuda") * 0.02).bfloat16()
    H = torch.randn(N, h, generator=g, device="cuda")
    out = W[2000:2000 + N].float()  # a column outside the entries for each row
    H = (H + out * (z0 / out.square().sum(1, keepdim=True))).bfloat16()
    ids = (torch.arange(K, device="cuda") * 97 + torch.arange(N, device="cuda")[:, None] * 13) % 1900
    a = torch.randn(N, K, generator=g, device="cuda")
    lse_t = torch.logsumexp(a, 1) + 0.5
    loss, lse, rest = (torch.empty(N, device="cuda") for _ in range(3))
    z_top, dH, dW = torch.empty(N, K, device="cuda"), torch.empty_like(H), torch.empty(V, h, device="cuda")
    ws = sao.distill_workspace(N, h, V, K)
    top = ids.int().contiguous()
    sao.sao_distill_loss_fwd(H, W, top, a, 1.0, loss, lse, rest, z_top, ws, teacher_lse=lse_t)
    sao.sao_distill_loss_bwd(H, W, top, a, 1.0, lse, rest, z_top, torch.ones(N, device="cuda"), dH, dW, ws,
                             teacher_lse=lse_t)
    Hd, Wd = H.double(), W.double()
    z = Hd @ Wd.T
    p = torch.exp(a.double() - lse_t.double()[:, None])
    outside = torch.ones_like(z, dtype=torch.bool).scatter_(1, ids, False)
    lr, l = torch.logsumexp(z.masked_fill(~outside, -torch.inf), 1), torch.logsumexp(z, 1)
    dz = torch.exp(z - lr[:, None]) * (torch.exp(lr - l) - (1 - p.sum(1)))[:, None]
    dz.scatter_(1, ids, torch.exp(z.gather(1, ids) - l[:, None]) - p)
    want = dz.T @ Hd
    S = (Hd.abs() @ Wd.abs().T).max().item()
    tol = 2.0 ** -16 + ((h / 16 + 32 + h / 256) * S + 64 * (1 + z.abs().max().item())) * U
    assert ((dW.double() - want).norm() / want.norm()).item() <= tol
