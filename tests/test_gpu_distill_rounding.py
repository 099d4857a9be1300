"""How many roundings to bf16 the gradients of 65 and more rows of a bf16 head lose.

dZ is rounded to bf16 once, and a bf16 output once more. A rounding moves an element of significand m in [1, 2) by
e uniform in +-2^-8 / m, which is sqrt(log2(e) 3 / 8 / 3) 2^-8 = 0.425 2^-8 = 0.00166 of it in the mean square
(significands spread evenly over their logarithm), so independent roundings leave r = 0.00166 of an fp32 dW and
sqrt(2) r = 0.00235 of a bf16 output. With n terms of like weight the mean square scatters by 0.9 / sqrt(n) (a
squared uniform's spread): 700 entries and more make that 3.4 % of the square, 1.7 % of the norm; the weights, which
are not alike, double it. Five of that, and 5 % for the logits' truncation and what the rest of the vocabulary adds:
1.22 r, 1.22 sqrt(2) r. Where a row has one entry, the 32 rows that lose most have second pieces, so the others'
largest losses are cut: no more than that either."""
import numpy as np
import pytest
import torch

from oracle import sao_oracle as O
from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

R = 0.425 * 2.0 ** -8


@pytest.mark.parametrize("N,K", [(140, 5), (256, 5), (512, 3), (700, 1), (2048, 1), (8192, 1), (8200, 1)])
def test_one_rounding_of_dZ_and_one_of_the_output(N, K):
    h, V = 64, 3000
    g = torch.Generator().manual_seed(N)
    H, W = torch.randn(N, h, generator=g).bfloat16(), (torch.randn(V, h, generator=g) * 0.05).bfloat16()
    r = np.random.Generator(np.random.PCG64(N))
    ids = np.stack([r.permutation(V)[:K] for _ in range(N)]).astype(np.int32)
    a = torch.randn(N, K, generator=g)
    G = r.uniform(0.5, 1.5, N).astype(np.float32)
    ref = O.distill_loss(H, W, ids, a, 1.0, grad=G)
    Hd, Wd, idd, ad, Gd = H.cuda(), W.cuda(), torch.from_numpy(ids).cuda(), a.cuda(), torch.from_numpy(G).cuda()
    loss, lse, rest = (torch.empty(N, device="cuda") for _ in range(3))
    z, dH = torch.empty(N, K, device="cuda"), torch.empty_like(Hd)
    ws = sao.distill_workspace(N, h, V, K)
    sao.sao_distill_loss_fwd(Hd, Wd, idd, ad, 1.0, loss, lse, rest, z, ws)
    err = {}
    for dt in (torch.float32, torch.bfloat16):
        dW = torch.empty(V, h, dtype=dt, device="cuda")
        sao.sao_distill_loss_bwd(Hd, Wd, idd, ad, 1.0, lse, rest, z, Gd, dH, dW, ws)
        err[dt] = np.linalg.norm(dW.double().cpu().numpy() - ref["dW"]) / np.linalg.norm(ref["dW"])
    dh = np.linalg.norm(dH.double().cpu().numpy() - ref["dH"]) / np.linalg.norm(ref["dH"])
    assert err[torch.float32] <= 1.22 * R
    assert max(err[torch.bfloat16], dh) <= 1.22 * np.sqrt(2) * R
