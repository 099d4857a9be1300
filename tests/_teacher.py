"""Teachers whose probabilities do not add up to 1, and the distillation loss differentiated."""
import numpy as np
import torch


def bf16_teacher(N, V, K, T, seed):
    """The largest K of V logits a row in bf16, and the log-sum-exp of the exact ones, as a server returns them:
    ids [N, K] int32, logits [N, K] bf16, log-sum-exp [N] fp32."""
    g = torch.Generator().manual_seed(seed)
    z = T * (20 + 4 * torch.randn(N, V, generator=g, dtype=torch.float64))
    top, ids = torch.topk(z, K, dim=1)
    return ids.int().numpy(), top.bfloat16(), torch.logsumexp(z / T, 1).float().numpy()


def distill_autograd(H, W, ids, a, T, lse, G):
    """Loss, dH and dW in fp64 by differentiating the definition (every row with all its entries)."""
    H, W = (torch.as_tensor(x).double().requires_grad_() for x in (H, W))
    idx, la = torch.as_tensor(ids).long(), torch.as_tensor(lse).double()[:, None]
    logq = torch.log_softmax(H @ W.T / T, 1)
    a = torch.as_tensor(a).double() / T - la
    p = a.exp()
    loss = (p * (a - logq.gather(1, idx))).sum(1)
    if ids.shape[1] < W.shape[0]:
        rho = (1 - p.sum(1)).clamp(min=0)
        rest = torch.logsumexp(logq.scatter(1, idx, -torch.inf), 1)
        loss = loss + torch.where(rho > 0, rho * (torch.log(rho.clamp(min=1e-300)) - rest), 0.0)
    (torch.as_tensor(G).double() * loss).sum().backward()
    return loss.detach().numpy(), H.grad.numpy(), W.grad.numpy()
