"""One training step of a mixture-of-experts policy with its auxiliary losses, on synthetic data.

The rows of one packed batch serve three objectives at once, as in a run that distils from a teacher beside RL:

  RL            advantages, log-probs of the sampled tokens, policy loss and its gradient, value loss
  distillation  KL to a teacher's top logits on the action tokens, over the same hidden states and LM head
  balance       load balance of the router, each trajectory by itself, over all tokens

The LM head's gradient is one fp32 buffer: the RL backward writes it, the distillation backward adds to it; the
hidden states' gradients are summed.

`whole_step` has what lies in front of and behind those losses too: the router's choice of experts, whose outputs join
the residual stream, the norm in front of the head, their gradients, and the clipping of all of them by their norm.
Run it as `python -m examples.moe_policy_step`.
"""
from __future__ import annotations

import torch

from paper_2607_07508_gb300 import sao, synthetic as S

DISTILL_WEIGHT, BALANCE_WEIGHT = 0.5, 0.01
EPS, MAX_NORM, ROUTE_SCALE = 1e-6, 0.1, 2.5
TEMPERATURE, TOP, EXPERTS, CHOSEN = 2.0, 20, 16, 2


def batch(device="cuda", seed=7):
    """A packed batch: the RL inputs, a teacher's answers and a router's logits and choices."""
    wl = S.make_custom([300, 0, 157, 64], 256, 1000, "bf16", seed=seed, device="cpu", obs_frac=0.25)
    g = torch.Generator().manual_seed(seed)
    dev = lambda x: torch.as_tensor(x).to(device)
    b = {"H": dev(wl.H), "W": dev(wl.W), "y": dev(wl.y), "mask": dev(wl.loss_mask), "cu": dev(wl.cu_seqlens),
         "values": dev(wl.values), "rewards": dev(wl.rewards), "xi": dev(wl.xi), "wl": wl}
    # what an inference server returns: the teacher's largest logits and its log-sum-exp over the vocabulary
    teacher = (wl.H.float() @ wl.W.float().t() + 0.5 * torch.randn(wl.N, wl.V, generator=g)) / TEMPERATURE
    top, ids = torch.topk(teacher * TEMPERATURE, TOP, dim=1)
    b["top_logits"], b["top_ids"] = dev(top), dev(ids.int())
    b["teacher_lse"] = dev(torch.logsumexp(teacher, 1))
    router = torch.randn(wl.N, EXPERTS, generator=g) + torch.linspace(-1, 1, EXPERTS)
    b["router"] = dev(router.bfloat16())
    b["experts"] = dev(torch.topk(router, CHOSEN, dim=1).indices.int())
    return b


def step(b):
    """The step's losses and gradients."""
    wl, H, W, mask = b["wl"], b["H"], b["W"], b["mask"]
    N, h, V = wl.N, wl.h, wl.V
    B, K, E = len(wl.rewards), b["top_ids"].shape[1], b["router"].shape[1]
    f = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device=H.device)
    ws = sao.workspace(N, h, V, H.dtype, device=H.device)
    actions = int(mask.sum())

    # RL
    adv, ret, logp, lse, grad_logp = (f(N) for _ in range(5))
    loss, counts, one = f(1), f(4, dtype=torch.int64), torch.ones(1, device=H.device)
    dH, dW = torch.empty_like(H), f(V, h)
    sao.sao_advantages(b["values"], b["rewards"], mask, b["cu"], wl.gamma, wl.lam, wl.lam_critic, wl.alpha, adv, ret, ws)
    sao.sao_token_logprobs_fwd(H, W, b["y"], logp, lse, ws, row_mask=mask)
    old = logp + b["xi"]
    sao.sao_policy_loss_fwd(logp, old, adv, mask, wl.eps_low, wl.eps_high, loss, counts, ws)
    sao.sao_policy_loss_bwd(logp, old, adv, mask, wl.eps_low, wl.eps_high, one, grad_logp, ws)
    sao.sao_token_logprobs_bwd(H, W, b["y"], lse, grad_logp, dH, dW, ws)

    # distillation on the action tokens; T^2 keeps its gradients at the scale of temperature 1
    kl, kl_lse, kl_rest, z_top = f(N), f(N), f(N), f(N, K)
    kl_dH = torch.empty_like(H)
    kl_ws = sao.distill_workspace(N, h, V, K, H.dtype, device=H.device)
    weight = mask.float() * (DISTILL_WEIGHT * TEMPERATURE ** 2 / actions)
    sao.sao_distill_loss_fwd(H, W, b["top_ids"], b["top_logits"], TEMPERATURE, kl, kl_lse, kl_rest, z_top, kl_ws,
                             teacher_lse=b["teacher_lse"], row_mask=mask)
    sao.sao_distill_loss_bwd(H, W, b["top_ids"], b["top_logits"], TEMPERATURE, kl_lse, kl_rest, z_top, weight, kl_dH, dW,
                             kl_ws, teacher_lse=b["teacher_lse"], accumulate_dW=True)

    # the router, each trajectory balanced by itself
    bal, sums, d_router = f(1), f(B, E), torch.empty_like(b["router"])
    load, rows = f(B, E, dtype=torch.int64), f(B, dtype=torch.int64)
    bal_ws = sao.balance_workspace(N, E, B, device=H.device)
    sao.sao_balance_loss_fwd(b["router"], b["experts"], sao.SAO_SCORE_SOFTMAX, bal, load, sums, rows, bal_ws,
                             cu_seqlens=b["cu"])
    sao.sao_balance_loss_bwd(b["router"], CHOSEN, sao.SAO_SCORE_SOFTMAX, load, rows,
                             torch.full_like(bal, BALANCE_WEIGHT), d_router, bal_ws, cu_seqlens=b["cu"])
    return {"policy": loss, "old": old, "adv": adv, "distill": (kl * weight).sum(), "balance": BALANCE_WEIGHT * bal,
            "load": load, "grad_logp": grad_logp, "kl": kl, "weight": weight, "dH": dH.float() + kl_dH.float(),
            "dW": dW, "d_router": d_router}


def layer(b, seed=8):
    """The last layer in front of the head: the stream, a balance bias, what each token's chosen experts answer (here
    drawn, for any choice: the experts' products are not the step's subject) and the norm's weight."""
    wl, E = b["wl"], b["router"].shape[1]
    g = torch.Generator().manual_seed(seed)
    dev = b["H"].device
    return {"residual": wl.H.to(dev), "bias": (0.1 * torch.randn(E, generator=g)).to(dev),
            "answers": torch.randn(wl.N, CHOSEN, wl.h, generator=g).to(b["H"].dtype).to(dev),
            "norm_weight": (1 + 0.2 * torch.randn(wl.h, generator=g)).to(dev)}


def whole_step(b, l):
    """Router, norm, the losses of `step`, and back: the gradients clipped by their global norm."""
    N, E, h = b["router"].shape[0], b["router"].shape[1], l["residual"].shape[1]
    f = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device=l["residual"].device)
    sigmoid = sao.SAO_SCORE_SIGMOID

    # forward: experts and their weights, the stream with their answers, its norm
    route_ws, norm_ws = sao.route_workspace(N, E), sao.norm_workspace(N, h)
    experts, weights = f(N, CHOSEN, dtype=torch.int32), f(N, CHOSEN)
    sao.sao_route_fwd(b["router"], sigmoid, experts, weights, route_ws, bias=l["bias"], groups=4, groups_kept=2,
                      group_score=sao.SAO_GROUP_TOP2, scale=ROUTE_SCALE)
    answer = (weights[:, :, None] * l["answers"].float()).sum(1).to(l["residual"].dtype)
    stream, H, rstd = torch.empty_like(answer), torch.empty_like(answer), f(N)
    sao.sao_rms_norm_fwd(answer, l["norm_weight"], EPS, norm_ws, residual=l["residual"], sum=stream, y=H, rstd=rstd)

    out = step({**b, "H": H, "experts": experts})

    # backward: the stream's gradient, the norm's weight's, the router's (onto the balance loss's)
    dH = out["dH"].to(H.dtype)
    d_stream, d_norm = torch.empty_like(H), f(h)
    sao.sao_rms_norm_bwd(stream, l["norm_weight"], rstd, dH, d_stream, d_norm, norm_ws)
    d_weights = (d_stream.float()[:, None] * l["answers"].float()).sum(2)
    balance_router, d_router = out["d_router"], out["d_router"].clone()
    sao.sao_route_bwd(b["router"], sigmoid, experts, weights, d_weights, d_router, route_ws, scale=ROUTE_SCALE,
                      accumulate=True)

    # one step over all of them
    grads, grad_ws = [out["dW"], d_norm, d_router], sao.grad_workspace()
    clipped = [torch.empty_like(g) for g in grads]
    sumsq, norm, coef = f(1, dtype=torch.float64), f(1), f(1)
    sao.sao_grad_sumsq(grads, sumsq, grad_ws)
    sao.sao_grad_clip(grads, sumsq, MAX_NORM, norm, coef, grad_ws, out=clipped)
    return {**out, "experts": experts, "weights": weights, "answer": answer, "stream": stream, "H": H, "dH_rounded": dH,
            "d_stream": d_stream, "d_weights": d_weights, "d_norm": d_norm, "balance_router": balance_router,
            "d_router": d_router, "norm": norm, "coef": coef, "clipped": clipped}


def main():
    b = batch()
    out = whole_step(b, layer(b))
    torch.cuda.synchronize()
    print("policy loss %.6f  distillation %.6f  balance %.6f" % (out["policy"].item(), out["distill"].item(),
                                                               out["balance"].item()))
    print("tokens per expert", out["load"].sum(0).tolist())
    print("gradient norms: hidden states %.4f  LM head %.4f  router %.6f" % tuple(
        out[k].float().norm().item() for k in ("dH", "dW", "d_router")))
    print("global norm %.4f, clipped by %.4f" % (out["norm"].item(), out["coef"].item()))


if __name__ == "__main__":
    main()
