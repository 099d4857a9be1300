"""The example's step: its losses and summed gradients against the oracle's. Bounds as for each operator alone: dZ
rounded to bf16 (2^-9) and the hidden states' gradients again, with a factor of two for their sum."""
import numpy as np
import pytest

from oracle import sao_oracle as O

pytestmark = pytest.mark.gpu


def test_moe_policy_step():
    from examples import moe_policy_step as M
    b = M.batch()
    out = {k: v.double().cpu().numpy() for k, v in M.step(b).items()}
    wl = b["wl"]
    mask = wl.loss_mask
    logp, lse = O.token_logprobs(wl.H, wl.W, wl.y)
    dH, dW = O.token_logprobs_bwd(wl.H, wl.W, wl.y, lse, out["grad_logp"])
    kl = O.distill_loss(wl.H, wl.W, b["top_ids"].cpu(), b["top_logits"].cpu(), M.TEMPERATURE,
                        b["teacher_lse"].cpu().numpy(), mask, out["weight"])
    bal = O.balance_loss(b["router"].cpu(), b["experts"].cpu(), "softmax", None, wl.cu_seqlens)
    pl = O.policy_loss(np.where(mask, logp, 0).astype(np.float32), out["old"].astype(np.float32),
                       out["adv"].astype(np.float32), mask, wl.eps_low, wl.eps_high)
    assert abs(out["policy"][0] - pl["loss"]) <= 1e-4 * abs(pl["loss"]) + 1e-6
    assert abs(out["distill"] - (kl["loss"] * out["weight"]).sum()) <= 1e-4 * abs(out["distill"])
    assert abs(out["balance"][0] - M.BALANCE_WEIGHT * bal["loss"]) <= 1e-5 * M.BALANCE_WEIGHT * bal["loss"]
    assert np.array_equal(out["load"], bal["counts"])
    for got, want in ((out["dH"], dH + kl["dH"]), (out["dW"], dW + kl["dW"]),
                      (out["d_router"], M.BALANCE_WEIGHT * bal["dlogits"])):
        assert np.linalg.norm(got - want) <= 2.0 ** -7 * np.linalg.norm(want)
