"""Gradient of the balance loss through sigmoid scores of large logits, relative to the slope.

d x = s (1 - sigmoid(x)) (w - sum s w). With u = 2^-24: e^-x is off by (|x| + 4) u of itself (the exponent's rounding,
the exponential), its reciprocal by 4 u, so the slope by (|x| + 16) u; w - sum s w by 24 u max |w|, and it is at most
2 max |w|. In all (2 |x| + 64) u slope max |w|, and 2^-8 of itself where it is written in bf16."""
import numpy as np
import pytest
import torch

from oracle import sao_oracle as O
from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gradient(x, ids, m, cu, score=sao.SAO_SCORE_SIGMOID):
    N, E = x.shape
    B = 1 if cu is None else len(cu) - 1
    xd, idd = x.cuda(), torch.from_numpy(ids).cuda()
    md, cud = (None if v is None else torch.from_numpy(v).cuda() for v in (m, cu))
    loss, sums, dx = torch.empty(1, device="cuda"), torch.empty(B, E, device="cuda"), torch.empty_like(xd)
    counts, rows = torch.empty(B, E, dtype=torch.int64, device="cuda"), torch.empty(B, dtype=torch.int64, device="cuda")
    ws = sao.balance_workspace(N, E, B)
    sao.sao_balance_loss_fwd(xd, idd, score, loss, counts, sums, rows, ws, row_mask=md, cu_seqlens=cud)
    sao.sao_balance_loss_bwd(xd, ids.shape[1], score, counts, rows, torch.ones(1, device="cuda"), dx, ws, row_mask=md,
                             cu_seqlens=cud)
    return dx.double().cpu().numpy()


def check(x, ids, m, cu, bf16):
    ref = O.balance_loss(x, ids, "sigmoid", m, cu)
    got = gradient(x, ids, m, cu)
    v = x.double().numpy()
    slope = ref["s"] / (1 + np.exp(np.minimum(v, 700)))
    tol = (2 * np.abs(np.clip(v, -700, 700)) + 64) * U * slope * np.abs(ref["w"]).max(1, initial=0, keepdims=True)
    d = ref["dlogits"]
    assert (np.abs(got - d) <= tol + (2.0 ** -8 * np.abs(d) if bf16 else 0) + 1e-37).all()
    return got, d


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,lens", [(16, None), (63, None), (160, None), (33, [100, 0, 1, 199]), (256, [140, 160])])
@pytest.mark.parametrize("low,high", [(8.0, 12.0), (12.0, 17.0), (17.0, 30.0), (-3.0, 30.0), (-90.0, -20.0)])
def test_slopes_of_large_logits(E, lens, dtype, low, high):
    g = torch.Generator().manual_seed(E)
    r = np.random.Generator(np.random.PCG64(E))
    N = 300
    x = (low + (high - low) * torch.rand(N, E, generator=g)).to(DT[dtype])
    ids = np.ascontiguousarray(np.argsort(r.random((N, E)) ** 3 * np.arange(1, E + 1), axis=1)[:, :4].astype(np.int32))
    m = (r.random(N) < 0.8).astype(np.uint8)
    cu = None if lens is None else np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    check(x, ids, m, cu, dtype == "bf16")


def test_logits_without_a_slope():
    """Infinities and the type's largest values beside ordinary columns: no slope, no NaN."""
    N, E = 64, 24
    x = torch.randn(N, E, generator=torch.Generator().manual_seed(1)) * 3
    ids = (np.arange(N, dtype=np.int32)[:, None] * np.array([1, 3], np.int32) % 5).astype(np.int32)
    big = torch.finfo(torch.float32).max
    x[:, 3], x[:, 7], x[:, 9], x[:, 11], x[:, 13] = float("inf"), -float("inf"), big, -big, -88.5
    with np.errstate(all="ignore"):
        got, _ = check(x, ids, None, None, False)
    assert (got[:, [3, 7, 9, 11]] == 0).all()
    x[:, :] = -200.0  # no sigmoid that fp32 can hold
    x[:, 7] = -float("inf")
    got, want = check(x, ids, None, None, False)
    assert (got[:, 7] == 0).all() and (want[:, 0] != 0).all()
