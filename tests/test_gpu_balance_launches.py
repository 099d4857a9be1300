"""Which balance forwards take one cluster, and that both forms are right on either side of the limits."""
import numpy as np
import pytest
import torch

from oracle import sao_oracle as O
from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("N,E,one", [(1, 1, True), (512, 8, True), (512, 1000, True), (513, 1024, False),
                                     (3072, 8, True), (3073, 1, False), (3073, 8, False), (4096, 8, False), (1536, 32, True),
                                     (1537, 32, False), (512, 128, True), (513, 128, False), (1024, 128, False)])
def test_one_cluster_where_it_is_the_faster_form(N, E, one):
    g = torch.Generator().manual_seed(N + E)
    x = torch.randn(N, E, generator=g)
    ids = torch.topk(x, min(E, 2), 1).indices.int()
    xd, idd = x.cuda(), ids.cuda()
    loss, sums = torch.empty(1, device="cuda"), torch.empty(1, E, device="cuda")
    counts, rows = torch.empty(1, E, dtype=torch.int64, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
    ws = sao.balance_workspace(N, E)
    sao.sao_profile_reset()
    sao.sao_profile_enable(True)
    try:
        sao.sao_balance_loss_fwd(xd, idd, sao.SAO_SCORE_SOFTMAX, loss, counts, sums, rows, ws)
        launched = set(sao.sao_profile_read())
    finally:
        sao.sao_profile_enable(False)
    assert launched == ({"balance_cluster"} if one else {"balance_partial", "balance_reduce"})
    ref = O.balance_loss(x, ids.numpy(), "softmax")
    rel = (16 + 4 * np.sqrt(N)) * U  # as in test_gpu_balance.py
    assert abs(loss.item() - ref["loss"]) <= rel * ref["loss"] and rows.item() == N
    assert np.array_equal(counts.cpu().numpy(), ref["counts"])
    assert (np.abs(sums.double().cpu().numpy() - ref["sums"]) <= rel * ref["sums"]).all()
