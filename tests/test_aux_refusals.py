"""What the auxiliary losses refuse before they touch the GPU."""
import ctypes

import pytest
import torch

P = ctypes.c_void_p
F32, BF16 = 0, 1
INVALID, SHAPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    from paper_2607_07508_gb300 import build, sao
    build.build()
    return sao.load()


def _dfwd(lib, H=16, W=16, dt=F32, ids=16, a=16, adt=F32, N=4, h=8, V=10, K=2, T=1.0, loss=16, z=16, ws=256, wsb=1 << 30):
    return lib.sao_distill_loss_fwd(P(H), P(W), dt, P(ids), P(a), adt, None, None, N, h, V, K, T, P(loss), P(16), P(16),
                                    P(z), P(ws), wsb, None)


def _dbwd(lib, dt=F32, dw_dt=F32, acc=0, N=4, h=8, dH=16, dW=16, K=2, T=1.0, ws=256, wsb=1 << 30):
    return lib.sao_distill_loss_bwd(P(16), P(16), dt, P(16), P(16), F32, None, P(16), P(16), P(16), P(16), N, h, 10, K, T,
                                    P(dH), P(dW), dw_dt, acc, P(ws), wsb, None)


def test_distill_refusals(lib):
    assert _dfwd(lib, K=0) == SHAPE and _dfwd(lib, K=1025) == SHAPE and _dfwd(lib, N=-1) == SHAPE
    assert _dfwd(lib, V=0) == SHAPE and _dfwd(lib, dt=BF16, h=12) == SHAPE
    assert _dfwd(lib, N=(1 << 31) - 1, V=1 << 30) == SHAPE      # tiles past 32 bits
    assert _dfwd(lib, dt=7) == UNSUPPORTED and _dfwd(lib, adt=2) == UNSUPPORTED
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert _dfwd(lib, T=T) == INVALID and _dbwd(lib, T=T) == INVALID
    for null in ("H", "W", "ids", "a", "loss", "z", "ws"):
        assert _dfwd(lib, **{null: None}) == INVALID, null
    assert _dfwd(lib, dt=BF16, H=18) == INVALID and _dfwd(lib, dt=BF16, W=24) == INVALID
    assert "16-byte" in lib.sao_last_error_string().decode()
    assert _dfwd(lib, ws=128) == INVALID and _dfwd(lib, wsb=256) == WORKSPACE
    assert _dfwd(lib, N=0, H=None, loss=None, ws=None) == 0
    assert _dbwd(lib, dt=F32, dw_dt=BF16) == UNSUPPORTED and _dbwd(lib, dt=BF16, dw_dt=BF16, acc=1) == UNSUPPORTED
    assert "added to" in lib.sao_last_error_string().decode()
    assert _dbwd(lib, dw_dt=5) == UNSUPPORTED and _dbwd(lib, dH=None) == INVALID and _dbwd(lib, dW=None) == INVALID
    assert _dbwd(lib, dt=BF16, dH=8) == INVALID and _dbwd(lib, dt=BF16, dw_dt=BF16, dW=8) == INVALID
    assert _dbwd(lib, wsb=300) == WORKSPACE


def _bfwd(lib, x=16, dt=F32, ids=16, cu=None, B=1, N=4, E=8, k=2, score=0, loss=16, counts=16, ws=256, wsb=1 << 30):
    return lib.sao_balance_loss_fwd(P(x), dt, P(ids), None, P(cu), B, N, E, k, score, P(loss), P(counts), P(16), P(16),
                                    P(ws), wsb, None)


def test_balance_refusals(lib):
    assert _bfwd(lib, E=0, k=0) == SHAPE and _bfwd(lib, E=1025) == SHAPE and _bfwd(lib, k=9) == SHAPE
    assert _bfwd(lib, k=0) == SHAPE and _bfwd(lib, N=-1) == SHAPE and _bfwd(lib, N=1 << 31) == SHAPE
    assert _bfwd(lib, cu=16, B=0) == SHAPE and _bfwd(lib, cu=16, B=-1) == SHAPE
    assert _bfwd(lib, cu=16, B=(1 << 31) - 1, E=1024) == SHAPE
    assert _bfwd(lib, dt=3) == UNSUPPORTED and _bfwd(lib, score=2) == INVALID
    for null in ("x", "ids", "loss", "counts", "ws"):
        assert _bfwd(lib, **{null: None}) == INVALID, null
    assert _bfwd(lib, ws=64) == INVALID and _bfwd(lib, wsb=256) == WORKSPACE
    st = lib.sao_balance_loss_bwd(P(16), F32, None, None, 1, 4, 8, 2, 0, None, P(16), P(16), P(16), P(256), 256, None)
    assert st == INVALID
    st = lib.sao_balance_loss_bwd(P(16), F32, None, None, 1, 4, 8, 2, 0, P(16), P(16), P(16), P(16), P(256), 255, None)
    assert st == WORKSPACE
    assert lib.sao_balance_loss_bwd(None, F32, None, None, 1, 0, 8, 2, 0, None, None, None, None, None, 0, None) == 0


def test_workspaces(lib):
    from paper_2607_07508_gb300 import sao
    assert sao.sao_distill_workspace_bytes(-1, 8, 8, 1) == 0 and sao.sao_distill_workspace_bytes(8, 8, 8, 1025) == 0
    assert sao.sao_balance_workspace_bytes(8, 1025) == 0 and sao.sao_balance_workspace_bytes(8, 64) > 256
    # neither the logits nor dZ for the whole vocabulary
    for N, h, V in ((65536, 2048, 151936), (262144, 6144, 154880)):
        assert sao.sao_distill_workspace_bytes(N, h, V, 64) < 2 * N * V


def test_binding_checks_tensors():
    from paper_2607_07508_gb300 import sao
    H, W = torch.zeros(4, 8), torch.zeros(10, 8)
    ids, a, z = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(4)
    call = lambda **k: sao.sao_distill_loss_fwd(*[k.get(n, v) for n, v in (
        ("H", H), ("W", W), ("ids", ids), ("a", a))], 1.0, z, z, z, torch.zeros(4, 2), torch.zeros(256))
    for k in ({"W": torch.zeros(10, 7)}, {"ids": ids[:3]}, {"a": torch.zeros(4, 3)}, {"a": a.double()},
              {"a": a.half()}, {"H": H.double()}, {}):
        with pytest.raises(ValueError):
            call(**k)
    with pytest.raises(ValueError):
        sao.sao_balance_loss_fwd(H, ids[:2], 0, z, z, z, z, z)
