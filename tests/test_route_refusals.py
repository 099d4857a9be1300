"""What routing refuses before it touches the GPU, and its plain form by hand."""
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


def _fwd(lib, x=16, dt=F32, bias=None, N=4, E=16, k=2, score=0, groups=1, kept=1, group_score=0, scale=1.0, replay=0, ids=16,
         w=16, ws=256, wsb=1 << 20):
    return lib.sao_route_fwd(P(x), dt, P(bias), None, N, E, k, score, groups, kept, group_score, 1, scale, replay, P(ids),
                             P(w), P(ws), wsb, None)


def _bwd(lib, x=16, dt=F32, N=4, E=16, k=2, score=0, scale=1.0, ids=16, w=16, g=16, dx=16, ws=256, wsb=1 << 20):
    return lib.sao_route_bwd(P(x), dt, None, N, E, k, score, 1, scale, P(ids), P(w), P(g), P(dx), 0, P(ws), wsb, None)


def test_refusals(lib):
    for call in (_fwd, _bwd):
        assert call(lib, E=0) == SHAPE and call(lib, E=1025) == SHAPE and call(lib, k=0) == SHAPE
        assert call(lib, k=17) == SHAPE and call(lib, E=64, k=33) == SHAPE and call(lib, N=-1) == SHAPE
        assert call(lib, N=1 << 31) == SHAPE and call(lib, dt=2) == UNSUPPORTED and call(lib, score=2) == INVALID
        for scale in (float("nan"), float("inf")):
            assert call(lib, scale=scale) == INVALID
        assert call(lib, x=18) == INVALID and call(lib, x=17, dt=BF16) == INVALID and call(lib, ids=18) == INVALID
        assert call(lib, w=18) == INVALID
        for null in ("x", "ids", "w", "ws"):
            assert call(lib, **{null: None}) == INVALID, null
        assert call(lib, ws=64) == INVALID and call(lib, wsb=255) == WORKSPACE
    assert _fwd(lib, groups=0) == SHAPE and _fwd(lib, groups=3) == SHAPE and _fwd(lib, E=66, groups=33) == SHAPE
    assert _fwd(lib, groups=4, kept=0) == SHAPE and _fwd(lib, groups=4, kept=5) == SHAPE
    assert _fwd(lib, groups=8, kept=1, k=3) == SHAPE and _fwd(lib, groups=8, kept=1, group_score=2) == INVALID
    assert _fwd(lib, bias=18) == INVALID
    assert _fwd(lib, N=0, x=None, ids=None, w=None, ws=None) == 0 and _bwd(lib, N=0, x=None, dx=None, ws=None) == 0
    assert _bwd(lib, g=None) == INVALID and _bwd(lib, dx=None) == INVALID and _bwd(lib, g=18) == INVALID
    assert _bwd(lib, dx=18) == INVALID


def test_workspace(lib):
    assert lib.sao_route_workspace_bytes(-1, 8) == 0 and lib.sao_route_workspace_bytes(8, 1025) == 0
    last = 0
    for N in (0, 1, 100, 1 << 20):
        assert last <= lib.sao_route_workspace_bytes(N, 8) <= lib.sao_route_workspace_bytes(N, 9)
        last = lib.sao_route_workspace_bytes(N, 8)


def test_binding_checks_tensors():
    from paper_2607_07508_gb300 import sao
    x, ids, w = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for call in (lambda: sao.sao_route_fwd(x, 0, ids, w, w), lambda: sao.sao_route_fwd(x, 0, ids[:3], w, w),
                 lambda: sao.sao_route_fwd(x, 0, ids[:, 0], w, w), lambda: sao.sao_route_fwd(x.half(), 0, ids, w, w),
                 lambda: sao.sao_route_fwd(x, 0, ids.long(), w, w), lambda: sao.sao_route_fwd(x[0], 0, ids, w, w),
                 lambda: sao.sao_route_bwd(x, 0, ids, w, w, x, w), lambda: sao.sao_route_bwd(x, 0, ids, w[:2], w, x, w)):
        with pytest.raises(ValueError):
            call()


def test_plain_form_by_hand():
    """Groups, ties and what is out, on rows small enough to do by hand."""
    from tests import _route as R
    inf = float("inf")
    x = torch.tensor([[1.0, 2.0, 2.0, 0.0], [-inf, -inf, 3.0, -inf], [0.0, 5.0, 4.0, 4.5]])
    assert R.choose(x, 2, "softmax").tolist() == [[1, 2], [2, -1], [1, 3]]
    assert R.choose(x, 2, "softmax", groups=2, kept=1).tolist() == [[1, 0], [2, -1], [1, 0]]
    assert R.choose(x, 2, "sigmoid", groups=2, kept=1, two=True).tolist() == [[1, 0], [2, -1], [3, 2]]
    assert R.choose(x, 1, "sigmoid", bias=torch.tensor([0.0, -inf, 0.0, 0.5])).tolist() == [[3], [2], [3]]
    on = torch.ones(3, dtype=torch.bool)
    w = R.weights(x, torch.tensor([[1, 2], [2, -1], [0, 0]]), "softmax", True, 3.0, on)
    assert torch.allclose(w, torch.tensor([[1.5, 1.5], [3.0, 0.0], [1.5, 1.5]], dtype=torch.float64))


def test_plain_gradient_against_autograd():
    from tests import _route as R
    g = torch.Generator().manual_seed(0)
    x = torch.randn(5, 9, generator=g, dtype=torch.float64).requires_grad_()
    grad = torch.randn(5, 3, generator=g, dtype=torch.float64)
    on = torch.tensor([True, True, False, True, True])
    for score in ("softmax", "sigmoid"):
        ids = R.choose(x.detach(), 3, score)
        ids[1, 2], ids[3, 1] = -1, ids[3, 0]
        for renorm in (True, False):
            w = R.weights(x, ids, score, renorm, 1.7, on)
            want, = torch.autograd.grad((w * grad).sum(), x)
            got, size = R.gradient(x.detach(), ids, w.detach(), grad, score, renorm, 1.7, on)
            assert torch.allclose(got, want, atol=1e-12) and (size >= got.abs() - 1e-15).all()
