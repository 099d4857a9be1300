"""What the gradient norm and clipping refuse before they touch the GPU."""
import ctypes

import pytest
import torch

P = ctypes.c_void_p
INVALID, SHAPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4


@pytest.fixture(scope="module")
def sao():
    from paper_2607_07508_gb300 import build, sao
    build.build()
    sao.load()
    return sao


def _list(sao, *entries):
    return (sao._Tensor * len(entries))(*entries)


def _sumsq(sao, grads, count=None, sumsq=16, ws=256, wsb=1 << 20):
    return sao.load().sao_grad_sumsq(grads, len(grads) if count is None else count, P(sumsq), P(ws), wsb, None)


def _clip(sao, grads, out=None, count=None, sumsq=16, limit=1.0, norm=16, coef=16, ws=256, wsb=1 << 20):
    return sao.load().sao_grad_clip(grads, out, len(grads) if count is None else count, P(sumsq), limit, P(norm), P(coef),
                                    P(ws), wsb, None)


def test_lists(sao):
    good = (4096, 10, 0)
    for call in (_sumsq, _clip):
        assert call(sao, _list(sao, good), count=-1) == SHAPE
        assert call(sao, None, count=1) == INVALID
        assert call(sao, _list(sao, (4096, 10, 2))) == UNSUPPORTED
        assert call(sao, _list(sao, (4096, -1, 0))) == SHAPE and call(sao, _list(sao, (4096, 1 << 48, 0))) == SHAPE
        assert call(sao, _list(sao, (None, 1, 0))) == INVALID
        assert call(sao, _list(sao, (4098, 1, 0))) == INVALID and call(sao, _list(sao, (4097, 1, 1))) == INVALID
        assert call(sao, _list(sao, good, (8192, 4, 1), good)) == INVALID        # twice
        assert call(sao, _list(sao, (4136, 3, 0), (8192, 4, 1), (4096, 11, 0))) == INVALID
        assert "overlap" in sao.load().sao_last_error_string().decode()
        assert call(sao, _list(sao, good), ws=None) == INVALID and call(sao, _list(sao, good), ws=128) == INVALID
        assert call(sao, _list(sao, good), wsb=255) == WORKSPACE
        assert call(sao, _list(sao, good), sumsq=None) == INVALID
    assert _sumsq(sao, _list(sao, good), wsb=256) == WORKSPACE


def test_clip(sao):
    g = _list(sao, (4096, 10, 0), (8192, 6, 1))
    for limit in (0.0, -1.0, float("nan")):
        assert _clip(sao, g, limit=limit) == INVALID
    assert _clip(sao, g, norm=None) == INVALID and _clip(sao, g, coef=None) == INVALID
    assert _clip(sao, g, _list(sao, (16384, 10, 0), (20480, 5, 1))) == SHAPE
    assert _clip(sao, g, _list(sao, (16384, 10, 0), (20480, 6, 3))) == UNSUPPORTED
    assert _clip(sao, g, _list(sao, (16384, 10, 0), (None, 6, 1))) == INVALID
    # out overlaps another gradient, itself, or its own gradient at another place or in another type
    for out in ([(8192, 10, 0), (20480, 6, 1)], [(16384, 10, 0), (16420, 6, 1)], [(4100, 10, 0), (8192, 6, 1)],
                [(4096, 10, 1), (8192, 6, 1)]):
        assert _clip(sao, g, _list(sao, *out)) == INVALID, out
        assert "overlap" in sao.load().sao_last_error_string().decode()


def test_binding_checks_tensors(sao):
    t = torch.zeros(4)
    for bad in ([t], [t.double()], [torch.zeros(4, 4)[:, ::2]]):
        with pytest.raises(ValueError):
            sao.TensorList(bad)
    empty = sao.TensorList([])
    assert len(empty) == 0
    with pytest.raises(ValueError):
        sao.sao_grad_clip(empty, t, 1.0, t, t, t, out=[t])
    with pytest.raises(ValueError):
        sao.sao_grad_sumsq(empty, t, t)
