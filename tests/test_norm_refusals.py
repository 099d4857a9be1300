"""What the root-mean-square norm refuses before it touches the GPU, and its workspaces."""
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


def _fwd(lib, x=16, residual=None, dt=F32, weight=16, w_dt=F32, eps=1e-6, N=4, h=8, sum=None, y=16, rstd=16, y8=None,
         scales=None, scaling=0, ws=256, wsb=1 << 20):
    return lib.sao_rms_norm_fwd(P(x), P(residual), dt, P(weight), w_dt, eps, N, h, P(sum), P(y), P(rstd), P(y8), P(scales),
                                scaling, P(ws), wsb, None)


def _bwd(lib, sum=16, dt=F32, weight=16, w_dt=F32, rstd=16, dy=16, dsum=None, N=4, h=8, dx=16, dw=16, ws=256, wsb=1 << 20):
    return lib.sao_rms_norm_bwd(P(sum), dt, P(weight), w_dt, P(rstd), P(dy), P(dsum), N, h, P(dx), P(dw), 0, P(ws), wsb,
                                None)


def test_refusals(lib):
    for call in (_fwd, _bwd):
        assert call(lib, h=0) == SHAPE and call(lib, h=16385) == SHAPE and call(lib, N=-1) == SHAPE
        assert call(lib, N=1 << 31) == SHAPE and call(lib, dt=2) == UNSUPPORTED and call(lib, w_dt=-1) == UNSUPPORTED
        assert call(lib, weight=None) == INVALID and call(lib, weight=18) == INVALID and call(lib, rstd=18) == INVALID
        assert call(lib, ws=None) == INVALID and call(lib, ws=64) == INVALID and call(lib, wsb=255) == WORKSPACE
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _fwd(lib, eps=eps) == INVALID
    assert _fwd(lib, x=None) == INVALID and _fwd(lib, y=None) == INVALID
    assert _fwd(lib, x=18) == INVALID and _fwd(lib, y=17, dt=BF16) == INVALID
    assert _fwd(lib, residual=16) == INVALID and _fwd(lib, sum=16) == INVALID
    assert "together" in lib.sao_last_error_string().decode()
    assert _fwd(lib, y8=16) == INVALID and _fwd(lib, y8=16, scales=16) == INVALID and _fwd(lib, scaling=1) == INVALID
    assert _fwd(lib, y8=16, scaling=2) == INVALID and _fwd(lib, scales=16, scaling=3) == INVALID
    assert _fwd(lib, y8=16, scales=16, scaling=4) == INVALID and _fwd(lib, y8=16, scales=18, scaling=1) == INVALID
    for null in ("sum", "rstd", "dy", "dx"):
        assert _bwd(lib, **{null: None}) == INVALID, null
    assert _bwd(lib, dsum=18) == INVALID and _bwd(lib, dw=18) == INVALID
    assert _bwd(lib, wsb=256) == WORKSPACE
    assert _fwd(lib, N=0, x=None, ws=None) == 0 and _bwd(lib, N=0, dw=None, ws=None) == 0


def test_workspaces_do_not_fall(lib):
    for bad in ((-1, 8), (4, 0), (4, 16385)):
        assert lib.sao_norm_workspace_bytes(*bad) == 0
    sizes = [0, 1, 2, 100, 319, 320, 321, 65536, 1 << 30]
    for h in (1, 100, 2048, 16383):
        for a, b in zip(sizes, sizes[1:]):
            assert 256 <= lib.sao_norm_workspace_bytes(a, h) <= lib.sao_norm_workspace_bytes(b, h)
            assert lib.sao_norm_workspace_bytes(a, h) <= lib.sao_norm_workspace_bytes(a, h + 1)


def test_binding_checks_tensors():
    from paper_2607_07508_gb300 import sao
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for call in (lambda: sao.sao_rms_norm_fwd(x, torch.zeros(9), 0.0, x, y=x), lambda: sao.sao_rms_norm_fwd(w, w, 0.0, x),
                 lambda: sao.sao_rms_norm_fwd(x.half(), w, 0.0, x), lambda: sao.sao_rms_norm_fwd(x, w, 0.0, x, y=x),
                 lambda: sao.sao_rms_norm_fwd(x, w, 0.0, x, scaling="rows"), lambda: sao.norm_out8(4, 8, "none", "cpu"),
                 lambda: sao.sao_rms_norm_bwd(x, w, w, x, x, w, x)):
        with pytest.raises(ValueError):
            call()
    y8, scales = sao.norm_out8(3, 130, "block", "cpu")
    assert y8.shape == (3, 130) and scales.shape == (3, 2) and scales.dtype is torch.float32
    assert sao.norm_out8(3, 130, "mx", "cpu")[1].shape == (3, 5) and sao.norm_out8(3, 130, "row", "cpu")[1].shape == (3, 1)
