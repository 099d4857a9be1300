"""The gradient norm's scalars have to be aligned to their types: refused before anything touches the GPU."""
from tests.test_grads_refusals import INVALID, _clip, _list, _sumsq, sao  # noqa: F401


def test_scalars_off_their_elements(sao):  # noqa: F811
    good = _list(sao, (4096, 10, 0))
    for off in (1, 2, 4):
        assert _sumsq(sao, good, sumsq=16 + off) == INVALID and _clip(sao, good, sumsq=16 + off) == INVALID
        assert "aligned" in sao.load().sao_last_error_string().decode()
    for off in (1, 2):
        assert _clip(sao, good, norm=16 + off) == INVALID and _clip(sao, good, coef=16 + off) == INVALID
        assert "aligned" in sao.load().sao_last_error_string().decode()
    empty = _list(sao)
    assert _sumsq(sao, empty, sumsq=20) == INVALID and _clip(sao, empty, sumsq=20) == INVALID
