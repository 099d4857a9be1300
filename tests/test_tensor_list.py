"""A TensorList whose tensors have moved to other memory since it was made is refused: its addresses are of memory that is
not theirs any more. The library's call is replaced by one that only counts, so that nothing touches the GPU."""
import pytest
import torch


@pytest.fixture
def sao(monkeypatch):
    from paper_2607_07508_gb300 import sao

    class Lib:
        calls = 0

        def sao_grad_sumsq(self, *a):
            self.calls += 1
            return 0

        sao_grad_clip = sao_grad_sumsq

    lib = Lib()
    monkeypatch.setattr(sao, "load", lambda: lib)
    monkeypatch.setattr(sao, "_ptr", lambda t: t.data_ptr())
    monkeypatch.setattr(sao, "_arg", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(sao, "_current", lambda device: None)
    monkeypatch.setattr(sao, "_stream", lambda s: 0)
    sao.lib = lib
    yield sao
    del sao.lib


def _calls(sao, grads, out=None):
    t, ws = torch.zeros(1), torch.zeros(4096, dtype=torch.uint8)
    return [lambda: sao.sao_grad_sumsq(grads, t, ws), lambda: sao.sao_grad_clip(grads, t, 1.0, t, t, ws, out=out)]


def _moves():
    def data(t):
        t.data = torch.zeros(t.numel())

    return {"set_": lambda t: t.set_(torch.zeros(t.numel())), "data": data, "resize_": lambda t: t.resize_(100000),
            "freed": lambda t: t.untyped_storage().resize_(0)}


@pytest.mark.parametrize("how", sorted(_moves()))
def test_a_moved_tensor_is_refused(sao, how):
    grads, out = [torch.zeros(10), torch.zeros(20)], [torch.zeros(10), torch.zeros(20)]
    lists = sao.TensorList(grads), sao.TensorList(out)
    for call in _calls(sao, *lists):
        call()
    assert sao.lib.calls == 2
    _moves()[how](out[1])
    with pytest.raises(ValueError, match="moved"):
        _calls(sao, *lists)[1]()
    _calls(sao, lists[0])[1]()
    _moves()[how](grads[0])
    for call in _calls(sao, lists[0]):
        with pytest.raises(ValueError, match="moved"):
            call()
    assert sao.lib.calls == 3


def test_values_and_views_may_change(sao):
    grads = [torch.zeros(10), torch.nn.Parameter(torch.zeros(4, 5)), torch.zeros(0)]
    held = sao.TensorList(grads)
    grads[0].fill_(3.0)
    with torch.no_grad():
        grads[1].mul_(2)
    for call in _calls(sao, held) + _calls(sao, grads):
        call()
    assert sao.lib.calls == 4


def test_the_memory_of_a_list_outlives_a_move(sao):
    """No other tensor can come to lie where a moved one was, which its address alone would not tell."""
    grads = [torch.zeros(1 << 18)]
    held, place = sao.TensorList(grads), grads[0].data_ptr()
    grads[0].data = torch.zeros(1)
    others = [torch.zeros(1 << 18) for _ in range(4)]
    assert all(t.data_ptr() != place for t in others)
    grads[0].data = others[0]
    with pytest.raises(ValueError, match="moved"):
        _calls(sao, held)[0]()
