"""What the binding hands over besides the weights: the choices of experts, and the router's bias.  The ABI knows neither their sizes nor
their strides, so what does not fit is refused before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2602_15563_amd import kmq

SHAPE, WORKSPACE = 3, 6
I32, F32 = torch.int32, torch.float32


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(kmq, "_stream", lambda: None)


def status(call, *args, **how):
    with pytest.raises(kmq.KmqError) as e:
        call(*args, **how)
    return e.value.status


def route(ids, gates, rows=2, top_k=2, bias=None):
    """Calls whose choices fit are refused for the workspace that they lack."""
    x, w = torch.zeros(rows, 64, dtype=torch.bfloat16), torch.zeros(16, 64, dtype=torch.bfloat16)
    return status(kmq.moe_route, x, 64, rows, w, 16, 64, ids, gates, top_k, bias=bias)


def experts(ids, gates, rows=2, top_k=2):
    a = 1 << 20                                           # never looked at
    m = kmq._MatrixStruct(a, a, a)
    w = kmq.MoeWeights.__new__(kmq.MoeWeights)
    w._struct = kmq._WeightsStruct(m, m, m, 512, 1024, 8, 4)
    w._at = ctypes.addressof(w._struct)
    x = torch.zeros(rows, 512, dtype=torch.bfloat16)
    return status(kmq.moe_experts, w, x, 512, rows, ids, gates, top_k, x, 512)


@pytest.mark.parametrize("call", (route, experts))
@pytest.mark.parametrize("ids,gates", (((1, 2), (2, 2)), ((2, 2), (1, 2)), ((2, 1), (2, 2)), ((3,), (4,)), ((4,), (3,)), ((0, 2), (2, 2))))
def test_choices_that_are_too_few(call, ids, gates):
    assert call(torch.zeros(ids, dtype=I32), torch.zeros(gates, dtype=F32)) == SHAPE


@pytest.mark.parametrize("call", (route, experts))
def test_choices_with_strides(call):
    ids, gates = torch.zeros(2, 2, dtype=I32), torch.zeros(2, 2, dtype=F32)
    for view in (lambda t: t.repeat(1, 2)[:, :2], lambda t: t.repeat(1, 2)[:, ::2], lambda t: t.t(), lambda t: t[:1].expand(2, 2)):
        assert call(view(ids), gates) == SHAPE and call(ids, view(gates)) == SHAPE


@pytest.mark.parametrize("call", (route, experts))
def test_choices_that_fit(call):
    """Also more of them than needed, and parts of a larger tensor that lie in one piece."""
    for rows, top_k in ((2, 2), (1, 4), (4, 1), (3, 1)):
        assert call(torch.zeros(2, 2, dtype=I32), torch.zeros(2, 2, dtype=F32), rows, top_k) == WORKSPACE
    assert call(torch.zeros(9, 2, dtype=I32)[3:5], torch.zeros(8, dtype=F32)[4:]) == WORKSPACE
    assert call(torch.zeros(2, 4, dtype=I32)[:, :2][:1], torch.zeros(2, 4, dtype=F32)[1:, 2:], rows=1) == WORKSPACE


@pytest.mark.parametrize("bias", (torch.zeros(16, dtype=torch.bfloat16), torch.zeros(16, dtype=torch.float64), torch.zeros(16, dtype=I32), torch.zeros(15),
                                  torch.zeros(32)[::2], torch.zeros(1).expand(16)))
def test_a_bias_of_another_type_or_size(bias):
    choice = torch.zeros(2, 2, dtype=I32), torch.zeros(2, 2)
    assert route(*choice, bias=bias) == SHAPE
    assert route(*choice, bias=torch.zeros(16)) == WORKSPACE and route(*choice, bias=torch.zeros(24)[8:]) == WORKSPACE
