"""Which calls of a MoeTrainLayer leave a backward pass possible: host logic, with a stand-in for the library's context.

backward() joins what forward_train() kept with the layer's tables and buffers.  Every call that writes those for another
batch or another plan has to make it refuse.
"""
import pytest
import torch

from paper_2506_07366_b200 import binding, layer as layer_module
from paper_2506_07366_b200.layer import MoeTrainLayer

SHAPE = binding.Shape(T=4, D=8, F=8, E=2, K=1, S=2, row_align=1)


class StandIn:
    """Takes every call of a Context and remembers its name; calls named in `refuse` raise."""

    def __init__(self, *_):
        self.calls, self.refuse = [], ()

    def __getattr__(self, name):
        def call(*args, **kwargs):
            self.calls.append(name)
            if name in self.refuse:
                raise ValueError(name)
        return call


@pytest.fixture
def layer(monkeypatch):
    monkeypatch.setattr(layer_module, "Context", StandIn)
    monkeypatch.setattr(layer_module, "workspace_bytes", lambda s: 16)
    monkeypatch.setattr(layer_module, "route_backward_workspace_bytes", lambda s: 16)
    s, bf = SHAPE, dict(dtype=torch.bfloat16)
    layer = MoeTrainLayer(s, torch.zeros(s.E, s.D, **bf), None, torch.zeros(s.E, s.F, s.D, **bf), torch.zeros(s.E, s.F, s.D, **bf),
                          torch.zeros(s.E, s.D, s.F, **bf))
    layer.plan(torch.ones(s.E, dtype=torch.int32))
    return layer


X = torch.zeros(SHAPE.T, SHAPE.D, dtype=torch.bfloat16)
HIST = torch.ones(SHAPE.E, dtype=torch.int32)
BETWEEN = {
    "forward": lambda l: l.forward(X),
    "forward into a buffer": lambda l: l.forward(X, out=torch.empty_like(X)),
    "forward_predicted": lambda l: (l.start_prediction(), l.forward_train(X), l.forward_predicted(X)),
    "forward_host": lambda l: l.forward_host(X, torch.empty_like(X)),
    "plan": lambda l: l.plan(HIST),
    "start_prediction": lambda l: l.start_prediction(),
}


@pytest.mark.parametrize("name", BETWEEN)
def test_backward_refuses_after(layer, name):
    layer.forward_train(X)
    BETWEEN[name](layer)
    before = list(layer.ctx.calls)
    with pytest.raises(RuntimeError, match="forward_train"):
        layer.backward(X)
    assert layer.ctx.calls == before                      # nothing was launched
    layer.forward_train(X)                                # and the next pass works
    layer.backward(X)


def test_backward_refuses_after_a_forward_pass_that_failed_on_its_way(layer):
    for call in (layer.forward_train, layer.forward):
        layer.ctx.refuse = ()
        layer.forward_train(X)
        layer.ctx.refuse = ("combine",)                   # by then the tables are the new batch's
        with pytest.raises(ValueError):
            call(X)
        with pytest.raises(RuntimeError, match="forward_train"):
            layer.backward(X)


def test_backward_may_be_tried_again(layer):
    layer.forward_train(X)
    layer.ctx.refuse = ("combine_backward",)
    with pytest.raises(ValueError):
        layer.backward(X)
    layer.ctx.refuse = ()
    layer.backward(X)
