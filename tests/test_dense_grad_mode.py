"""What the differentiable forms ask of the forward where no gradient can follow: no z, no statistics (no GPU: the
forwards are replaced by records of their calls)."""
import pytest
import torch

from paper_2609_08443_gb300 import binding

MODES = {"no_grad": torch.no_grad, "inference": torch.inference_mode}


@pytest.fixture
def asked(monkeypatch):
    """(call, whether it was asked for what its gradient takes) of every forward"""
    calls = []

    def linear(x, weight, bias=None, activation=None, residual=None, want_pre=False, ws=None):
        calls.append(("linear", want_pre))
        y = x.new_ones((*x.shape[:-1], weight.shape[0]))
        return (y, y.clone()) if want_pre else y

    def norm(x, weight=None, bias=None, residual=None, eps=1e-5, dtype=None, want_stats=False):
        calls.append(("norm", want_stats))
        y = torch.ones_like(x)
        return (y, x.new_ones((*x.shape[:-1], 2))) if want_stats else y

    monkeypatch.setattr(binding, "sa_linear_fwd", linear)
    monkeypatch.setattr(binding, "sa_layer_norm_fwd", norm)
    return calls


def parameters(grad=True):
    return (torch.nn.Parameter(torch.ones(4, 8), requires_grad=grad), torch.nn.Parameter(torch.ones(8), requires_grad=grad))


@pytest.mark.parametrize("mode", MODES)
def test_without_gradients(asked, mode):
    w, v = parameters()
    x = torch.ones(3, 8)
    with MODES[mode]():
        y = binding.sa_linear(x, w, activation="silu")
        n = binding.sa_layer_norm(x, v, residual=x)
    assert asked == [("linear", False), ("norm", False)] and not y.requires_grad and not n.requires_grad


def test_without_leaves(asked):
    w, v = parameters(False)
    x = torch.ones(3, 8)
    assert not binding.sa_linear(x, w, activation="silu").requires_grad
    assert not binding.sa_layer_norm(x, v).requires_grad
    assert asked == [("linear", False), ("norm", False)]


def test_with_gradients(asked):
    w, v = parameters()
    x = torch.ones(3, 8)
    assert binding.sa_linear(x, w, activation="silu").requires_grad
    assert binding.sa_layer_norm(x, v).requires_grad
    r = torch.ones(3, 4, requires_grad=True)
    assert binding.sa_linear(x, w.detach(), activation="silu", residual=r).requires_grad  # its gradient is dy
    assert asked == [("linear", True), ("norm", True), ("linear", False)]
