"""The trainer's layer norm as torch differentiates it, with the two calls stood in for by torch operations on the CPU."""
import pytest
import torch

from paper_2509_05207_amd import train


class Calls:
    """rg_layer_norm and its gradients by the formulas; what was asked for is kept."""

    def __init__(self):
        self.wanted = []

    def rg_layer_norm(self, x, weight, bias, eps):
        mean = x.mean(1)
        rstd = 1 / ((x - mean[:, None]).square().mean(1) + eps).sqrt()
        return ((x - mean[:, None]) * rstd[:, None]) * weight + bias, mean, rstd

    def rg_layer_norm_backward(self, dy, x, weight, mean, rstd, want_dx=True, want_dweight=True, want_dbias=True):
        self.wanted.append((want_dx, want_dweight, want_dbias))
        h, q = (x - mean[:, None]) * rstd[:, None], dy * weight
        dx = rstd[:, None] * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True))
        return dx if want_dx else None, (dy * h).sum(0) if want_dweight else None, dy.sum(0) if want_dbias else None


def inputs(*needs):
    g = torch.Generator().manual_seed(0)
    return [torch.randn(s, generator=g, dtype=torch.float64, requires_grad=n) for s, n in zip(((5, 7), (7,), (7,)), needs)]


def test_gradients_are_torchs():
    mine, plain = inputs(True, True, True), inputs(True, True, True)
    (train.layer_norm(Calls())(*mine) ** 3).sum().backward()
    (torch.nn.functional.layer_norm(plain[0], (7,), plain[1], plain[2], 1e-5) ** 3).sum().backward()
    for a, b in zip(mine, plain):
        assert torch.allclose(a.grad, b.grad, rtol=1e-12, atol=1e-12)


def test_a_second_derivative_raises():
    """The gradients come from the library, which torch does not see into: a penalty on them must not go without its term."""
    x, w, b = inputs(True, True, True)
    loss = (train.layer_norm(Calls())(x, w, b) ** 3).sum()
    dx, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        (loss + dx.square().sum()).backward()


@pytest.mark.parametrize("needs", [(False, True, True), (True, False, False), (True, True, False), (False, False, True)])
def test_only_gradients_that_are_asked_for_are_computed(needs):
    calls = Calls()
    at = inputs(*needs)
    train.layer_norm(calls)(*at).sum().backward()
    assert calls.wanted == [needs]
    assert [t.grad is not None for t in at] == list(needs)
