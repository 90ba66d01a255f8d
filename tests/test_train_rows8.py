"""The trainer's product on held rows as torch differentiates it, with the calls stood in for by torch operations on the CPU."""
import pytest
import torch

from paper_2509_05207_amd import train


class Calls:
    """The calls by their formulas; a held row is a codes' matrix and its scales.  What was asked for is kept."""

    def __init__(self):
        self.wanted, self.tables = [], []

    def rg_quantize_rows(self, x):
        scale = x.detach().abs().amax(1, keepdim=True) / 127
        self.tables.append((torch.round(x.detach() / scale), scale))
        return torch.tensor([len(self.tables) - 1])

    def values(self, held):
        return torch.mul(*self.tables[int(held)])

    def rg_rows8_product(self, x, w, cols, dtype):
        return (self.values(x) @ self.values(w).t()).to(dtype)

    def rg_rows8_product_backward(self, dy, x, w, cols, want_dx=True, want_dweight=True, want_dbias=True, weight_dtype=None):
        self.wanted.append((want_dx, want_dweight, want_dbias))
        return dy @ self.values(w) if want_dx else None, (dy.t() @ self.values(x)).to(weight_dtype) if want_dweight else None, None


def inputs(*needs):
    g = torch.Generator().manual_seed(0)
    return [torch.randn(s, generator=g, dtype=torch.float64, requires_grad=n) for s, n in zip(((5, 7), (3, 7)), needs)]


def test_gradients_are_those_of_what_is_held():
    calls, (x, w) = Calls(), inputs(True, True)
    (train.linear8(calls)(x, w) ** 3).sum().backward()
    plain = [calls.values(t).requires_grad_() for t in range(2)]
    ((plain[0] @ plain[1].t()) ** 3).sum().backward()
    assert torch.allclose(x.grad, plain[0].grad, rtol=1e-12) and torch.allclose(w.grad, plain[1].grad, rtol=1e-12)


@pytest.mark.parametrize("needs", [(False, True), (True, False), (True, True)])
def test_only_gradients_that_are_asked_for_are_computed(needs):
    calls, at = Calls(), inputs(*needs)
    train.linear8(calls)(*at).sum().backward()
    assert calls.wanted == [(*needs, False)] and [t.grad is not None for t in at] == list(needs)


def test_a_second_derivative_raises():
    x, w = inputs(True, True)
    loss = (train.linear8(Calls())(x, w) ** 2).sum()
    dx, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        (loss + dx.square().sum()).backward()


def test_nothing_but_held_rows_is_kept():
    calls, (x, w) = Calls(), inputs(True, True)
    y = train.linear8(calls)(x, w)
    assert all(t.dtype == torch.int64 for t in y.grad_fn.saved_tensors)
