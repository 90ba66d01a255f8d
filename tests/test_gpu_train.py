"""The trainer that runs the norms, their gradients and the weights' update together, on the schedule's blocks and gathered rows."""
import math

import pytest
import torch

from paper_2509_05207_amd import synth, train

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def workload(name):
    return synth.make_workload(name, device="cuda", feature_device="cuda", remote_device="cuda")


class PlainMuon(train.Muon):
    """The same step out of torch's operations."""

    @torch.no_grad()
    def step(self):
        o = self.options
        for w, m in zip(self.model.weights, self.momenta):
            m.mul_(o["momentum"]).add_(w.grad.float())
            x = w.grad.float() + o["momentum"] * m
            tall = x.shape[0] > x.shape[1]
            x = x.t() if tall else x
            x = x / (x.norm() + 1e-7)
            for _ in range(5):
                a = x @ x.t()
                x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
            x = x.t() if tall else x
            w.copy_(w.float() * (1 - o["lr"] * o["weight_decay"]) - o["lr"] * math.sqrt(max(1.0, w.shape[0] / w.shape[1])) * x)
        for v in self.model.scales + self.model.shifts:
            v -= self.vector_lr * v.grad
        for p in self.model.weights + self.model.scales + self.model.shifts:
            p.grad = None


def plain_norm(x, weight, bias):
    return torch.nn.functional.layer_norm(x.float(), (x.shape[1],), weight, bias, 1e-5).to(x.dtype)


@pytest.mark.parametrize("name", ["small", "mid_bf16"])
def test_learns(rg, name):
    """Padded rows of an even and of an odd width; the loss falls well below that of guessing."""
    W = workload(name)
    model = train.Sage(W.cfg.feat_dim, 64, 8, len(W.cfg.fanout), W.local_rows.dtype)
    optimiser, norm, labels = train.Muon(rg, model), train.layer_norm(rg), train.labels_of(W, 8)
    losses = torch.cat([train.train_epoch(rg, train.Batches(rg, W, e), model, optimiser, labels, norm) for e in range(4)])
    assert bool(losses.isfinite().all())
    # guessing costs ln 8 = 2.08; the classes follow from a node's own row, which the last layer sees: half of it is far above what a few dozen steps reach
    assert float(losses[-3:].mean()) < 0.5 * math.log(8)


def test_first_steps_are_the_plain_ones(rg):
    """Three steps of the same model out of torch's operations: losses that differ by what fp32 rounding does (sums in another order, amplified by the steps'
    products: 1e-5 on an update of size one, 2e-2 a step on weights of size 0.1; 1e-3 leaves a factor of a hundred)."""
    W = workload("small")
    batches = train.Batches(rg, W)
    got = []
    for make, norm in ((train.Muon, train.layer_norm(rg)), (PlainMuon, plain_norm)):
        model = train.Sage(W.cfg.feat_dim, 64, 8, len(W.cfg.fanout), W.local_rows.dtype)
        got.append((train.train_epoch(rg, batches, model, make(rg, model), train.labels_of(W, 8), norm)[:3], [w.detach().clone() for w in model.weights]))
    assert torch.allclose(got[0][0], got[1][0], rtol=1e-3)


class FewBatches(train.Batches):
    steps = 1

    def __len__(self):
        return self.steps


@pytest.mark.parametrize("steps,bound", [(1, 1e-3), (3, 1e-2)])
def test_parameters_are_the_plain_ones(rg, steps, bound):
    """Every weight, scale, shift and momentum of the two models, relative to how far it has come.  Gradients differ by fp32's roundings, 1e-6 of them, which five steps of products multiply by 485 where
    singular values are small: 5e-4 of an update, and as much again for the momentum's share; behind three steps three times that, and what follows from it through the model, for which there is a factor of
    three."""
    W = workload("small")
    batches = FewBatches(rg, W)
    batches.steps = steps
    models, momenta = [], []
    for make, norm in ((train.Muon, train.layer_norm(rg)), (PlainMuon, plain_norm)):
        model = train.Sage(W.cfg.feat_dim, 64, 8, len(W.cfg.fanout), W.local_rows.dtype)
        optimiser = make(rg, model)
        train.train_epoch(rg, batches, model, optimiser, train.labels_of(W, 8), norm)
        models.append([t.detach().double() for t in model.weights + model.scales + model.shifts])
        momenta.append([t.double() for t in optimiser.momenta])
    start = train.Sage(W.cfg.feat_dim, 64, 8, len(W.cfg.fanout), W.local_rows.dtype)
    before = [t.detach().double() for t in start.weights + start.scales + start.shifts]
    assert len(before) == 3 * len(W.cfg.fanout)
    for k, (a, b, s) in enumerate(zip(*models, before)):
        assert float((b - s).norm()) > 0 and float((a - b).norm()) <= bound * float((b - s).norm()), k
    for k, (a, b) in enumerate(zip(*momenta)):
        assert float((a - b).norm()) <= bound * float(b.norm()), k
