"""The trainer on features held in 8 bits and products of held rows: store, cache, gather, reading back, norms, products, gradients and update together."""
import sys

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


def workload(name, remote="cuda"):
    return synth.make_workload(name, device="cuda", feature_device="cuda", remote_device=remote)


@pytest.mark.parametrize("name,remote", [("small", "cuda"), ("small", "cpu"), ("mid_bf16", "cuda")])
def test_held_rows_come_through_the_gather_as_they_are(rg, name, remote):
    """Every batch's held rows are those of the batch's feature rows, to the bit, out of the store, the cache and pinned host memory."""
    W = workload(name, remote)
    if remote == "cpu" and not W.remote_rows.is_pinned():
        W.remote_rows = W.remote_rows.pin_memory()
    held = train.held_tables(rg, W)
    assert held[0].is_cuda and held[1].is_cuda == (remote == "cuda")
    plain, mine = train.Batches(rg, W), train.Batches(rg, W, held=held)
    assert len(plain) == len(mine) > 0
    for b in range(len(plain)):
        rows = plain.rows(b)
        assert torch.equal(mine.gathered(b), rg.rg_quantize_rows(rows))
        assert torch.equal(mine.rows(b), rg.rg_dequantize_rows(rg.rg_quantize_rows(rows), W.cfg.feat_dim, dtype=rows.dtype))


@pytest.mark.parametrize("name", ["small", "mid_bf16"])
def test_gradients_of_a_layer(rg, name):
    """Of a batch's rows through norm and product, against the formulas in 64 bits on what the held rows stand for.  A sum's terms are off by 2^-16 of themselves (16-bit types' parts) and
    2^-20 for up to 4,096 terms added in 32 bits; a result by half a unit in its last place, 2^-8 of itself at most."""
    W = workload(name)
    batches = train.Batches(rg, W, held=train.held_tables(rg, W))
    rows = batches.rows(0)
    x = rows.clone().requires_grad_()
    model = train.Sage(W.cfg.feat_dim, 64, 8, 1, rows.dtype)
    w = (model.weights[0][:, : W.cfg.feat_dim]).detach().clone().requires_grad_()
    y = train.linear8(rg)(x, w)
    dy = torch.randn(y.shape, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").to(y.dtype)
    y.backward(dy)
    vx, vw = (rg.rg_dequantize_rows(rg.rg_quantize_rows(t.detach()), t.shape[1]).double() for t in (x, w))
    g = dy.double()
    ulp = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[rows.dtype]
    for got, ref, size in ((y.detach(), vx @ vw.t(), vx.abs() @ vw.abs().t()), (x.grad, g @ vw, g.abs() @ vw.abs()), (w.grad, g.t() @ vx, g.abs().t() @ vx.abs())):
        assert bool(((got.double() - ref).abs() <= ulp * ref.abs() + 2.0 ** -15 * size).all())


@pytest.mark.parametrize("name", ["small", "mid_bf16"])
def test_an_epoch_runs(rg, name):
    """Every parameter gets a gradient that is a number, and is changed."""
    W = workload(name)
    model = train.Sage(W.cfg.feat_dim, 64, 8, len(W.cfg.fanout), W.local_rows.dtype)
    before = [t.detach().clone() for t in model.weights + model.scales + model.shifts]
    batches = train.Batches(rg, W, held=train.held_tables(rg, W))
    losses = train.train_epoch(rg, batches, model, train.Muon(rg, model), train.labels_of(W, 8), train.layer_norm(rg), train.linear8(rg))
    assert losses.shape == (len(batches),) and bool(losses.isfinite().all())
    for a, b in zip(before, model.weights + model.scales + model.shifts):
        assert bool(b.isfinite().all()) and not torch.equal(a, b)


def test_the_command_runs(rg, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["train", "--workload", "tiny", "--epochs", "1", "--hidden", "32", "--classes", "4", "--rows8"])
    train.main()
    assert "epoch 0: loss" in capsys.readouterr().out
