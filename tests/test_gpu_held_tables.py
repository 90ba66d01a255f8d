"""A feature table in pinned host memory is held in 8 bits by parts, so that it need not fit on the device."""
from types import SimpleNamespace

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


def workload(rows, cols, pad):
    g = torch.Generator(device="cuda").manual_seed(rows)
    local = torch.randn((100, cols + pad), generator=g, device="cuda").bfloat16()
    remote = synth.pinned_empty((rows, cols + pad), torch.bfloat16)
    for first in range(0, rows, 50_000):
        remote[first: first + 50_000].copy_(torch.randn((min(50_000, rows - first), cols + pad), generator=g, device="cuda").bfloat16())
    return SimpleNamespace(cfg=SimpleNamespace(feat_dim=cols), local_rows=local, remote_rows=remote)


@pytest.mark.parametrize("rows,cols,pad", [(400_001, 512, 0), (3, 100, 4), (1, 7, 1), (0, 16, 0)])
def test_parts(rg, rows, cols, pad):
    W = workload(rows, cols, pad)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    local, remote = train.held_tables(rg, W)
    assert torch.cuda.max_memory_allocated() - before <= 80 << 20                       # of 211 MB of the largest
    assert remote.shape == (rows, rg.rg_rows8_bytes(cols)) and not remote.is_cuda and (rows == 0 or remote.is_pinned()) and local.is_cuda
    assert torch.equal(local, rg.rg_quantize_rows(W.local_rows[:, :cols]))
    for first in range(0, rows, 50_000):
        assert torch.equal(remote[first: first + 50_000].cuda(), rg.rg_quantize_rows(W.remote_rows[first: first + 50_000].cuda()[:, :cols]))


def test_smaller_parts_make_the_same(rg):
    W = workload(1000, 33, 2)
    whole = train.held_tables(rg, W)[1]
    for at_once in (1, 48, 500, 47_999):
        assert torch.equal(train.held_tables(rg, W, at_once)[1], whole)
