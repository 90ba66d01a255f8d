"""Which device the operators of the training step run on: that of their operands, whatever the current one is.  The library and the tensors are stood in for,
so that two devices need none."""
import contextlib

import pytest
import torch

from paper_2509_05207_amd import binding as rg

THERE, HERE = torch.device("cuda", 1), torch.device("cuda", 0)


class Tensor:
    """What the marshalling asks of a tensor."""

    def __init__(self, shape, device=THERE, dtype=torch.float32):
        self.shape, self.device, self.dtype, self.is_cuda = torch.Size(shape), device, dtype, True

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def element_size(self):
        return self.dtype.itemsize

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return True

    def __getitem__(self, k):
        return Tensor(self.shape[1:], self.device, self.dtype)


@pytest.fixture
def ran_on(monkeypatch):
    """The device that is current in each of the library's calls."""
    current, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], d.index
        yield
        current[0] = before

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                seen.append(current[0])
                return rg.RG_OK
            return entry
    monkeypatch.setattr(rg, "lib", Library)
    monkeypatch.setattr(rg, "_stream_and_use", lambda device, stream, *made: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch, "empty", lambda size, dtype, device: Tensor(size if isinstance(size, tuple) else (size,), device, dtype))
    monkeypatch.setattr(torch.autograd.graph, "increment_version", lambda t: None)
    return seen


def test_calls_go_to_the_operands_device(ran_on):
    x, v, s = Tensor((4, 8)), Tensor((8,)), Tensor((4,))
    rg.rg_layer_norm(x, v, v, out=x)
    rg.rg_layer_norm_backward(x, x, v, s, s, out=x)
    rg.rg_update_workspace([x])
    rg.rg_orthogonalize([x], out=[x])
    rg.rg_muon_step([x], [x], [x], lr=0.1)
    assert len(ran_on) >= 7 and set(ran_on) == {1}
    del ran_on[:]
    here = Tensor((4, 8), HERE)
    rg.rg_layer_norm(here, out=here)
    rg.rg_orthogonalize([here], out=[here])
    assert set(ran_on) == {0}


def test_operands_of_two_devices_are_refused(ran_on):
    x, v, s = Tensor((4, 8)), Tensor((8,)), Tensor((4,))
    y, w, t = Tensor((4, 8), HERE), Tensor((8,), HERE), Tensor((4,), HERE)
    for call in (lambda: rg.rg_layer_norm(x, out=y), lambda: rg.rg_layer_norm(x, w, out=x), lambda: rg.rg_layer_norm(x, v, w, out=x), lambda: rg.rg_layer_norm_backward(y, x, v, s, s, out=x),
                 lambda: rg.rg_layer_norm_backward(x, x, w, s, s, out=x), lambda: rg.rg_layer_norm_backward(x, x, v, t, s, out=x), lambda: rg.rg_layer_norm_backward(x, x, v, s, t, out=x),
                 lambda: rg.rg_layer_norm_backward(x, x, v, s, s, out=y), lambda: rg.rg_layer_norm_backward(x, x, v, s, s, out=x, workspace=w),
                 lambda: rg.rg_orthogonalize([x, y], out=[x, y]), lambda: rg.rg_orthogonalize([x], out=[y]), lambda: rg.rg_orthogonalize([x], out=[x], workspace=w),
                 lambda: rg.rg_muon_step([y], [x], [x], lr=0.1), lambda: rg.rg_muon_step([x], [x], [y], lr=0.1), lambda: rg.rg_muon_step([x], [x], [x], lr=0.1, out_weights=[y]),
                 lambda: rg.rg_muon_step([x], [x], [x], lr=0.1, out_momenta=[y]), lambda: rg.rg_update_workspace([x, y])):
        with pytest.raises(AssertionError):
            call()
    assert all(d == 1 for d in ran_on)
