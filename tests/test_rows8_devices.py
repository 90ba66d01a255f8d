"""Which device the calls on held rows run on: that of their operands, whatever the current one is.  The library and the tensors are stood in for, so that two devices
need none."""
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

    def is_pinned(self):
        return False

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


def held(rows, cols, device=THERE):
    return Tensor((rows, (cols + 19) // 16 * 16), device, torch.uint8)


def test_calls_go_to_the_operands_device(ran_on):
    x, at, bias = Tensor((4, 100)), Tensor((3,), dtype=torch.int64), Tensor((7,))
    assert rg.rg_quantize_rows(x).device == THERE
    assert rg.rg_quantize_rows(x, rows=at).shape == (3, 112)
    assert rg.rg_dequantize_rows(held(4, 100), 100, rows=at).shape == (3, 100)
    assert rg.rg_rows8_product(held(4, 100), held(7, 100), 100, bias=bias).device == THERE
    dx, dw, db = rg.rg_rows8_product_backward(Tensor((4, 7)), held(4, 100), held(7, 100), 100)
    assert (dx.shape, dw.shape, db.shape) == ((4, 100), (7, 100), (7,)) and dx.device == dw.device == db.device == THERE
    assert len(ran_on) >= 5 and set(ran_on) == {1}
    del ran_on[:]
    rg.rg_quantize_rows(Tensor((4, 100), HERE))
    assert set(ran_on) == {0}


def test_operands_of_two_devices_are_refused(ran_on):
    x, at, dy = Tensor((4, 100)), Tensor((3,), HERE, torch.int64), Tensor((4, 7))
    for call in (lambda: rg.rg_quantize_rows(x, rows=at), lambda: rg.rg_quantize_rows(x, out=held(4, 100, HERE)), lambda: rg.rg_dequantize_rows(held(4, 100), 100, rows=at),
                 lambda: rg.rg_dequantize_rows(held(4, 100), 100, out=Tensor((4, 100), HERE)), lambda: rg.rg_rows8_product(held(4, 100), held(7, 100, HERE), 100),
                 lambda: rg.rg_rows8_product(held(4, 100), held(7, 100), 100, bias=Tensor((7,), HERE)), lambda: rg.rg_rows8_product(held(4, 100), held(7, 100), 100, out=Tensor((4, 7), HERE)),
                 lambda: rg.rg_rows8_product(held(4, 100), held(7, 100), 100, workspace=Tensor((7,), HERE)), lambda: rg.rg_rows8_product_backward(Tensor((4, 7), HERE), held(4, 100), held(7, 100), 100),
                 lambda: rg.rg_rows8_product_backward(dy, held(4, 100), held(7, 100, HERE), 100), lambda: rg.rg_rows8_product_backward(dy, held(4, 100), held(7, 100), 100, out=Tensor((4, 100), HERE)),
                 lambda: rg.rg_rows8_product_backward(dy, held(4, 100), held(7, 100), 100, workspace=Tensor((9,), HERE))):
        with pytest.raises(AssertionError):
            call()
    assert all(d == 1 for d in ran_on)
