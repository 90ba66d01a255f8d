"""Every way that products of held rows and their gradients take, on padded rows with odd sides, against 64 bits.

Bounds element by element, and half a unit of the result's type on top:
  product     that of test_gpu_rows8: of 16 bits, 2^-24 of the product twice and of the result once; of 32, 2^-44 of both (test_gpu_rows8_rounding)
  dx, dweight of T, the sum of the terms' sizes: dy * scale is rounded to 24 bits (2^-24), which go in as three bf16 numbers.  A matrix operation adds 32 terms, at most eight at a time in
              whatever order and with whatever direction of rounding: 2^-23 T for every eight terms of every part, and for up to 80 sums of splits in a row
  dbias       (64 + rows / 256) 2^-24 sum |dy|"""
import pytest
import torch

from rows8_ways import GRADIENTS, PRODUCTS
from test_gpu_rows8 import TYPES, U, check, held_bytes, made, random_held, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def padded(held, pad, fill):
    """The same rows in a buffer of rows of `pad` more bytes."""
    buf = torch.full((held.shape[0], held.shape[1] + pad), fill, dtype=torch.uint8, device="cuda")
    buf[:, pad // 2: pad // 2 + held.shape[1]] = held
    return buf[:, pad // 2: pad // 2 + held.shape[1]]


@pytest.mark.parametrize("n,m,d", PRODUCTS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("bias", [None, "float32", "same"])
def test_products(rg, n, m, d, dtype, bias):
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    b = None if bias is None else (50 * torch.randn(m, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda")).to(torch.float32 if bias == "float32" else dtype)
    buf, out = strided(n, m, dtype, 3, 1)
    assert held_bytes(d) == x.shape[1]
    rg.rg_rows8_product(padded(x, 32, 255), padded(w, 64, 254), d, bias=b, out=out)
    product = (qx @ qw.t().contiguous()) * sx.double()[:, None] * sw.double()
    ref = product if b is None else product + b.double()
    check("y", out, ref, U * (ref.abs() + 2.001 * product.abs()) if dtype != torch.float32 else 2.0 ** -44 * ((ref - product).abs() + product.abs()))
    out.fill_(3.0)
    assert bool((buf == 3).all())


@pytest.mark.parametrize("n,m,d", GRADIENTS)
@pytest.mark.parametrize("dtype,weight", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float32)], ids=str)
def test_gradients(rg, n, m, d, dtype, weight):
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    dy = made(n, m, dtype, 7, pad=5, lead=1)
    buf, out = strided(n, d, dtype, 5, 1)
    _, dw, db = rg.rg_rows8_product_backward(dy, padded(x, 32, 255), padded(w, 64, 254), d, weight_dtype=weight, out=out)
    g = dy.double()

    def bound(k):
        return U + 2.0 ** -40 + 2.0 ** -23 * (3 * (k / 8 + 8) + 80)
    check("dx", out, (g * sw.double()) @ qw, bound(m) * ((g.abs() * sw.double()) @ qw.abs()))
    check("dweight", dw, (g * sx.double()[:, None]).t().contiguous() @ qx, bound(n) * ((g.abs() * sx.double()[:, None]).t().contiguous() @ qx.abs()))
    check("dbias", db, g.sum(0), (64 + n / 256) * U * g.abs().sum(0))
    out.fill_(3.0)
    assert bool((buf == 3).all())


def test_a_thousand_million_outputs(rg):
    """As many as there may be, in tiles of which a launch holds as many; small whole numbers, of which nothing is rounded."""
    m = 2**30
    held = torch.zeros((3, 16), dtype=torch.uint8, device="cuda")
    held[:, 0] = torch.tensor([1, 2, 255], dtype=torch.uint8)
    held.view(torch.float32)[:, -1] = 1.0
    dy = torch.empty((3, m), dtype=torch.bfloat16, device="cuda")
    for n in range(3):
        for first in range(0, m, 2**28):
            dy[n, first: first + 2**28] = (torch.arange(first, first + 2**28, device="cuda") * 7 + n) % (5 + n)
    _, dw, db = rg.rg_rows8_product_backward(dy, held, None, 1, want_dx=False)
    for first in range(0, m, 2**28):
        a, b, c = dy[:, first: first + 2**28]
        assert torch.equal(dw[first: first + 2**28, 0], a + 2 * b - c) and torch.equal(db[first: first + 2**28], a + b + c)
