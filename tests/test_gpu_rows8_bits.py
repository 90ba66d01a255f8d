"""How many bits of dy the gradients on held rows have, whatever its type.

With one element of a row of dy (of a column, for dweight) that is not zero, a gradient is that element times its scale, which is rounded to 24 bits (2^-24 of it), times a code.  Of the parts that the
product goes in as, which hold all 24 bits, each gives an exact term, and two of three additions may round, in whatever direction: 2^-23 of the sum of parts, which the first two exceed by 2^-7 at
most.  Sums with zeros are exact.  So a result before it is rounded to its type is off by no more than 2^-24 + 2 2^-23 (1 + 2^-7) < 3 2^-23 of itself, and rounding does not change an order: it lies
between what both ends of that range are rounded to."""
import pytest
import torch

from test_gpu_rows8 import made, packed, random_held

pytestmark = pytest.mark.gpu
OFF = 3 * 2.0 ** -23


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def between(what, got, ref):
    lo, hi = (ref - OFF * ref.abs()).to(got.dtype), (ref + OFF * ref.abs()).to(got.dtype)
    bad = ~((lo <= got) & (got <= hi))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()}, first at {bad.nonzero()[0].tolist()}: {float(got[bad][0])!r} for {float(ref[bad][0])!r}"


@pytest.mark.parametrize("n,m,d", [(4, 64, 256), (65, 33, 130), (300, 270, 602), (5000, 257, 130), (20_000, 64, 128), (70_001, 256, 96)])
@pytest.mark.parametrize("dtype,weight", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32)], ids=str)
def test_single_terms(rg, n, m, d, dtype, weight):
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    values = made(n, m, dtype, 7)
    at = torch.randint(m, (n,), generator=torch.Generator().manual_seed(3)).cuda()
    dy = torch.zeros_like(values).scatter_(1, at[:, None], values.gather(1, at[:, None]))
    dx, _, _ = rg.rg_rows8_product_backward(dy, x, w, d)
    between("dx", dx, (values.gather(1, at[:, None]).double() * sw.double()[at][:, None]) * qw[at])
    at = torch.randint(n, (m,), generator=torch.Generator().manual_seed(4)).cuda()
    dy = torch.zeros_like(values).scatter_(0, at[None], values.gather(0, at[None]))
    _, dw, db = rg.rg_rows8_product_backward(dy, x, w, d, weight_dtype=weight)
    between("dweight", dw, (values.gather(0, at[None])[0].double() * sx.double()[at])[:, None] * qx[at])
    assert torch.equal(db, values.gather(0, at[None])[0].to(weight))


@pytest.mark.parametrize("n,m,d", [(16_384, 4096, 4096), (70_001, 256, 130), (30_011, 5, 40), (8192, 300, 64)])
@pytest.mark.parametrize("want_dweight", [True, False])
def test_long_sums_of_columns(rg, n, m, d, want_dweight):
    """dbias is off by (64 + rows / 256) 2^-24 sum |dy| at most: no sum of it is longer than that.  The same number in all rows, whose last bits every addition beyond 512 of them loses, if they are added up one by one."""
    value = 1 + 2.0 ** -15 - 2.0 ** -23
    dy = torch.full((n, m), value, device="cuda")
    x = torch.zeros((n, (d + 19) // 16 * 16), dtype=torch.uint8, device="cuda") if want_dweight else None
    _, _, db = rg.rg_rows8_product_backward(dy, x, None, d, want_dx=False, want_dweight=want_dweight)
    assert bool(((db.double() - n * value).abs() <= (64 + n / 256) * 2.0 ** -24 * n * value).all()), float((db.double() / (n * value) - 1).abs().max() * 2 ** 24)


@pytest.mark.parametrize("n,m,d", [(70, 40, 100), (300, 270, 602), (20_000, 64, 128), (5000, 257, 130), (4096, 2060, 600)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("sign", [1, -1])
def test_products_beyond_the_range(rg, n, m, d, dtype, sign):
    """dy and a scale that are numbers, whose product is none in 32 bits: an infinity with a code other than zero, nothing with a code of zero, and all else as it was."""
    _, qx, sx = random_held(n, d, 1)
    _, qw, sw = random_held(m, d, 2)
    i, j = n // 2, m // 3
    sx[i], sw[j] = 100.0, 100.0
    qx[i], qw[j] = torch.arange(d, device="cuda") % 5 - 2, torch.arange(d, device="cuda") % 3 - 1
    x, w = packed(qx, sx), packed(qw, sw)
    dy = made(n, m, dtype, 7)
    dy[i, j] = 0
    clean = rg.rg_rows8_product_backward(dy, x, w, d)
    dy[i, j] = sign * 2.0 ** 127
    got = rg.rg_rows8_product_backward(dy, x, w, d)
    for a, b, row, codes in ((got[0], clean[0], i, qw[j]), (got[1], clean[1], j, qx[i])):
        keep = torch.arange(a.shape[0], device="cuda") != row
        assert torch.equal(a[keep], b[keep])
        none = codes == 0
        assert torch.equal(a[row][none], b[row][none]) and bool((a[row][~none] == sign * torch.sign(codes[~none]) * float("inf")).all())
    assert float(got[2][j]) == sign * 2.0 ** 127
