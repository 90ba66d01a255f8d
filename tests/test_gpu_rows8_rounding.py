"""The last bits of the product of held rows: where the bias takes the product away, beside rows of zeros, and with scales and biases of every size.

A result of 32 bits is off by half a step, by 2^-44 of what the product and the bias are by themselves, and by 2^-149.  (u = 2^-24: the sum of codes and the scales' product are numbers of 24 bits and what these
leave over, u of them at most; the rounding of their product t leaves u |t|.  Added up in two roundings of numbers of 2 u |t| and 3 u |t|, with the product of both remainders, u^2 |t|, left out, and then with what the
addition of the bias leaves, u |t + bias| at most, in another rounding: (2 + 3 + 1 + 3) u^2 |t| + u^2 |t + bias| < 2^-44 (|t| + |bias|).  Below 2^-126 a step is 2^-149 whatever the size, and product and rest are rounded to it each by
themselves.)"""
import pytest
import torch

from test_gpu_rows8 import HALF_ULP, TYPES, held_bytes, packed, product_sum, random_held

pytestmark = pytest.mark.gpu

# few rows; few rows of many codes; tiles of 64, 128, 128 with four stages, 256; split codes; thin ones by their registers, and with their outputs shared out
SHAPES = [(40, 30, 50), (1000, 40, 2600), (1000, 300, 500), (5000, 1030, 200), (1000, 2050, 50), (20_011, 517, 1300), (300, 1000, 8192), (20_011, 40, 50), (20_011, 130, 500), (20_011, 130, 700), (40_001, 1030, 200)]


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def within(y, product, bias):
    ref = product + bias
    off, tol = (y.double() - ref).abs(), 2.0 ** -24 * ref.abs() + 2.0 ** -44 * (product.abs() + bias.abs()) + 2.0 ** -149
    beyond = torch.isinf(y) & (ref * torch.sign(y.double()) >= float.fromhex("0x1.ffffffp+127") - tol)      # half a step behind the largest
    bad = ~((off <= tol) | beyond)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()}, worst {float((off / tol)[bad].max()):.3g} times the bound, first at {bad.nonzero()[0].tolist()}: {float(y[bad][0])!r} for {float(ref[bad][0])!r}"


def taken_away(product):
    """A bias that is one of an output's products, rounded, with the other sign: another row's for every output."""
    n, m = product.shape
    return -product[(torch.arange(m, device="cuda") * 7) % n, torch.arange(m, device="cuda")].float()


@pytest.mark.parametrize("n,m,d", SHAPES)
@pytest.mark.parametrize("zeros", ["none", "x", "w", "both", "every"])
def test_a_bias_that_takes_the_product_away(rg, n, m, d, zeros):
    """Beside rows of zeros too.  What is made of those is the bias."""
    _, qx, sx = random_held(n, d, 1)
    _, qw, sw = random_held(m, d, 2)
    b = taken_away(product_sum(qx, qw) * sx.double()[:, None] * sw.double())
    if zeros in ("x", "both", "every"):
        rows = torch.arange(n, device="cuda") % (7 if zeros == "every" else n) == (3 if zeros == "every" else n // 3)
        qx[rows], sx[rows] = 0, 2.0 ** -126
    if zeros in ("w", "both"):
        qw[m // 2], sw[m // 2] = 0, 2.0 ** -126
    y = rg.rg_rows8_product(packed(qx, sx), packed(qw, sw), d, bias=b)
    within(y, product_sum(qx, qw) * (sx.double()[:, None] * sw.double()), b.double())
    if zeros in ("x", "both", "every"):
        assert torch.equal(y[rows], b.expand(n, m)[rows])
    if zeros in ("w", "both"):
        assert bool((y[:, m // 2] == b[m // 2]).all())


@pytest.mark.parametrize("n,m,d", SHAPES)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_result_does_not_depend_on_what_lies_beside_it(rg, n, m, d, dtype):
    """Rows of zeros, of other sizes and of NaN, and biases of other sizes, leave the bits of the rest as they were."""
    _, qx, sx = random_held(n, d, 1)
    _, qw, sw = random_held(m, d, 2)
    b = taken_away(product_sum(qx, qw) * sx.double()[:, None] * sw.double())
    for dt in {torch.float32, dtype}:
        bias = b.to(dt)
        want = rg.rg_rows8_product(packed(qx, sx), packed(qw, sw), d, bias=bias, dtype=dtype)
        for scale in (2.0 ** -126, 2.0 ** -60, 2.0 ** 100, float("nan")):
            x2, s2, v2, c2 = qx.clone(), sx.clone(), sw.clone(), bias.clone()
            x2[n // 3], s2[n // 3], s2[n - 1], v2[m // 2], c2[0] = 0, 2.0 ** -126, scale, scale, 60000.0 if dt == torch.float16 else 2.0 ** 125
            got = rg.rg_rows8_product(packed(x2, s2), packed(qw, v2), d, bias=c2, dtype=dtype)
            rows, outs = torch.ones(n, dtype=torch.bool, device="cuda"), torch.ones(m, dtype=torch.bool, device="cuda")
            rows[n // 3] = rows[n - 1] = outs[m // 2] = outs[0] = False
            assert torch.equal(got[rows][:, outs], want[rows][:, outs])


@pytest.mark.parametrize("n,m,d", [(40, 30, 50), (300, 270, 602), (1000, 300, 500), (20_011, 130, 300)])
def test_scales_and_biases_of_every_size(rg, n, m, d):
    """Scales from 2^-126 to 2^121 on either side, in one block; biases from nothing to the largest number, and some that take the product away."""
    _, qx, _ = random_held(n, d, 1)
    _, qw, _ = random_held(m, d, 2)
    g = torch.Generator().manual_seed(5)
    sx, sw = ((2.0 ** (torch.rand(k, generator=g, dtype=torch.float64) * 247 - 126)).float().cuda() for k in (n, m))
    product = product_sum(qx, qw) * (sx.double()[:, None] * sw.double())
    some = torch.arange(m, device="cuda")
    sizes = (2.0 ** (torch.rand(m, generator=g, dtype=torch.float64) * 276 - 149)).float().cuda()
    away = taken_away(product.clamp(-3.4e38, 3.4e38))
    for b in (torch.zeros(m, device="cuda"), torch.where(some % 2 == 0, sizes, -sizes), away):
        y = rg.rg_rows8_product(packed(qx, sx), packed(qw, sw), d, bias=b)
        assert not bool(torch.isnan(y).any())
        within(y, product, b.double())
    b = torch.zeros(m, device="cuda")
    b[0], b[1], b[2] = float("inf"), float("-inf"), float("nan")
    y = rg.rg_rows8_product(packed(qx, sx), packed(qw, sw), d, bias=b)
    sane = product.abs() < 3e38
    assert bool((y[:, 0][sane[:, 0]] == float("inf")).all()) and bool((y[:, 1][sane[:, 1]] == float("-inf")).all()) and bool(torch.isnan(y[:, 2]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_scales_of_every_size_in_16_bits(rg, dtype):
    """A sum of codes, the scales' product and their product with the bias rounded to 32 bits, and that to 16."""
    n, m, d = 300, 270, 602
    _, qx, _ = random_held(n, d, 1)
    _, qw, _ = random_held(m, d, 2)
    g = torch.Generator().manual_seed(5)
    sx = (2.0 ** (torch.rand(n, generator=g, dtype=torch.float64) * 247 - 126)).float().cuda()
    sw = (2.0 ** (torch.rand(m, generator=g, dtype=torch.float64) * 40 - 20)).float().cuda() / sx[torch.arange(m, device="cuda")].clamp(min=2.0 ** -100)
    product, b = product_sum(qx, qw) * (sx.double()[:, None] * sw.double()), torch.randn(m, device="cuda")
    y = rg.rg_rows8_product(packed(qx, sx), packed(qw, sw), d, bias=b, dtype=dtype)
    ref, (rel, least) = product + b.double(), HALF_ULP[dtype]
    tol = 2.0 ** -24 * (ref.abs() + 2.001 * product.abs()) + 2.0 ** -149
    tol = tol + (ref.abs() + tol) * rel + least
    big = torch.finfo(dtype).max * (1 + rel)
    bad = ~(((y.double() - ref).abs() <= tol) | (torch.isinf(y) & (ref * torch.sign(y.double()) >= big - tol)))
    assert not bool(bad.any())


@pytest.mark.parametrize("d", [50, 300])
def test_rows_at_no_position(rg, d):
    """Rows of zeros as the gather and the calls on held rows leave them: by a position of -1, and out of zeros."""
    x = torch.randn(20_011, d, device="cuda")
    rows = torch.arange(20_011, device="cuda")
    rows[5::9] = -1
    x[100:140] = 0
    held = rg.rg_quantize_rows(x, rows=rows)
    w, _, _ = random_held(60, d, 2)
    b = torch.randn(60, device="cuda")
    y = rg.rg_rows8_product(held, w, d, bias=b)
    none = (rows < 0) | ((rows >= 100) & (rows < 140))
    assert held.shape[1] == held_bytes(d) and bool((y[none] == b).all()) and bool((y[~none] != b).any(1).all())


@pytest.mark.parametrize("n,m,d", SHAPES + [(20_011, 40, 64), (20_011, 40, 61), (1000, 300, 129)])
def test_rows_of_the_least_scale_that_are_not_zero(rg, n, m, d):
    """One code in the first or the last place, in rows or in outputs that have the scale of rows of zeros; results below the smallest normal numbers among them."""
    _, qx, sx = random_held(n, d, 1)
    _, qw, sw = random_held(m, d, 2)
    none = torch.zeros(m, device="cuda")
    for place in (0, d - 1):
        for code in (1, -127):
            for rows, sizes in ((True, sw * 2.0 ** 20), (True, sw / 2.0 ** 20), (False, sx * 2.0 ** 20)):
                a, s, b, t = qx.clone(), sx.clone(), qw.clone(), sw.clone()
                q, least, other = (a, s, t) if rows else (b, t, s)
                other.copy_(sizes)
                at = torch.tensor([0, len(least) // 2, len(least) - 1], device="cuda")
                q[at], least[at] = 0, 2.0 ** -126
                q[at[1:], place] = code
                y = rg.rg_rows8_product(packed(a, s), packed(b, t), d, bias=none)
                product = product_sum(a, b) * (s.double()[:, None] * t.double())
                within(y, product, none.double())
                assert bool(((y if rows else y.t())[at[1:]] != 0).any()) == bool((product.abs() if rows else product.t().abs())[at[1:]].max() > 2.0 ** -149)


@pytest.mark.parametrize("n,m,d", [(40, 30, 50), (300, 270, 602), (20_011, 130, 300), (20_011, 517, 1300)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_an_infinity_of_the_bias_stands_against_numbers_of_any_size(rg, n, m, d, dtype):
    """Products of scales and codes that pass 32 bits are numbers still; a scale that is none makes a NaN."""
    _, qx, sx = random_held(n, d, 1)
    _, qw, sw = random_held(m, d, 2)
    sx[:], sw[:] = 2.0 ** 120, 2.0 ** 121
    b = torch.zeros(m, device="cuda")
    b[0::3], b[1::3] = float("inf"), float("-inf")
    for scale in (2.0 ** 120, 2.0 ** 90, float("nan")):
        sx[n // 2] = scale
        y = rg.rg_rows8_product(packed(qx, sx), packed(qw, sw), d, bias=b, dtype=dtype)
        rows = torch.arange(n, device="cuda") != n // 2 if scale != scale else torch.ones(n, dtype=torch.bool, device="cuda")
        assert bool(torch.isnan(y[~rows]).all())
        assert bool((y[rows][:, 0::3] == float("inf")).all()) and bool((y[rows][:, 1::3] == float("-inf")).all())
        assert bool((y[rows][:, 2::3] == (torch.sign(product_sum(qx, qw)) * float("inf")).nan_to_num(nan=0.0, posinf=float("inf"), neginf=float("-inf"))[rows][:, 2::3]).all())
