"""Rows held in 8 bits and the products on them through the C ABI, against their definitions in 64 bits.

Codes and scales have to be equal to the bit.  What is read back is code * scale in 32 bits, rounded to its type: equal to the bit as well.
Elsewhere a result may be off by half a unit in the last place of its type (its smallest normal number's at least), and by what stands here, element by element.
  product     of 32 bits: 2^-23 of its rounding.  Of 16: the sum of codes, the scales' product and their product with the bias are rounded to 32 bits before the
              result is to 16, so that it is off by 2^-24 of the product twice, of the result once, and the product of these errors
  dx, dweight terms t = dy * scale * code of T = sum |t|: dy * scale is rounded (2^-24) and goes in as two bf16 numbers, the first cut off, which leaves less than
              2^-7, the second rounded: 2^-7 2^-9; of fp32 as three, which hold all 24 bits.  A matrix operation adds 32 terms, at most eight
              at a time in whatever order and with whatever direction of rounding: 2^-23 T for every eight terms of every part, and for each of up to 512 splits.
  dbias       (64 + rows / 256) 2^-24 sum |dy|: a thread's sum of a part of the rows, and the parts'."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -133), torch.float16: (2.0 ** -11, 2.0 ** -24)}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def rand(g, *size):
    return torch.randn(size, generator=g, device="cuda", dtype=torch.float64)


def made(rows, cols, dtype, seed, pad=0, lead=0):
    """Rows as a view of rows of cols + pad elements that start `lead` elements into their buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows * (cols + pad) + lead + 8,), 7.0, dtype=dtype, device="cuda")
    v = buf[lead: lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_((rand(g, rows, cols) * torch.exp(rand(g, rows, 1))).to(dtype))
    return v


ONE_127TH = torch.tensor(float.fromhex("0x1.020408p-7"), dtype=torch.float32)


def definition(x):
    """(codes, scale) of rows in 64 bits."""
    x = x.detach().cpu()
    largest = x.float().abs().amax(1)
    scale = (largest * ONE_127TH).clamp(min=2.0 ** -126, max=float.fromhex("0x1.020406p+121"))
    q = x.double() / scale.double()[:, None]
    low = torch.floor(q)
    part = q - low
    codes = low + ((part > 0.5) | ((part == 0.5) & (torch.remainder(low, 2) == 1)))
    bad = ~torch.isfinite(x.double()).all(1)
    codes[bad] = 0
    scale[bad] = float("nan")
    return codes, scale


def held_bytes(cols):
    return (cols + 4 + 15) // 16 * 16


def packed(codes, scale, device="cuda"):
    held = torch.zeros((codes.shape[0], held_bytes(codes.shape[1])), dtype=torch.uint8)
    held[:, : codes.shape[1]] = codes.cpu().to(torch.int8).view(torch.uint8)
    held.view(torch.float32)[:, -1] = scale.float().cpu()
    return held.to(device)


def random_held(rows, cols, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(-127, 128, (rows, cols), generator=g)
    scale = torch.exp(spread * torch.randn(rows, generator=g, dtype=torch.float64)).float() / 64
    return packed(codes, scale), codes.double().cuda(), scale.cuda()


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8).cpu(), b.contiguous().view(torch.uint8).cpu())


def same_held(got, want, cols):
    """Equal to the bit, but that any NaN stands for a NaN."""
    a, b = got.cpu().view(torch.float32)[:, -1], want.cpu().view(torch.float32)[:, -1]
    assert torch.equal(got.cpu()[:, :-4], want.cpu()[:, :-4])
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)], b[~torch.isnan(b)])


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 11, 12, 13, 15, 16, 17, 28, 31, 60, 61, 100, 124, 125, 127, 128, 129, 252, 253, 255, 256, 500, 602, 1020, 1021, 1023, 2044, 2045, 4097, 8191, 16_380, 16_381, 32_764,
          32_765, 70_001, 131_072]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_held_rows_of_every_width(rg, cols, dtype):
    x = made(13, cols, dtype, cols)
    held = rg.rg_quantize_rows(x)
    codes, scale = definition(x)
    same_held(held, packed(codes, scale, "cpu"), cols)
    values = (codes.float() * scale[:, None])
    for to in TYPES:
        assert same_bits(rg.rg_dequantize_rows(held, cols, dtype=to), values.to(to)), to


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols,pad,lead", [(1, 64, 0, 0), (7, 602, 2, 0), (300, 33, 1, 1), (1, 1, 0, 1), (5000, 9, 3, 2), (70_000, 16, 0, 0), (64, 2049, 5, 3)])
def test_strides_and_places(rg, dtype, rows, cols, pad, lead):
    x = made(rows, cols, dtype, rows + cols, pad, lead)
    b = held_bytes(cols)
    buf = torch.full((rows, b + 32), 85, dtype=torch.uint8, device="cuda")
    rg.rg_quantize_rows(x, out=buf[:, 16: 16 + b])
    same_held(buf[:, 16: 16 + b], packed(*definition(x), "cpu"), cols)
    assert bool((buf[:, :16] == 85).all()) and bool((buf[:, 16 + b:] == 85).all())
    out = torch.full((rows, cols + 3), 5.0, dtype=dtype, device="cuda")
    rg.rg_dequantize_rows(buf[:, 16: 16 + b], cols, out=out[:, 1: 1 + cols])
    assert same_bits(out[:, 1: 1 + cols], rg.rg_dequantize_rows(buf[:, 16: 16 + b].contiguous(), cols, dtype=dtype))
    assert bool((out[:, 0] == 5).all()) and bool((out[:, 1 + cols:] == 5).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cols", [6, 130, 40_000])
def test_rows_of_special_values(rg, dtype, cols):
    f = torch.finfo(dtype)
    x = torch.zeros((14, cols), dtype=torch.float64)
    x[1, 0] = float("inf")
    x[2, cols - 1] = float("-inf")
    x[3, cols // 2] = float("nan")
    x[4, 0], x[4, 1] = float("nan"), float("inf")
    x[5, 0], x[5, 1] = f.max, f.min
    x[6, 0], x[6, 1] = f.tiny, -f.tiny
    x[7, 0] = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    x[8, :] = -3.0
    x[9, :5] = torch.tensor([127.0, 0.5, 1.5, -2.5, -63.5])              # ties to even, at a scale of one
    x[10, :4] = torch.tensor([254.0, 1.0, 3.0, -5.0])                    # the same at two
    x[11, 0], x[11, 1] = 2.0 ** -10, 2.0 ** -14
    x[12, cols - 1] = -1.0
    x[13, 0] = -0.0
    x = x.to(dtype).cuda()
    held = rg.rg_quantize_rows(x)
    codes, scale = definition(x)
    same_held(held, packed(codes, scale, "cpu"), cols)
    back = rg.rg_dequantize_rows(held, cols, dtype=torch.float32).cpu()
    assert bool(torch.isnan(back[1:5]).all()) and bool((back[[0, 13]] == 0).all()) and bool(torch.isfinite(back[5:]).all())


def test_quotients_next_to_a_border(rg):
    """Elements at and one unit beside (k + 1/2) s, of scales with all 24 bits."""
    g = torch.Generator().manual_seed(3)
    largest = (torch.rand(64, generator=g) * 4 + 0.1).float()
    scale = largest * ONE_127TH
    x = torch.zeros((64, 3 * 126 + 1), dtype=torch.float32)
    x[:, 0] = largest
    for k in range(126):
        at = ((k + 0.5) * scale.double()).float()
        x[:, 1 + 3 * k], x[:, 2 + 3 * k], x[:, 3 + 3 * k] = at, torch.nextafter(at, torch.tensor(0.0)), -torch.nextafter(at, torch.tensor(9e9))
    held = rg.rg_quantize_rows(x.cuda())
    same_held(held, packed(*definition(x), "cpu"), x.shape[1])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cols", [3, 128, 602, 20_000])
def test_positions(rg, dtype, cols):
    """The same row twice, none (-1), and positions that are no row's."""
    x = made(40, cols, dtype, 5, pad=3)
    rows = torch.tensor([39, 0, 0, -1, 7, 40, -2, 2**40, 7, 39, -2**63, 2**63 - 1, 12], device="cuda")
    inside = (rows >= 0) & (rows < 40)
    want = torch.zeros((13, cols), dtype=torch.float64)
    want[inside.cpu()] = x.cpu().double()[rows[inside].cpu()]
    want[(~inside & (rows != -1)).cpu()] = float("nan")
    held = rg.rg_quantize_rows(x, rows=rows)
    same_held(held, packed(*definition(want.to(dtype)), "cpu"), cols)
    whole = rg.rg_quantize_rows(x)
    for to in TYPES:
        a, b = rg.rg_dequantize_rows(whole, cols, dtype=to, rows=rows), rg.rg_dequantize_rows(held, cols, dtype=to)
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert rg.rg_quantize_rows(x, rows=none).shape == (0, held_bytes(cols)) and rg.rg_dequantize_rows(whole, cols, rows=none).shape == (0, cols)


def test_rows_in_pinned_host_memory(rg):
    x = torch.randn(500, 77).pin_memory()
    rows = torch.randint(500, (64,), device="cuda")
    held = rg.rg_quantize_rows(x, rows=rows)
    assert same_bits(held, rg.rg_quantize_rows(x.cuda()[rows]))
    there = held.cpu().pin_memory()
    assert same_bits(rg.rg_dequantize_rows(there, 77), rg.rg_dequantize_rows(held, 77))


def test_a_table_beyond_32_bits(rg):
    """Offsets past 4 GiB on either side of both calls."""
    n, d = 2_200_000, 2000
    held = torch.zeros((n, held_bytes(d)), dtype=torch.uint8, device="cuda")
    last = made(3, d, torch.float32, 9)
    rg.rg_quantize_rows(last, out=held[-3:])
    rows = torch.tensor([n - 1, 0, n - 3, n], device="cuda")
    got = rg.rg_dequantize_rows(held, d, rows=rows)
    codes, scale = definition(last)
    values = codes.float() * scale[:, None]
    assert same_bits(got[0], values[2]) and same_bits(got[2], values[0]) and bool((got[1] == 0).all()) and bool(torch.isnan(got[3]).all())
    del held
    x = torch.zeros((600_000, d), dtype=torch.float32, device="cuda")
    x[-1] = last[0]
    held = rg.rg_quantize_rows(x)
    same_held(held[-1:], packed(*definition(last[:1]), "cpu"), d)
    assert bool((held[:-1, :-4] == 0).all())


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 601), (torch.bfloat16, 1203), (torch.float16, 40_001)], ids=str)
def test_results_larger_than_the_caches(rg, dtype, cols):
    rows = 150_000_000 // (cols * dtype.itemsize)
    held, codes, scale = random_held(500, cols, 5)
    at = torch.randint(-1, 500, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    buf, out = strided(rows, cols, dtype, 1, 1)
    rg.rg_dequantize_rows(held, cols, rows=at, out=out)
    values = torch.cat([(codes.float() * scale[:, None]).to(dtype), torch.zeros((1, cols), dtype=dtype, device="cuda")])
    for first in range(0, rows, 10_000):
        assert torch.equal(out[first: first + 10_000], values[at[first: first + 10_000]])
    out.fill_(3.0)
    assert bool((buf == 3).all())


def rounding(ref, dtype):
    rel, least = HALF_ULP[dtype]
    return ref.abs() * rel + least


def check(what, got, ref, tol):
    """What lies half a unit beyond the largest number of a type, or further, rounds to infinity."""
    f = torch.finfo(got.dtype)
    border = f.max + 2.0 ** math.floor(math.log2(f.max)) * f.eps / 2
    beyond = torch.isinf(got) & (ref * torch.sign(got.double()) >= border - tol)
    tol = tol + rounding(ref.abs() + tol, got.dtype)
    off = torch.where(beyond, 0.0, (got.double() - ref).abs())
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((off / tol).max()):.3g} times it, first at {bad.nonzero()[0].tolist()}: {float(got[bad][0])} for {float(ref[bad][0])}"


def product_sum(x, w):
    """codes_x codes_w^T, exactly: whole numbers below 2^53."""
    return x @ w.t().contiguous()


PRODUCTS = [(1, 1, 1), (1, 4096, 4096), (3, 5, 13), (16, 16, 64), (17, 33, 12), (2, 1000, 8191), (64, 64, 128), (65, 63, 129), (130, 257, 1001), (128, 256, 16), (1, 1, 131_072), (200, 3, 20_011), (33, 700, 28),
            (1000, 41, 602), (511, 513, 256), (48, 2048, 512), (300, 300, 140), (1025, 129, 384), (2048, 1024, 272), (5000, 17, 60), (4099, 515, 1300), (300, 1000, 8192), (130, 127, 20_011), (257, 65, 6001), (700, 515, 4100), (30_011, 70, 300),
            (20_000, 333, 700)]


@pytest.mark.parametrize("n,m,d", PRODUCTS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("bias", [None, "float32", "same"])
def test_product(rg, n, m, d, dtype, bias):
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    b = None if bias is None else (50 * rand(torch.Generator(device="cuda").manual_seed(m), m)).to(torch.float32 if bias == "float32" else dtype)
    y = rg.rg_rows8_product(x, w, d, bias=b, dtype=dtype)
    ref = product_sum(qx, qw) * sx.double()[:, None] * sw.double()
    if b is not None:
        ref = ref + b.double()
    product = product_sum(qx, qw).abs() * sx.double()[:, None] * sw.double()
    check("y", y, ref, U * (ref.abs() + 2.001 * product) if dtype != torch.float32 else 2.0 ** -46 * (ref.abs() + product))


@pytest.mark.parametrize("d", [13, 16, 17, 28, 29, 100, 602, 1001, 4096, 131_072])
def test_largest_sums(rg, d):
    """All codes 127 and -127: the largest sums there are, and codes of one sign in the last places."""
    codes = torch.full((20, d), 127)
    codes[1::2] = -127
    x = packed(codes, torch.full((20,), 1.9999999))
    w = packed(codes, torch.full((20,), -float(2**-20) * 1.7))
    y = rg.rg_rows8_product(x, w, d)
    q = codes.double().cuda()
    ref = product_sum(q, q) * x.view(torch.float32)[:, -1:].double() * w.view(torch.float32)[:, -1].double()
    check("y", y, ref, 2.0 ** -46 * ref.abs())


@pytest.mark.parametrize("n,m,d", [(5, 7, 100), (300, 270, 602), (1, 500, 4096)])
def test_scales_of_every_size(rg, n, m, d):
    """Scales whose product leaves fp32's range, where the result does not; rows that are NaN; rows of zeros."""
    x, qx, sx = random_held(n, d, 3)
    w, qw, sw = random_held(m, d, 4)
    sx[:], sw[:] = 2.0 ** -126, 2.0 ** 120
    sw[0], sw[m - 1] = float("nan"), 2.0 ** -100
    sw[1] = 0.0
    x, w = packed(qx, sx), packed(qw, sw)
    y = rg.rg_rows8_product(x, w, d)
    ref = product_sum(qx, qw) * (sx.double()[:, None] * sw.double())
    assert bool(torch.isnan(y[:, 0]).all()) and bool(torch.isfinite(y[:, 1:]).all()) and bool((y[:, 1] == 0).all())
    check("y", y[:, 1:], ref[:, 1:], 2.0 ** -46 * ref[:, 1:].abs())
    sx[n - 1] = float("nan")
    y2 = rg.rg_rows8_product(packed(qx, sx), w, d)
    assert bool(torch.isnan(y2[n - 1]).all()) and torch.equal(y2[: n - 1, 1:], y[: n - 1, 1:])


def strided(rows, cols, dtype, pad, lead, fill=3.0):
    buf = torch.full((rows * (cols + pad) + lead + 8,), fill, dtype=dtype, device="cuda")
    return buf, buf[lead: lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,m,d", [(3, 5, 13), (300, 270, 602), (65, 1000, 129), (2048, 515, 256)])
def test_strides_of_the_product(rg, dtype, n, m, d):
    x, w = random_held(n, d, 1)[0], random_held(m, d, 2)[0]
    want = rg.rg_rows8_product(x, w, d, dtype=dtype)
    b = held_bytes(d)
    wide_x = torch.full((n, b + 48), 255, dtype=torch.uint8, device="cuda")
    wide_w = torch.full((m, b + 16), 254, dtype=torch.uint8, device="cuda")
    wide_x[:, 16: 16 + b], wide_w[:, :b] = x, w
    buf, out = strided(n, m, dtype, 3, 1)
    rg.rg_rows8_product(wide_x[:, 16: 16 + b], wide_w[:, :b], d, out=out)
    assert torch.equal(out, want)
    out.fill_(3.0)
    assert bool((buf == 3).all())


def gradient_reference(dy, qx, sx, qw, sw):
    g = dy.double()
    return dict(dx=(g * sw.double()) @ qw, dweight=(g * sx.double()[:, None]).t().contiguous() @ qx, dbias=g.sum(0))


def gradient_bounds(dy, qx, sx, qw, sw):
    n, m = dy.shape
    g, parts = dy.double().abs(), 3 if dy.dtype == torch.float32 else 2
    term = U + (0 if parts == 3 else 2.0 ** -16) + 2.0 ** -40

    def of(k):
        return term + 2.0 ** -23 * (parts * (k / 8 + 8) + 512 * (k > 512))
    return dict(dx=of(m) * ((g * sw.double().abs()) @ qw.abs()), dweight=of(n) * ((g * sx.double().abs()[:, None]).t().contiguous() @ qx.abs()), dbias=(64 + n / 256) * U * g.sum(0))


GRADIENTS = [(1, 1, 1), (1, 300, 200), (300, 1, 33), (2, 3, 13), (64, 64, 64), (65, 63, 129), (130, 257, 1001), (1000, 41, 602), (33, 700, 28), (256, 256, 256), (5000, 17, 60), (513, 255, 300), (4099, 130, 515),
             (20_000, 64, 128), (16, 2048, 1024), (300, 3000, 96), (40_000, 47, 256), (33_000, 130, 64), (70_001, 256, 130), (600, 1030, 770)]


@pytest.mark.parametrize("n,m,d", GRADIENTS)
@pytest.mark.parametrize("dtype,weight", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16)], ids=str)
def test_gradients(rg, n, m, d, dtype, weight):
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    dy = made(n, m, dtype, 7)
    dx, dw, db = rg.rg_rows8_product_backward(dy, x, w, d, weight_dtype=weight)
    assert (dx.dtype, dw.dtype, db.dtype) == (dtype, weight, weight)
    ref, tol = gradient_reference(dy, qx, sx, qw, sw), gradient_bounds(dy, qx, sx, qw, sw)
    for name, got in (("dx", dx), ("dweight", dw), ("dbias", db)):
        check(name, got, ref[name], tol[name])


@pytest.mark.parametrize("n,m,d", [(1, 1, 1), (40, 48, 100), (63, 65, 13), (300, 270, 130)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradients_without_roundings(rg, n, m, d, dtype):
    """Few terms of whole numbers times powers of two: every product and sum has a place in 24 bits, so that nothing may be off at all.  dy * scale takes 16 bits."""
    g = torch.Generator().manual_seed(n + d)
    codes = lambda r: torch.randint(-127, 128, (r, d), generator=g)                                        # noqa: E731
    cx, cw = codes(n), codes(m)
    sx, sw = torch.full((n,), 129.0 / 128), torch.full((m,), 255.0 / 4)
    dy = torch.zeros(n, m)
    for i in range(max(n, m)):                                                                             # up to two of a row and of a column
        dy[i % n, (i * 7) % m] = float(torch.randint(129, 256, (1,), generator=g))
    if n > 1 and m > 1:
        dy[torch.rand(n, m, generator=g) < 0.5] = 0
    x, w, dy = packed(cx, sx), packed(cw, sw), dy.to(dtype).cuda()
    dx, dw, db = rg.rg_rows8_product_backward(dy, x, w, d, weight_dtype=torch.float32)
    ref = gradient_reference(dy, cx.double().cuda(), sx.cuda(), cw.double().cuda(), sw.cuda())
    most = 2.0 ** 24 / 128                                                                                 # of sums of whole numbers / 128
    for name, got in (("dweight", dw), ("dbias", db)):
        assert float(ref[name].abs().max()) < most and torch.equal(got.double(), ref[name]), name
    assert torch.equal(dx, ref["dx"].float().to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,m,d", [(3, 5, 13), (300, 270, 602), (65, 1000, 129)])
def test_strides_of_the_backward_pass(rg, dtype, n, m, d):
    x, w = random_held(n, d, 1)[0], random_held(m, d, 2)[0]
    dy = made(n, m, dtype, 7, pad=3, lead=1)
    want = rg.rg_rows8_product_backward(dy.contiguous(), x, w, d)
    b = held_bytes(d)
    wide_x = torch.full((n, b + 48), 255, dtype=torch.uint8, device="cuda")
    wide_w = torch.full((m, b + 16), 254, dtype=torch.uint8, device="cuda")
    wide_x[:, 16: 16 + b], wide_w[:, :b] = x, w
    buf, out = strided(n, d, dtype, 5, 1)
    got = rg.rg_rows8_product_backward(dy, wide_x[:, 16: 16 + b], wide_w[:, :b], d, out=out)
    assert got[0] is out and all(torch.equal(a, b) for a, b in zip(got, want))
    out.fill_(3.0)
    assert bool((buf == 3).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,m,d", [(300, 70, 100), (5000, 517, 64), (40, 3, 602)])
def test_gradients_of_a_broadcast(rg, dtype, n, m, d):
    """One row of dy for all rows: a stride of zero."""
    x, w = random_held(n, d, 1)[0], random_held(m, d, 2)[0]
    dy = made(1, m, dtype, 7).expand(n, m)
    assert dy.stride(0) == 0
    for a, b in zip(rg.rg_rows8_product_backward(dy, x, w, d), rg.rg_rows8_product_backward(dy.contiguous(), x, w, d)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,m,d", [(70, 5, 33), (1000, 70, 100), (3000, 517, 300)])
def test_nothing_beyond_a_row_counts(rg, dtype, n, m, d):
    """What lies between dy's rows, and beside codes that a row's end cuts off, is not a number."""
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    buf, dy = strided(n, m, dtype, 11, 3, fill=float("nan"))
    dy.copy_(made(n, m, dtype, 7))
    for name, got in zip(("dx", "dweight", "dbias"), rg.rg_rows8_product_backward(dy, x, w, d)):
        check(name, got, gradient_reference(dy, qx, sx, qw, sw)[name], gradient_bounds(dy, qx, sx, qw, sw)[name])


@pytest.mark.parametrize("wanted", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)])
@pytest.mark.parametrize("n,m,d", [(70, 30, 100), (3000, 64, 128), (20, 2000, 300)])
def test_what_is_not_wanted(rg, wanted, n, m, d):
    x, w = random_held(n, d, 1)[0], random_held(m, d, 2)[0]
    dy = made(n, m, torch.bfloat16, 7)
    whole = rg.rg_rows8_product_backward(dy, x, w, d)
    got = rg.rg_rows8_product_backward(dy, x if wanted[1] else None, w if wanted[0] else None, d, want_dx=bool(wanted[0]), want_dweight=bool(wanted[1]), want_dbias=bool(wanted[2]))
    for k in range(3):
        assert (got[k] is None) == (not wanted[k]) and (got[k] is None or torch.equal(got[k], whole[k]))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradients_with_infinities_and_nan(rg, dtype):
    """An infinity times a code of zero is a NaN, as the formula has it; elsewhere it stays an infinity, and what it does not reach stays as it was."""
    n, m, d = 70, 40, 100
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    qx[3], qw[5] = 1, 1
    qx[3, 0], qw[5, 0] = 0, 0
    x, w = packed(qx, sx), packed(qw, sw)
    dy = made(n, m, dtype, 7)
    clean = rg.rg_rows8_product_backward(dy, x, w, d)
    dy[3, 5] = float("inf")
    dx, dw, db = rg.rg_rows8_product_backward(dy, x, w, d)
    assert bool(torch.isnan(dx[3, 0])) and bool((dx[3, 1:] == float("inf")).all()) and bool(torch.isnan(dw[5, 0])) and bool((dw[5, 1:] == float("inf")).all()) and float(db[5]) == float("inf")
    for a, b, row in ((dx, clean[0], 3), (dw, clean[1], 5)):
        keep = torch.arange(a.shape[0], device="cuda") != row
        assert torch.equal(a[keep], b[keep])
    dy[3, 5] = float("nan")
    dx, dw, db = rg.rg_rows8_product_backward(dy, x, w, d)
    assert bool(torch.isnan(dx[3]).all()) and bool(torch.isnan(dw[5]).all()) and bool(torch.isnan(db[5])) and not bool(torch.isnan(db[6]))
    sx[9] = float("nan")
    dx, dw, db = rg.rg_rows8_product_backward(clean[0].new_ones(n, m), packed(qx, sx), w, d)
    assert bool(torch.isfinite(dx).all()) and bool(torch.isnan(dw).all()) and bool(torch.isfinite(db).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradients_of_every_size(rg, dtype):
    """dy near the ends of its type's range, where parts of 16 bits have theirs: no infinity comes out of numbers."""
    n, m, d = 33, 20, 70
    f = torch.finfo(dtype)
    x, qx, sx = random_held(n, d, 1, spread=0)
    w, qw, sw = random_held(m, d, 2, spread=0)
    big = min(float(f.max), 1e35)
    for size in (big, max(float(f.tiny) * 64, 2.0 ** -86)):
        dy = (made(n, m, torch.float32, 7).clamp(-1, 1) * size).to(dtype)
        dx, dw, db = rg.rg_rows8_product_backward(dy, x, w, d, weight_dtype=torch.float32)
        ref, tol = gradient_reference(dy, qx, sx, qw, sw), gradient_bounds(dy, qx, sx, qw, sw)
        for name, got in (("dweight", dw), ("dbias", db)) + ((("dx", dx),) if dtype != torch.float16 else ()):
            check(name, got, ref[name], tol[name])


@pytest.mark.parametrize("n,m,d", [(0, 5, 13), (5, 0, 13), (0, 0, 1)])
def test_nothing(rg, n, m, d):
    x = torch.empty((n, held_bytes(d)), dtype=torch.uint8, device="cuda")
    w = torch.empty((m, held_bytes(d)), dtype=torch.uint8, device="cuda")
    assert rg.rg_rows8_product(x, w, d).shape == (n, m)
    dx, dw, db = rg.rg_rows8_product_backward(torch.empty((n, m), device="cuda"), x, w, d)
    assert bool((dx == 0).all()) and bool((dw == 0).all()) and bool((db == 0).all())
    assert dx.shape == (n, d) and dw.shape == (m, d) and db.shape == (m,)
    assert rg.rg_quantize_rows(torch.empty((0, d), device="cuda")).shape[0] == 0


def test_gradients_are_the_differences(rg):
    """y is linear in what a code stands for: one more of a code changes <dy, y> by its scale times its gradient."""
    n, m, d = 37, 29, 50
    x, qx, sx = random_held(n, d, 1)
    w, qw, sw = random_held(m, d, 2)
    dy = made(n, m, torch.float32, 3)
    dx, dw, db = rg.rg_rows8_product_backward(dy, x, w, d)
    qx.clamp_(-126, 126)
    qw.clamp_(-126, 126)

    def loss(a, b):
        return (dy.double() * rg.rg_rows8_product(packed(a, sx), packed(b, sw), d).double()).sum()
    dx, dw, _ = rg.rg_rows8_product_backward(dy, packed(qx, sx), packed(qw, sw), d)
    size = (dy.double().abs().sum(0) * sw.double()).max() * d * 127 * 127 * sx.double().max()              # of the sums that the differences are made of
    for k in range(12):
        i, j, c = k * 3, k * 2 + 1, k * 4
        up, down = qx.clone(), qx.clone()
        up[i, c] += 1
        down[i, c] -= 1
        assert abs(float((loss(up, qw) - loss(down, qw)) / 2 - sx[i].double() * dx[i, c].double())) <= 4 * U * float(size)
        up, down = qw.clone(), qw.clone()
        up[j, c] += 1
        down[j, c] -= 1
        assert abs(float((loss(qx, up) - loss(qx, down)) / 2 - sw[j].double() * dw[j, c].double())) <= 4 * U * float(size)


def run_all(rg, x32, rows, w, bias, dy, d, **kw):
    """The calls as a layer makes them: rows held, the product, its gradients, rows read back."""
    held = rg.rg_quantize_rows(x32, rows=rows, **kw)
    y = rg.rg_rows8_product(held, w, d, bias=bias, dtype=dy.dtype, **kw)
    dx, dw, db = rg.rg_rows8_product_backward(dy, held, w, d, **kw)
    return held, y, dx, dw, db, rg.rg_dequantize_rows(held, d, dtype=dy.dtype, **kw)


SIZES = [(1500, 96, 200), (3, 700, 1001), (700, 300, 64), (300, 200, 9000)]


def inputs(n, m, d, seed=0):
    x = made(n + 10, d, torch.float32, seed)
    rows = torch.randperm(n + 10, generator=torch.Generator().manual_seed(seed))[:n].cuda()
    return x, rows, random_held(m, d, 2)[0], torch.randn(m, device="cuda"), made(n, m, torch.bfloat16, seed + 1)


@pytest.mark.parametrize("n,m,d", SIZES)
def test_the_same_call_gives_the_same_bits(rg, n, m, d):
    a = inputs(n, m, d)
    first = run_all(rg, *a, d)
    torch.empty(1 << 28, dtype=torch.uint8, device="cuda").fill_(255)
    for _ in range(3):
        for u, v in zip(run_all(rg, *a, d), first):
            assert torch.equal(u, v)


@pytest.mark.parametrize("n,m,d", SIZES)
def test_another_stream(rg, n, m, d):
    a = inputs(n, m, d)
    first = run_all(rg, *a, d)
    side = torch.cuda.Stream()
    got = run_all(rg, *a, d, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for u, v in zip(got, first):
        assert torch.equal(u, v)


@pytest.mark.parametrize("n,m,d", SIZES)
def test_captured_and_replayed(rg, n, m, d):
    """Two graphs that share their workspaces, replayed by turns on changed inputs, with eager work between."""
    a = inputs(n, m, d)
    dt = a[4].dtype
    works = [torch.empty(max(rg.rg_rows8_product_workspace(n, m, d, dt), 16), dtype=torch.uint8, device="cuda"),
             torch.empty(max(rg.rg_rows8_product_backward_workspace(n, m, d, dt), 16), dtype=torch.uint8, device="cuda")]

    def step():
        held = rg.rg_quantize_rows(a[0], rows=a[1])
        y = rg.rg_rows8_product(held, a[2], d, bias=a[3], dtype=dt, workspace=works[0])
        return (held, y, *rg.rg_rows8_product_backward(a[4], held, a[2], d, workspace=works[1]), rg.rg_dequantize_rows(held, d, dtype=dt))
    step()
    graphs = []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for turn in range(4):
        b = inputs(n, m, d, seed=turn + 5)
        for to, fr in zip(a, b):
            to.copy_(fr)
        works[0].fill_(255)
        works[1].fill_(255)
        want = run_all(rg, *b, d)
        g, out = graphs[turn % 2]
        g.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, want):
            assert torch.equal(u, v)


def test_two_calls_at_once(rg):
    """On two streams, each with its own workspace."""
    a = [inputs(n, m, d, 3) for n, m, d in SIZES]
    want = [run_all(rg, *x, s[2]) for x, s in zip(a, SIZES)]
    streams = [torch.cuda.Stream() for _ in SIZES]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [run_all(rg, *x, s[2], stream=st) for x, s, st in zip(a, SIZES, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for u, v in zip(g, w):
                assert torch.equal(u, v)


def test_workspaces(rg):
    """Just as many bytes as are asked for are enough, and no byte behind them is touched."""
    for n, m, d in SIZES + [(30_000, 64, 100)]:
        x, rows, w, bias, dy = inputs(n, m, d)
        held = rg.rg_quantize_rows(x, rows=rows)
        sizes = rg.rg_rows8_product_workspace(n, m, d, dy.dtype), rg.rg_rows8_product_backward_workspace(n, m, d, dy.dtype)
        for size, call in zip(sizes, (lambda ws: [rg.rg_rows8_product(held, w, d, dtype=dy.dtype, workspace=ws)], lambda ws: rg.rg_rows8_product_backward(dy, held, w, d, workspace=ws))):
            buf = torch.full((size + 4096,), 171, dtype=torch.uint8, device="cuda")
            for u, v in zip(call(buf[:size]), call(None)):
                assert torch.equal(u, v)
            assert bool((buf[size:] == 171).all())


def test_what_is_refused(rg):
    x, w = random_held(5, 100, 1)[0], random_held(7, 100, 2)[0]
    dy = torch.ones((5, 7), device="cuda")
    for call in (lambda: rg.rg_rows8_product(x, w, 101 + 16), lambda: rg.rg_rows8_product(x[:, 1:], w, 100), lambda: rg.rg_rows8_product(x, random_held(7, 300, 2)[0], 100),
                 lambda: rg.rg_rows8_product(x, w, 100, bias=torch.ones(6, device="cuda")), lambda: rg.rg_rows8_product(x, w, 100, out=torch.ones((5, 8), device="cuda")),
                 lambda: rg.rg_rows8_product(x.cpu(), w, 100), lambda: rg.rg_quantize_rows(torch.ones(3, 4)), lambda: rg.rg_quantize_rows(dy.t()),
                 lambda: rg.rg_quantize_rows(dy, rows=torch.ones(3, device="cuda")), lambda: rg.rg_quantize_rows(dy, rows=torch.ones(3, dtype=torch.int64)),
                 lambda: rg.rg_quantize_rows(dy, out=torch.empty((4, 16), dtype=torch.uint8, device="cuda")), lambda: rg.rg_dequantize_rows(x, 100, out=torch.ones((4, 100), device="cuda")),
                 lambda: rg.rg_rows8_product_backward(dy, w, x, 100), lambda: rg.rg_rows8_product_backward(dy, x, w, 100, out=torch.ones((5, 101), device="cuda"))):
        with pytest.raises(AssertionError):
            call()
    big = torch.full((5 * 130,), 0, dtype=torch.uint8, device="cuda")
    odd = big[: 5 * 128].view(5, 128)[:, 8: 120]
    with pytest.raises(rg.RgError) as e:
        rg.rg_dequantize_rows(odd, 100)
    assert e.value.status == rg.RG_EINVAL
    need = rg.rg_rows8_product_backward_workspace(5, 7, 100, torch.float32)
    assert need > 0
    with pytest.raises(rg.RgError) as e:
        rg.rg_rows8_product_backward(dy, x, w, 100, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == rg.RG_ERANGE
