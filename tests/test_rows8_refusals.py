"""What the calls on held rows refuse, and the launch shapes they take: neither needs a GPU, since nothing is launched."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_05207_amd", "csrc")
F32, BF16, F16 = 0, 1, 2
P = 4096                                   # an address that suits everything; nothing reads it


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding, build
    build.build(force=False)
    binding.lib()
    return binding


def test_bytes(rg):
    for cols in list(range(1, 300)) + [602, 4096, rg.RG_MAX_HELD_COLS]:
        b = rg.rg_rows8_bytes(cols)
        assert b % 16 == 0 and cols + 4 <= b < cols + 20
    for cols, status in ((0, rg.RG_EINVAL), (rg.RG_MAX_HELD_COLS + 1, rg.RG_ERANGE)):
        with pytest.raises(rg.RgError) as e:
            rg.rg_rows8_bytes(cols)
        assert e.value.status == status
    assert rg.lib().rg_rows8_bytes(5, None) == rg.RG_EINVAL


def call(rg, name, order, good, **change):
    args = dict(good, **change)
    return getattr(rg.lib(), name)(*[args[k] for k in order])


QUANTIZE = ("x", "x_stride", "n", "d", "type", "rows", "n_out", "held", "held_stride", "stream")
GOOD_Q = dict(x=P, x_stride=400, n=5, d=100, type=F32, rows=P, n_out=3, held=P, held_stride=112, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(type=3), "RG_EINVAL"), (dict(d=0), "RG_EINVAL"), (dict(d=131_073), "RG_ERANGE"), (dict(n=2**40), "RG_ERANGE"), (dict(n_out=2**40), "RG_ERANGE"), (dict(x=None), "RG_EINVAL"),
    (dict(x=P + 2), "RG_EINVAL"), (dict(x_stride=402), "RG_EINVAL"), (dict(x_stride=2**41), "RG_ERANGE"), (dict(rows=None), "RG_EINVAL"), (dict(rows=P + 4), "RG_EINVAL"), (dict(held=None), "RG_EINVAL"),
    (dict(held=P + 8), "RG_EINVAL"), (dict(held_stride=120), "RG_EINVAL"), (dict(held_stride=96), "RG_EINVAL"), (dict(held_stride=2**41), "RG_ERANGE")])
def test_quantize(rg, change, status):
    assert call(rg, "rg_quantize_rows", QUANTIZE, GOOD_Q, **change) == getattr(rg, status)
    assert rg.lib().rg_last_error()


DEQUANTIZE = ("held", "held_stride", "n", "d", "rows", "n_out", "type", "out", "out_stride", "stream")
GOOD_D = dict(held=P, held_stride=112, n=5, d=100, rows=P, n_out=3, type=BF16, out=P, out_stride=200, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(type=9), "RG_EINVAL"), (dict(d=0), "RG_EINVAL"), (dict(d=131_073), "RG_ERANGE"), (dict(held=None), "RG_EINVAL"), (dict(held=P + 1), "RG_EINVAL"), (dict(held_stride=104), "RG_EINVAL"),
    (dict(rows=None), "RG_EINVAL"), (dict(out=None), "RG_EINVAL"), (dict(out=P + 1), "RG_EINVAL"), (dict(out_stride=201), "RG_EINVAL"), (dict(out_stride=198), "RG_EINVAL")])
def test_dequantize(rg, change, status):
    assert call(rg, "rg_dequantize_rows", DEQUANTIZE, GOOD_D, **change) == getattr(rg, status)


PRODUCT = ("x", "x_stride", "n", "w", "w_stride", "m", "d", "bias", "bias_type", "y", "y_stride", "type", "ws", "ws_bytes", "stream")
GOOD_P = dict(x=P, x_stride=112, n=5, w=P, w_stride=112, m=7, d=100, bias=P, bias_type=F32, y=P, y_stride=14, type=BF16, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(type=3), "RG_EINVAL"), (dict(bias_type=F16), "RG_EINVAL"), (dict(bias_type=7), "RG_EINVAL"), (dict(bias=P + 2), "RG_EINVAL"), (dict(d=0), "RG_EINVAL"), (dict(d=131_073), "RG_ERANGE"),
    (dict(n=2**30 + 1), "RG_ERANGE"), (dict(m=2**30 + 1), "RG_ERANGE"), (dict(x=None), "RG_EINVAL"), (dict(w=None), "RG_EINVAL"), (dict(x=P + 4), "RG_EINVAL"), (dict(w_stride=100), "RG_EINVAL"),
    (dict(y=None), "RG_EINVAL"), (dict(y=P + 1), "RG_EINVAL"), (dict(y_stride=12), "RG_EINVAL"), (dict(y_stride=15), "RG_EINVAL"),
    (dict(x_stride=2**24), "RG_ERANGE"), (dict(w_stride=2**24), "RG_ERANGE"), (dict(y_stride=2**41), "RG_ERANGE")])
def test_product(rg, change, status):
    assert call(rg, "rg_rows8_product", PRODUCT, GOOD_P, **change) == getattr(rg, status)


BACKWARD = ("dy", "dy_stride", "x", "x_stride", "w", "w_stride", "n", "m", "d", "type", "dx", "dx_stride", "dw", "dw_stride", "db", "weight_type", "ws", "ws_bytes", "stream")
GOOD_B = dict(dy=P, dy_stride=14, x=P, x_stride=112, w=P, w_stride=112, n=5, m=7, d=100, type=BF16, dx=P, dx_stride=200, dw=P, dw_stride=400, db=P, weight_type=F32, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(type=3), "RG_EINVAL"), (dict(weight_type=F16), "RG_EINVAL"), (dict(d=0), "RG_EINVAL"), (dict(d=131_073), "RG_ERANGE"), (dict(n=2**30 + 1), "RG_ERANGE"), (dict(m=2**30 + 1), "RG_ERANGE"),
    (dict(dy=None), "RG_EINVAL"), (dict(dy=P + 1), "RG_EINVAL"), (dict(dy_stride=13), "RG_EINVAL"), (dict(x=None), "RG_EINVAL"), (dict(w=None), "RG_EINVAL"), (dict(x_stride=104), "RG_EINVAL"),
    (dict(w=P + 8), "RG_EINVAL"), (dict(dx=P + 1), "RG_EINVAL"), (dict(dx_stride=198), "RG_EINVAL"), (dict(dw=P + 2), "RG_EINVAL"), (dict(dw_stride=396), "RG_EINVAL"), (dict(db=P + 2), "RG_EINVAL")])
def test_backward(rg, change, status):
    assert call(rg, "rg_rows8_product_backward", BACKWARD, GOOD_B, **change) == getattr(rg, status)


def test_workspaces(rg):
    b = C.c_uint64()
    L = rg.lib()
    assert L.rg_rows8_product_workspace(5, 5, 5, F32, None) == rg.RG_EINVAL and L.rg_rows8_product_workspace(5, 5, 0, F32, C.byref(b)) == rg.RG_EINVAL
    for n, m in ((0, 5), (5, 0), (0, 0)):
        b.value = 7
        assert L.rg_rows8_product_workspace(n, m, 64, F32, C.byref(b)) == rg.RG_OK and b.value == 0
    assert L.rg_rows8_product_workspace(2**31, 5, 5, F32, C.byref(b)) == rg.RG_ERANGE and L.rg_rows8_product_workspace(5, 5, 5, 9, C.byref(b)) == rg.RG_EINVAL
    assert L.rg_rows8_product_backward_workspace(5, 5, 5, F32, 1, 1, 1, None) == rg.RG_EINVAL
    assert L.rg_rows8_product_backward_workspace(5, 5, 5, 3, 1, 1, 1, C.byref(b)) == rg.RG_EINVAL


DRIVER = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    long long rows, cols, bytes, cu, read;
    while (scanf("%lld %lld %lld %lld %lld", &rows, &cols, &bytes, &cu, &read) == 5) {
        const rg::HoldShape s = read ? rg::read_shape(rows, cols, (int)bytes, (int)cu) : rg::hold_shape(rows, cols, (int)bytes, (int)cu);
        printf("%d %d %d %u %llu\n", s.pack, s.lanes, s.packs, s.grid, (unsigned long long)rg::held_bytes(cols));
    }
}
"""
READ_KERNELS = {(8, 1), (16, 1), (32, 1), (32, 2), (32, 3), (32, 4), (32, 5), (64, 3), (64, 4)}
HOLD_KERNELS = READ_KERNELS | {(64, 5), (256, 2), (256, 3), (256, 4), (256, 5), (1024, 2), (1024, 3), (1024, 4), (1024, 5)}


def test_every_width_has_a_kernel_that_holds_it(tmp_path):
    (tmp_path / "driver.cpp").write_text(DRIVER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    widths = list(range(1, 2100)) + [k * 256 + d for k in range(9, 140) for d in (-5, -4, -3, -1, 0, 1, 7)] + [65_535, 131_071, 131_072]
    cases = [(r, c, b, 256, 0) for c in widths for b in (2, 4) for r in (1, 100_000)] + [(r, c, b, 256, 1) for c in widths for b in (2, 4) for r in (1, 2**40 - 1)]
    out = subprocess.run([str(tmp_path / "driver")], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True, check=True).stdout.split("\n")
    for (rows, cols, element, cu, read), line in zip(cases, out):
        pack, lanes, packs, grid, held = map(int, line.split())
        assert held == (cols + 19) // 16 * 16 and 1 <= grid and (grid <= 8 * cu if lanes else grid * (256 if read else 1024) < 2**32)
        if read:
            assert pack == (16 // element if cols >= 16 // element else 1)
            assert (lanes, packs) in READ_KERNELS and (packs - 1) * lanes * pack < cols <= packs * lanes * pack if lanes else cols > 256 * pack
            assert pack > 1 or (lanes, packs) == (8, 1)
        else:
            assert pack == 16 // element and held % pack == 0
            if lanes == 0:
                assert held // pack > 4096
            else:
                assert (lanes, packs) in HOLD_KERNELS and (packs - 1) * lanes * pack < held <= packs * lanes * pack, (cols, lanes, packs)


WAYS = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    unsigned long long n, m, d, bytes;
    int cu;
    while (scanf("%llu %llu %llu %llu %d", &n, &m, &d, &bytes, &cu) == 5) {
        const rg::ProductCut c = rg::product_cut(n, m, d, bytes, cu);
        const rg::ThinShape s = c.way == rg::ProductWay::THIN ? rg::thin_shape(n, m, d, cu) : rg::ThinShape{};
        printf("%d %u %u %u %u %d %d\n", (int)c.way, s.outs, s.shares, s.lds, s.grid, c.splits, c.each);
    }
}
"""


def test_ways_of_the_product(tmp_path):
    """Each way is taken somewhere, launches hold its tiles, and what THIN puts into LDS fits and covers the outputs."""
    (tmp_path / "driver.cpp").write_text(WAYS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    sizes = [1, 2, 15, 16, 17, 64, 100, 999, 4096, 40_000, 150_000, 1_000_000, 2**24, 2**30]
    cases = [(n, m, d, b, cu) for n in sizes for m in sizes for d in (1, 16, 61, 64, 500, 602, 768, 769, 4096, 131_072) for b in (2, 4) for cu in (64, 256) if n * m <= 2**37]
    out = subprocess.run([str(tmp_path / "driver")], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True, check=True).stdout.split("\n")
    seen = set()
    for (n, m, d, b, cu), line in zip(cases, out):
        way, outs, shares, lds, grid, splits, each = map(int, line.split())
        seen.add(way)
        steps = -(-d // 128)
        assert splits >= 1 and (splits - 1) * each < steps <= splits * each and (splits == 1 or (way >= 3 and each >= 4))
        if way == 2:
            assert d <= 768 and outs % 32 == 0 and outs * shares >= m > outs * (shares - 1) and lds <= 160 * 1024 and outs * ((d + 15) // 16 * 16 + 8) + 16 == lds
            assert grid % shares == 0 and 0 < grid // shares <= (n + 127) // 128 and grid <= max(2 * cu, shares)
        else:
            side, threads = {0: (16, 256), 1: (16, 1024), 3: (64, 256), 4: (128, 512), 5: (128, 512), 6: (256, 512)}[way]
            assert -(-n // side) * -(-m // side) * threads * splits < 2**32, (n, m, d)
            assert splits == 1 or (-(-n // side) * -(-m // side) * splits <= 4 * cu and n * -(-m // 4) < 2**32)
    assert seen == set(range(7))


CUTS = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    unsigned long long i, j, k;
    int parts, cu, along;
    while (scanf("%llu %llu %llu %d %d %d", &i, &j, &k, &parts, &cu, &along) == 6) {
        const rg::GradCut c = rg::grad_cut(i, j, k, parts, cu, along != 0);
        const rg::ThinShape s = c.way == rg::GradWay::THIN ? rg::grad_thin_shape(i, j, k <= 32 ? 32 : k <= 64 ? 64 : k <= 128 ? 128 : 256, parts == 2 ? 32 : 16, cu) : rg::ThinShape{};
        printf("%d %llu %d %d %u %u %u %u\n", (int)c.way, (unsigned long long)c.tiles, c.splits, c.each, s.outs, s.shares, s.lds, s.grid);
    }
}
"""


def test_cuts_of_the_backward_pass(tmp_path):
    """Every split has a part of the sum and together they have all of it; launches hold the tiles; what the thin way puts into LDS fits and covers the columns."""
    (tmp_path / "driver.cpp").write_text(CUTS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    sizes = [0, 1, 31, 32, 33, 64, 255, 256, 257, 999, 4096, 40_000, 150_000, 2**24, 2**30]
    cases = [(i, j, k, p, cu, a) for i in sizes for j in (1, 60, 256, 602, 4096, 131_072) for k in sizes for p in (2, 3) for cu in (64, 256) for a in (0, 1) if i * j <= 2**37]
    out = subprocess.run([str(tmp_path / "driver")], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True, check=True).stdout.split("\n")
    seen = set()
    for (i, j, k, p, cu, a), line in zip(cases, out):
        way, tiles, splits, each, outs, shares, lds, grid = map(int, line.split())
        seen.add(way)
        if way == 4:
            assert a and 0 < k <= 256 and outs % 32 == 0 and outs * shares >= j > outs * (shares - 1) and lds <= 160 * 1024 and grid % shares == 0 and grid > 0
            continue
        ti, tj = {0: (64, 64), 1: (64, 256), 2: (128, 128), 3: (256, 256)}[way]
        assert tiles == -(-i // ti) * -(-j // tj) and 1 <= splits and each % 32 == 0 and each > 0
        assert (splits - 1) * each < max(k, 1) <= splits * each and each < 2**31
        assert splits == 1 or splits * tiles <= 4 * cu
    assert seen == set(range(5))
