"""Launch shapes of layer norm, computed on the host and compiled by themselves: a shape holds its row, and there is a kernel for it."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_05207_amd", "csrc")
DRIVER = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    long long rows, cols, bytes, cu, backward;
    while (scanf("%lld %lld %lld %lld %lld", &rows, &cols, &bytes, &cu, &backward) == 5) {
        const rg::NormShape s = rg::norm_shape(rows, cols, (int)bytes, (int)cu, backward != 0, false);
        printf("%d %d %d %u %u %u\n", s.pack, s.lanes, s.packs, s.grid, s.n_partial, s.column_grid);
    }
}
"""
KERNELS = {(8, 1), (16, 1), (32, 1), (64, 1), (64, 2), (64, 3), (64, 4), (256, 1), (256, 2), (256, 3), (256, 4), (1024, 1), (1024, 2), (1024, 3), (1024, 4)}


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    d = tmp_path_factory.mktemp("shapes")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(d / "driver"), str(d / "driver.cpp")])

    def ask(cases):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in cases) + "\n"
        out = subprocess.run([str(d / "driver")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [[int(x) for x in line.split()] for line in out[: len(cases)]]
    return ask


@pytest.mark.parametrize("element", [2, 4])
@pytest.mark.parametrize("backward", [0, 1])
def test_every_width_has_a_kernel_that_holds_it(shapes, element, backward):
    widths = list(range(1, 2100)) + [k * 256 + d for k in range(9, 140) for d in (-1, 0, 1, 7)] + [65_535, 131_071, 2**20 + 1, 2**31 - 1]
    for cols, (pack, lanes, packs, grid, n_partial, column_grid) in zip(widths, shapes([(1000, c, element, 256, backward) for c in widths])):
        full = 16 // element
        assert pack == (full if cols >= full else 1)
        if lanes == 0:
            assert cols > (16_384 if backward or element == 4 else 32_768)
            assert 1 <= n_partial <= 1000 and column_grid * 256 * full >= cols
            continue
        assert (lanes, packs) in KERNELS and pack * packs <= (16 if backward else 32), (cols, lanes, packs)
        assert (packs - 1) * lanes * pack < cols <= packs * lanes * pack          # only a lane's last pack can leave the row


@pytest.mark.parametrize("rows", [0, 1, 3, 255, 100_000, 2**31, 2**40 - 1])
@pytest.mark.parametrize("cols", [1, 64, 602, 8192, 40_000, 2**31 - 1])
def test_grids(shapes, rows, cols):
    for element in (2, 4):
        pack, lanes, packs, grid, n_partial, column_grid = shapes([(rows, cols, element, 256, 1)])[0]
        assert 1 <= grid <= 2048
        assert n_partial <= max(rows, 0) and (n_partial > 0) == (rows > 0) and n_partial <= 65_535
        assert column_grid < 2**31


LAUNCHES = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    long long rows, cols, bytes, cu, backward, in_place;
    while (scanf("%lld %lld %lld %lld %lld %lld", &rows, &cols, &bytes, &cu, &backward, &in_place) == 6) {
        const rg::NormShape s = rg::norm_shape(rows, cols, (int)bytes, (int)cu, backward != 0, in_place != 0);
        printf("%u %u %u %u\n", s.grid, s.column_grid, s.sum_grid, s.parts);
    }
}
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    (d / "driver.cpp").write_text(LAUNCHES)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(d / "driver"), str(d / "driver.cpp")])

    def ask(cases):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in cases) + "\n"
        out = subprocess.run([str(d / "driver")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [[int(x) for x in line.split()] for line in out[: len(cases)]]
    return ask


@pytest.mark.parametrize("element", [2, 4])
@pytest.mark.parametrize("backward", [0, 1])
def test_no_launch_is_past_the_limit_of_work_items(launches, element, backward):
    """Threads of a workgroup: at most 1,024 for rows, 256 for columns of long rows, 1,024 for the partial sums."""
    cases = [(r, c, element, cu, backward, p) for r in (1, 7, 1000, 2**40 - 1) for c in (1, 602, 40_000, 2**27 - 32, 2**27 - 31, 2**27, 2**29 + 1, 2**31 - 1) for cu in (4, 256) for p in (0, 1)]
    for (rows, cols, _, cu, _, in_place), (grid, column_grid, sum_grid, parts) in zip(cases, launches(cases)):
        for g, threads in ((grid, 1024), (column_grid, 256), (sum_grid, 1024)):
            assert g * threads < 2**32, (rows, cols, g)
        assert 1 <= sum_grid <= (cols + 31) // 32 and (sum_grid == (cols + 31) // 32 or (sum_grid + 1) * 1024 >= 2**32)
        assert parts == 1 or not in_place                      # a row whose place the result takes has one workgroup
