"""How the products of an orthogonalised update are cut, computed on the host and compiled by itself: every matrix has one kind, by itself alone, and
every kind a tile that there is a kernel for."""
import os
import subprocess

import pytest

from update_cases import CUT_OTHERWISE, EVERY_TILE

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_05207_amd", "csrc")
DRIVER = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    long long rows, cols, wide, copies;
    while (scanf("%lld %lld %lld %lld", &rows, &cols, &wide, &copies) == 4) {
        const rg::UpdateKind k = rg::update_kind(rows, cols, wide != 0, 256);
        const unsigned long long n = (std::min(rows, cols) + 63) / 64 * 64, m = (std::max(rows, cols) + 63) / 64 * 64;
        const int half = k.half_tile ? k.half_tile : rg::update_tile([&](int t) { return copies * rg::half_tiles(n, rg::tile_side(t)); }, 256, k.split);
        const int whole = k.whole_tile ? k.whole_tile : rg::update_tile([&](int t) { return copies * rg::whole_tiles(n, m, rg::tile_side(t)); }, 256, k.split);
        printf("%d %d %d %d %d %d\n", k.tiny, k.split, k.half_tile, k.whole_tile, half, whole);
    }
}
"""
SHARED, PAIR = 65, 129


@pytest.fixture(scope="module")
def kinds(tmp_path_factory):
    d = tmp_path_factory.mktemp("kinds")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(d / "driver"), str(d / "driver.cpp")])

    def ask(cases):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in cases) + "\n"
        out = subprocess.run([str(d / "driver")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [[int(x) for x in line.split()] for line in out[: len(cases)]]
    return ask


SIDES = [1, 2, 16, 31, 32, 33, 47, 63, 64, 65, 100, 255, 256, 257, 512, 602, 640, 1000, 1024, 1500, 2047, 2048, 4096, 9000, 16_384]


@pytest.mark.parametrize("wide", [0, 1])
@pytest.mark.parametrize("copies", [1, 12])
def test_every_matrix_has_tiles(kinds, wide, copies):
    cases = [(r, c, wide, copies) for r in SIDES for c in SIDES]
    for (r, c, _, _), (tiny, split, fixed_half, fixed_whole, half, whole) in zip(cases, kinds(cases)):
        n, m = min(r, c), max(r, c)
        assert tiny == (n <= 64 and m <= 256)
        if tiny:
            continue
        assert split == (wide or n <= 32)
        assert half in (SHARED, 64, 96, 128, PAIR, 192) and whole in (SHARED, 64, 96, 128, PAIR, 192)
        # operands in two parts: what is reflected goes by the matrix alone; and shared tiles always do
        assert fixed_half or not split
        assert half != SHARED or fixed_half == SHARED
        assert whole != SHARED or fixed_whole == SHARED


def test_the_same_either_way_round(kinds):
    a, b = kinds([(r, c, w, 3) for r in SIDES for c in SIDES for w in (0, 1)]), kinds([(c, r, w, 3) for r in SIDES for c in SIDES for w in (0, 1)])
    assert a == b


@pytest.mark.parametrize("rows,cols,wide,copies,half,whole", [
    # measured: see update_tile and update_kind
    (4096, 4096, 0, 1, 192, PAIR),
    (1024, 4096, 0, 6, 128, PAIR),
    (2048, 2048, 1, 1, 96, 128),
    (1999, 517, 1, 1, SHARED, 64),
    (256, 1204, 1, 1, SHARED, SHARED),
])
def test_tiles_by_what_is_done_first(kinds, rows, cols, wide, copies, half, whole):
    assert kinds([(rows, cols, wide, copies)])[0][4:] == [half, whole]


TILES = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    long long rows, cols, copies;
    while (scanf("%lld %lld %lld", &rows, &cols, &copies) == 3) {
        const rg::UpdateKind k = rg::update_kind(rows, cols, true, 256);
        const unsigned long long n = (std::min(rows, cols) + 63) / 64 * 64, m = (std::max(rows, cols) + 63) / 64 * 64;
        const auto half = [&](int t) { return copies * rg::half_tiles(n, rg::tile_side(t)); };
        const auto whole = [&](int t) { return copies * rg::whole_tiles(n, m, rg::tile_side(t)); };
        const auto pick = [&](int asked, auto &&count) { return asked == rg::UPDATE_TILE_SHARED ? rg::shared_tile(count, 256) : asked ? asked : rg::update_tile(count, 256, true); };
        printf("%d %d %d\n", k.tiny, k.tiny ? 0 : pick(k.half_tile, half), k.tiny ? 0 : pick(k.whole_tile, whole));
    }
}
"""
ALL_TILES = {32, SHARED, 64, 96, 128, PAIR, 192}


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    (d / "driver.cpp").write_text(TILES)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(d / "driver"), str(d / "driver.cpp")])

    def ask(cases):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in cases) + "\n"
        out = subprocess.run([str(d / "driver")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [[int(x) for x in line.split()] for line in out[: len(cases)]]
    return ask


def test_every_tile_that_the_rules_give_is_run_on_the_gpu(tiles):
    given = tiles([(r, c, k) for r in SIDES for c in SIDES for k in (1, 2, 5, 12)])
    halves, wholes = {h for t, h, _ in given if not t}, {w for t, _, w in given if not t}
    assert halves <= ALL_TILES and wholes <= ALL_TILES
    run = tiles([(r, c, 1) for r, c in EVERY_TILE])
    assert {h for _, h, _ in run} == ALL_TILES and {w for _, _, w in run} == ALL_TILES


def test_matrices_that_are_cut_otherwise_beside_others(tiles):
    alone, beside = tiles([(r, c, 1) for r, c, _ in CUT_OTHERWISE]), tiles(CUT_OTHERWISE)
    for (_, h, w), (_, half, whole) in zip(alone, beside):
        assert h == half and w != whole and not {w, whole} & {32, SHARED}


UNITS = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    for (int n_cu : {32, 64, 256})
        for (unsigned n : {100u, 300u, 500u, 700u, 1000u, 1100u})
            for (unsigned m : {100u, 1000u, 4000u, 16000u}) {
                const rg::UpdateKind k = rg::update_kind(n, m, true, n_cu);
                const unsigned long long least = n < m ? n : m, most = n < m ? m : n, units = n_cu;
                const bool whole = rg::whole_tiles(least, most, 64) <= units, half = whole || rg::half_tiles(least, 32) <= units;
                if (k.tiny) continue;
                printf("%d %d\n", (k.whole_tile == rg::UPDATE_TILE_SHARED) == whole, (k.half_tile == rg::UPDATE_TILE_SHARED) == half);
            }
}
"""


def test_tiles_are_shared_by_the_compute_units_that_there_are(tmp_path):
    (tmp_path / "driver.cpp").write_text(UNITS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    lines = subprocess.run([str(tmp_path / "driver")], capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
    assert len(lines) >= 60 and set(lines) == {"1 1"}


NARROW = r"""
#include "rg_launch.h"
#include <cstdio>
int main()
{
    for (unsigned long long m = 1; m <= 16384; ++m)
        printf("%llu %u %u %u %u\n", m, rg::narrow_part(m), rg::narrow_parts(m), rg::narrow_share(m), rg::narrow_shares(m));
}
"""


def test_columns_of_narrow_matrices_are_all_shared_out(tmp_path):
    """Parts of whole passes, shares of whole tiles, none of them empty, 32 at most, and one part where one workgroup does it all."""
    (tmp_path / "driver.cpp").write_text(NARROW)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    for line in subprocess.run([str(tmp_path / "driver")], capture_output=True, text=True, check=True).stdout.split("\n")[:-1]:
        m, part, parts, share, shares = (int(x) for x in line.split())
        assert part % 256 == 0 and share % 16 == 0
        assert (parts - 1) * part < m <= parts * part and (shares - 1) * share < m <= shares * share
        assert 1 <= parts <= 32 and 1 <= shares <= 32 and (parts == 1) == (m <= 256)


def test_what_is_narrow(tmp_path):
    """Either way round, and no wider than what the kernels hold."""
    (tmp_path / "driver.cpp").write_text(NARROW.split("int main")[0] + """int main()
{
    for (unsigned n = 1; n <= 70; ++n)
        for (unsigned m : {1u, 32u, 33u, 48u, 49u, 256u, 257u, 1024u, 1025u, 16384u})
            printf("%u %u %d %d\\n", n, m, rg::narrow(n, m), rg::narrow(m, n));
}
""")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    for line in subprocess.run([str(tmp_path / "driver")], capture_output=True, text=True, check=True).stdout.split("\n")[:-1]:
        a, b, is_narrow, turned = (int(x) for x in line.split())
        n, m = min(a, b), max(a, b)
        assert is_narrow == turned == int(n <= 36 or (n <= 48 and m > 1024))
