"""The shapes that the GPU tests of every way run are those that the rules send there, on a card of 256 compute units: a change of a rule's numbers that leaves a way without a test fails here."""
import subprocess

from rows8_ways import GRADIENTS, PRODUCTS
from test_rows8_refusals import CSRC, CUTS, WAYS


def ask(tmp_path, source, cases):
    (tmp_path / "driver.cpp").write_text(source)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    out = subprocess.run([str(tmp_path / "driver")], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True, check=True).stdout
    return [tuple(map(int, line.split())) for line in out.strip().split("\n")]


def registers(d):
    """Steps of 64 codes that a kernel of the thin way has registers for."""
    return next(k for k in (1, 2, 4, 6, 8, 10, 12) if d <= 64 * k)


FEW, FEW_LONG, THIN, TILES_64, TILES_128, TILES_128_DEEP, TILES_256 = range(7)


def test_products(tmp_path):
    for element in (2, 4):
        seen = set()
        for (n, m, d), (way, outs, shares, lds, grid, splits, each) in zip(PRODUCTS, ask(tmp_path, WAYS, [(*c, element, 256) for c in PRODUCTS])):
            seen.add((way, registers(d), shares > 1) if way == THIN else (way, splits > 1))
        assert {(FEW, False), (FEW_LONG, False)} | {(w, s) for w in (TILES_64, TILES_128, TILES_128_DEEP, TILES_256) for s in (False, True)} <= seen
        assert {s[1] for s in seen if s[0] == THIN and not s[2]} == {1, 2, 4, 6, 8, 10, 12}
        assert {s[1] for s in seen if s[0] == THIN and s[2]} >= {4, 8, 10, 12}


def test_gradients(tmp_path):
    tiles = {(w, s) for w in range(4) for s in (False, True)}
    seen = {(r[0], r[2] > 1) for r in ask(tmp_path, CUTS, [(m, d, n, 3, 256, 0) for n, m, d in GRADIENTS])}
    assert seen == tiles
    seen = set()
    for (n, m, d), (way, _, splits, _, _, shares, _, _) in zip(GRADIENTS, ask(tmp_path, CUTS, [(n, d, m, 3, 256, 1) for n, m, d in GRADIENTS])):
        seen.add((way, next(k for k in (32, 64, 128, 256) if m <= k), shares > 1) if way == 4 else (way, splits > 1))
    assert seen >= tiles | {(4, k, s) for k in (32, 64, 128, 256) for s in (False, True)}, seen


def test_launches_hold_the_tiles_of_the_largest_gradients(tmp_path):
    """Up to 2^37 elements, as of the product: a way that a launch does not hold is not chosen."""
    sizes = [1, 3, 64, 300, 2**20, 2**24, 2**28, 2**30]
    cases = [(i, j, k, 3, 256, along) for i in sizes for j in (1, 16, 64, 128, 300, 4096, 131_072) for k in (0, 1, 3, 300, 100_000, 2**30) for along in (0, 1) if i * j <= 2**37]
    for (i, j, k, _, _, _), (way, tiles, splits, *_) in zip(cases, ask(tmp_path, CUTS, cases)):
        assert way == 4 or tiles * splits * (512 if way == 3 else 256) < 2**32, (i, j, k)
