"""Which kernel a product or a weight gradient takes (CPU), and that the sizes
the GPU tests run reach every one that the planner gives."""

import itertools
import os
import shutil
import subprocess

import pytest

from tests import linear_shapes as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_16981_amd", "csrc")
TABLES = {"product": S.PRODUCT, "exact": S.EXACT, "grad": S.GRAD}


@pytest.fixture(scope="module")
def choices(tmp_path_factory):
    """choices([(kind, rows, cols, long, workspace), ...]) -> [(tile rows, tile
    columns, whole, parts) or None for few rows, ...]."""
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe = tmp_path_factory.mktemp("choice") / "linear_choice"
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC,
                        os.path.join(ROOT, "tests", "native", "linear_choice.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]

    def ask(lines):
        text = "".join(" ".join(map(str, line)) + "\n" for line in lines)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [None if v == "few" else tuple(map(int, v.split())) for v in out.splitlines()]

    return ask


@pytest.mark.parametrize("kind", list(TABLES))
def test_the_listed_plans(choices, kind):
    got = choices([(kind, *size, S.WORKSPACE) for size in TABLES[kind]])
    assert dict(zip(TABLES[kind], got)) == TABLES[kind]


def _way(choice):
    """A kernel and what it does with its tiles."""
    bm, bn, whole, parts = choice
    return bm, bn, "last round in parts" if whole else "in parts" if parts > 1 else "not divided"


@pytest.mark.parametrize("kind", list(TABLES))
def test_every_way_is_listed(choices, kind):
    """Over a grid of sizes, odd ones and whole blocks."""
    side = [17, 63, 64, 129, 256, 383, 512, 777, 1024, 1333, 2048, 2560, 3000, 3333, 4096, 5000, 6143, 8192, 14336]
    along = [1, 33, 100, 128, 333, 600, 1000, 2048, 2049, 4096, 8000, 14336, 16384]
    sizes = itertools.product(side, side, along)
    seen = {_way(c) for c in choices([(kind, *s, S.WORKSPACE) for s in sizes]) if c}
    assert seen <= {_way(c) for c in TABLES[kind].values()}


def test_few_rows_take_no_tile(choices):
    assert choices([("product", 16, 4096, 4096, S.WORKSPACE), ("exact", 1, 1, 1, 0)]) == [None, None]


@pytest.mark.parametrize("kind", list(TABLES))
def test_sums_fit_the_workspace(choices, kind):
    """Parts only where their sums do, none without a workspace."""
    sizes = [(m, n, k) for m in (17, 300, 1111, 4096) for n in (64, 777, 4096) for k in (1000, 16384)]
    for workspace in (0, 1 << 20, 8 << 20, S.WORKSPACE):
        for (m, n, k), c in zip(sizes, choices([(kind, *s, workspace) for s in sizes])):
            bm, bn, whole, parts = c
            tiles = -(-m // bm) * -(-n // bn)
            assert parts == 1 or (tiles - whole) * parts * bm * bn * 4 <= workspace
            assert 1 <= parts <= 8 and tiles - whole <= (4096 if parts > 1 else tiles)
