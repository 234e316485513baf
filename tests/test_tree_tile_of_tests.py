"""Which row tile the calls of the GPU tests of the tree attention take, by the rule that the library goes
by (hq_tree_tile), on the CPU: a test that names a tile reaches the kernel of that tile."""
import os
import subprocess

import pytest

from tests import test_gpu_cache_tree_full_tiles as full
from tests import test_gpu_cache_tree_range as ranges
from tests import test_gpu_cache_tree_tiles as tiles

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_23406_amd", "csrc")
PROGRAM = r"""
#include <stdio.h>
#include "hq_internal.h"
int main() {
  long batch, rows, most, heads, group, tokens, window, sinks;
  while (scanf("%ld %ld %ld %ld %ld %ld %ld %ld", &batch, &rows, &most, &heads, &group, &tokens, &window, &sinks) == 8) {
    const long all = rows < batch * most ? rows : batch * most;
    printf("%d\n", (int)hq_tree_tile(most * group, all * group, batch, heads, hq_cache_seen(tokens, window, sinks, most)));
  }
}
"""
SEQUENCES = [([0, 1, 2, 15, 16, 17, 33, 64, 65, 100, 129, 511], [0, 1, 2, 9, 16, 1, 30, 30, 5, 12, 13, 29]),
             ([3000, 1025, 40, 1024, 513], [30, 17, 30, 4, 8]), ([300, 64, 65, 80, 513, 1, 0, 2000], [20, 30, 1, 30, 30, 1, 0, 28]),
             ([400, 90, 1500], [9, 20, 30]), ([200], [4]), ([100, 70, 1300, 40], [5, 9, 30, 8]), ([300, 40, 1100], [9, 30, 20])]
WINDOWS = [(0, 0), (64, 0), (70, 17), (100, 300), (900, 5)]


@pytest.fixture(scope="module")
def tile_of(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("tree_tile")
    src, exe = tmp / "tile.cpp", tmp / "tile"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True, timeout=300)

    def of(calls):
        out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls), check=True, capture_output=True,
                             text=True, timeout=60).stdout
        return list(map(int, out.split()))

    return of


def call(all_rows):
    """A stand-in for Case (all_rows: for Full, whose calls have as many rows as all sequences could): what
    the library is called with."""
    def made(hq, fmt, lens, trees, heads, group, bt, window=0, sinks=0, max_tree=None, **kw):
        most = max_tree or max(max(trees), 1)
        rows = len(lens) * most if all_rows else sum(trees)
        return len(lens), rows, most, heads, group, max(1, -(-max(lens) // bt)) * bt, window, sinks
    return made


@pytest.fixture
def recorded(monkeypatch):
    for module in (tiles, ranges):
        monkeypatch.setattr(module, "Case", call(False))
    for module in (full, ranges):
        monkeypatch.setattr(module, "Full", call(True))


# Of tiles.py the cases named 128 take tiles of 32: their rows fill those of 128 to a few percent.
@pytest.mark.parametrize("name,tile", [("16 of few", 16), ("16 of many", 16), ("32", 32), ("128", 32)])
def test_tiles(tile_of, recorded, name, tile):
    calls = [tiles.case(None, "int8", name, *s, window=w, sinks=n) for s in SEQUENCES for w, n in WINDOWS]
    assert set(tile_of(calls)) == {tile}


def test_full_tiles(tile_of, recorded):
    calls = [full.case(None, "int8", *s, window=w, sinks=n) for s in SEQUENCES for w, n in WINDOWS]
    for heads, group in ((1, 16), (3, 5), (5, 7), (8, 4)):
        rows = min(64, 120 // group)
        calls.append(full.Full(None, "int8", [301, 64, 130] + [3] * 600, [rows] * 603, heads, group, 32, max_tree=rows))
    for group, trees in ((4, [64, 63, 50, 64]), (8, [32, 31, 16, 20]), (16, [24, 8, 7, 64])):
        calls.append(full.Full(None, "int8", [4000, 2500, 1030, 700] + [40] * 12, trees + [1] * 12, 8, group, 48, max_tree=max(trees)))
    assert set(tile_of(calls)) == {128}


@pytest.mark.parametrize("name", ranges.TILES)
def test_ranges(tile_of, recorded, name):
    calls = [ranges.case(None, "int8", name, *s) for s in SEQUENCES + [([16000], [4]), ([1], [1])]]
    assert set(tile_of(calls)) == {int(name)}
