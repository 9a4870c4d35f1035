"""The choice of tile and splits of the weight gradient (csrc/cf_wgrad_plan.h),
asked on the CPU: the header is compiled into a small program."""
import os
import shutil
import subprocess

import pytest

from test_wgrad_gpu import FAR, MORE_TILES, TILES

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_03617_amd", "csrc")
CUS = 256  # of an MI355X


def run_cpp(tmp_path, body):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text('#include "cf_wgrad_plan.h"\n#include <stdio.h>\nusing namespace cf::wgrad;\n'
                   "int main() {\n%s\nreturn 0;\n}\n" % body)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    return r.stdout


def test_the_shapes_of_the_tile_tests_take_every_tile(tmp_path):
    """The tests of the tiles (test_wgrad_gpu.py) run each one whole and with its
    rows split, and with vectors that lie in their rows, that meet their ends, and
    element by element (rows shorter than a vector, or 2^25 elements apart): a
    choice that moves their shapes fails here."""
    shapes = TILES + MORE_TILES + FAR
    out = run_cpp(tmp_path, "".join(
        "{ const Plan p = plan_of(%d, %d, %d, %d); printf(\"%%d %%d %%d\\n\", p.tile, p.splits, TILES[p.tile].qb); }\n"
        % (*s, CUS) for s in shapes) + 'printf("%d\\n", TILE_COUNT);')
    lines = out.split("\n")
    seen = set()
    for n, ((rows, K, C), line) in enumerate(zip(shapes, lines)):
        tile, splits, qb = (int(v) for v in line.split())
        far = n >= len(TILES) + len(MORE_TILES)
        ends = "any" if far or K < 8 or C < qb else "shift" if K % 8 or C % qb else "even"
        seen |= {(tile, "split" if splits > 1 else "whole"), (tile, ends)}
    tiles = int(lines[len(shapes)])
    missing = {(t, k) for t in range(tiles) for k in ("whole", "split", "any", "shift", "even")} - seen
    assert not missing, missing


def test_splits_hold_all_rows_and_fit_the_room(tmp_path):
    """Splits are whole steps of 64 rows, none is empty, together they are all of
    the rows, their partial sums fit the room, and one workgroup per tile and split
    stays below 2^32 threads."""
    run_cpp(tmp_path, """
    const int sizes[] = {1, 7, 64, 100, 511, 1000, 3008, 4096, 12288, 65536, 1 << 20};
    for (int K : sizes)
        for (int C : sizes)
            for (int64_t rows = 0; rows < (int64_t)1 << 31; rows += rows / 2 + 1) {
                if ((double)K * C > 1.5e11)
                    continue;
                const Plan p = plan_of(rows, K, C, %d);
                const Tile &t = TILES[p.tile];
                const double groups = (double)tiles_of(t, K, C) * p.splits;
                const bool ok = p.splits >= 1 && p.chunk %% 64 == 0 && p.chunk * p.splits >= rows &&
                                (p.splits == 1 || (p.chunk * (p.splits - 1) < rows && p.splits * 4.0 * K * (C + 1.0) <= PART_BYTES)) &&
                                groups * 64 * t.waves < 4294967296.0;
                if (!ok) {
                    printf("rows %%lld K %%d C %%d: tile %%d, %%d splits of %%lld\\n", (long long)rows, K, C, p.tile, p.splits,
                           (long long)p.chunk);
                    return 1;
                }
            }
    """ % CUS)
