"""How 4-bit products are dealt to launches: the header alone, in a CPU build."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include "mx4_plan.h"
using namespace oscars;
int main(int, char** argv) {
  const long long rows = atoll(argv[1]);
  const int in = atoi(argv[2]), outs = atoi(argv[3]);
  const Mx4Plan p = mx4_plan(rows, in, outs);
  printf("%d %.6f %.6f\n", p.tile, p.us, mx4_small_us(rows, in, outs));
  long long count = 0;
  mx4_launches(rows, in, outs, [&](int tile, int64_t at, int64_t n) {
    printf("%d %lld %lld\n", tile, (long long)at, (long long)n);
    return ++count < 1000;
  });
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("mx4_plan")
    src = d / "plan.cpp"
    src.write_text(SOURCE)
    exe = d / "plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2102_08550_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True)

    def run(rows, inputs, outs):
        out = subprocess.run([str(exe), str(rows), str(inputs), str(outs)], check=True,
                             capture_output=True, text=True).stdout.split("\n")
        tile, us, small = out[0].split()
        return int(tile), float(us), float(small), [tuple(map(int, l.split())) for l in out[1:] if l]
    return run


@pytest.mark.parametrize("rows,inputs,outs,tile", [
    (1, 1, 1, 32), (64, 512, 256, 32), (256, 4096, 1000, 32), (256, 4096, 4096, 64),
    (1024, 2048, 2048, 64), (2048, 4096, 2048, 128), (2048, 4096, 4096, 128),
    (4096, 256, 4096, 128), (4096, 4096, 4096, 256), (8192, 4096, 4096, 256)])
def test_tiles(plan, rows, inputs, outs, tile):
    """The tile that was measured fastest."""
    assert plan(rows, inputs, outs)[0] == tile


@pytest.mark.parametrize("rows,inputs,outs", [
    (1, 1, 1), (17, 784, 512), (33, 300, 4097), (8191, 4096, 4096), (2 ** 31 - 1, 1, 1),
    (2 ** 31 - 1, 4096, 2 ** 24), (5, 2 ** 24, 2 ** 24), (2 ** 31 - 1, 2 ** 24, 31)])
def test_launches_cover_the_rows(plan, rows, inputs, outs):
    tile, _, _, launches = plan(rows, inputs, outs)
    at = 0
    for t, start, n in launches[:-1] if len(launches) == 1000 else launches:
        assert t == tile and start == at and n >= 1
        threads = 512 if t == 256 else 256
        tiles = -(-outs // t) * -(-n // t)
        assert tiles * threads < 2 ** 32 and tiles < 2 ** 31
        assert n == rows - at or n % t == 0
        at += n
    if len(launches) < 1000:
        assert at == rows


def test_the_gpu_tests_reach_every_tile(plan):
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    import test_gpu_mx4
    tiles = {plan(rows, inputs, outs)[0] for outs, inputs, rows in test_gpu_mx4.PRODUCTS}
    assert tiles == {32, 64, 128, 256}


def test_the_gpu_test_of_two_launches_makes_two(plan):
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    import test_gpu_mx4
    rows, inputs, outs = test_gpu_mx4.TWO_LAUNCHES
    launches = plan(rows, inputs, outs)[3]
    assert len(launches) == 2 and launches[1][1] > 0
    assert rows - launches[1][1] < 300  # the rows that it gives values reach into the first


def test_the_gpu_tests_of_gradients_reach_the_large_tiles(plan):
    """dw's product alone; beside dx's it goes by itself too, not as small tiles."""
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    import test_gpu_mx4
    tiles = []
    for rows, inputs, outs in test_gpu_mx4.LARGE_GRADIENTS:
        dw, dx = plan(outs, rows, inputs), plan(rows, outs, inputs)
        assert rows > 256 and dw[2] + dx[2] - 3.0 > dw[1] + dx[1]
        tiles.append(dw[0])
    assert tiles == [64, 128, 256]
