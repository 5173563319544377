"""The launches of an 8-bit product (csrc/int8_plan.h), on the CPU: they take every
row once, and none has the 2^32 threads that the runtime refuses."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2102_08550_amd", "csrc")
SHIM = r"""
#include "int8_plan.h"
extern "C" int launches(int64_t rows, int in, int outs, int64_t* out, int most) {
  int n = 0;
  oscars::i8_launches(rows, in, outs, [&](int tile, int64_t at, int64_t count) {
    if (n == most) return false;
    out[4 * n] = tile;
    out[4 * n + 1] = at;
    out[4 * n + 2] = count;
    out[4 * n + 3] = oscars::i8_threads(tile);
    ++n;
    return true;
  });
  return n;
}
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("int8_plan")
    src, lib = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-fPIC", "-shared",
                    "-I", CSRC, str(src), "-o", str(lib)], check=True)
    fn = ctypes.CDLL(str(lib)).launches
    fn.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int64),
                   ctypes.c_int]

    def call(rows, inputs, outs):
        out = (ctypes.c_int64 * (4 * 4096))()
        n = fn(rows, inputs, outs, out, 4096)
        return [tuple(out[4 * i:4 * i + 4]) for i in range(n)]

    return call


def _assert_covers(parts, rows, outs):
    done = 0
    for tile, at, n, threads in parts:
        assert at == done and n > 0
        groups = -(-outs // tile) * -(-n // tile)
        assert groups * threads < 1 << 32, (rows, outs, tile, n)
        done += n
    assert done == rows


@pytest.mark.parametrize("outs", [1, 10, 32, 33, 128, 65536])
@pytest.mark.parametrize("rows", [1, (1 << 29) - 32, 1 << 29, (1 << 29) + 5, (1 << 31) - 1])
def test_a_grid_has_less_than_2_32_threads(launches, rows, outs):
    for inputs in (1, 128, 1000, 65536):
        _assert_covers(launches(rows, inputs, outs), rows, outs)


def test_launches_take_every_row_once(launches):
    rng = random.Random(3)
    for _ in range(3000):
        rows, inputs, outs = (int(2 ** rng.uniform(0, top)) for top in (30.9, 16, 16))
        _assert_covers(launches(rows, inputs, outs), rows, outs)


def test_ordinary_calls_are_one_launch_or_two(launches):
    """The measured sizes beside the rule: tiles, and rows past whole turns of the CUs."""
    assert [p[:3] for p in launches(256, 4096, 1000)] == [(32, 0, 256)]
    assert [p[0] for p in launches(1024, 2048, 2048)] == [128]
    assert [p[0] for p in launches(4096, 4096, 4096)] == [256]
    assert len(launches(9216, 2048, 2048)) == 1
    assert [p[1:3] for p in launches(4352, 2048, 2048)] == [(0, 4096), (4096, 256)]
