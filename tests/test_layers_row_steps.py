"""How the dropout kernels step from row to row, replayed on the host: row_step.h is compiled into a small library, and every step is compared with the
division that defines it, up to the most positions that a call may have."""
import ctypes
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1902_01981_amd", "csrc")
WRAPPER = r"""
#include "row_step.h"
extern "C" void step(int64_t *point, int *position, int points_on, int positions_on, int positions)
{
    const cr::RowPlace to = cr::row_place_on(cr::RowPlace{*point, *position}, points_on, positions_on, positions);
    *point = to.point;
    *position = to.position;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("steps")
    (d / "w.cpp").write_text(WRAPPER)
    # an overflow of a signed number wraps here, so that a step that has one is a wrong answer and not an undefined one
    subprocess.run([gxx, "-O1", "-fwrapv", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "w.cpp"), "-o", str(d / "w.so")], check=True)
    return ctypes.CDLL(str(d / "w.so"))


@pytest.mark.parametrize("positions", [1, 2, 9, 255, 256, 257, 100_000, (1 << 31) - 257, (1 << 31) - 256, (1 << 31) - 2, (1 << 31) - 1])
@pytest.mark.parametrize("apart", [1, 3, 32, 255, 256])
def test_steps(lib, positions, apart):
    """Rows `apart` apart, from the start and across the borders of the first points."""
    for first in sorted({0, 1, max(0, positions - 2 * apart - 1), max(0, positions - 1), positions, 5 * positions - 1}):
        row = first
        point, position = ctypes.c_int64(row // positions), ctypes.c_int(row % positions)
        for _ in range(8):
            row += apart
            lib.step(ctypes.byref(point), ctypes.byref(position), apart // positions, apart % positions, positions)
            assert (point.value, position.value) == (row // positions, row % positions)
