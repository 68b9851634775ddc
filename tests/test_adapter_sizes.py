"""CPU checks of the row arithmetic of projections with adapters near the largest row count (csrc/adapter_plan.h, compiled here with g++)."""
import ctypes
import os
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LARGEST = 2**31 - 257  # rows, what leann_adapter_rows_create takes
SOURCE = """
#include "adapter_plan.h"
extern "C" int has_rows(int tile, int height, int rows) { return tile_has_rows(tile, height, rows); }
extern "C" int slot(int first, int n, int base) { return chunk_slot(first, n, base); }
"""


@pytest.fixture(scope="module")
def plan():
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "plan.cpp"), "w").write(SOURCE)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2506_08276_amd", "csrc"),
                               "-o", os.path.join(d, "plan.so"), os.path.join(d, "plan.cpp")])
        yield ctypes.CDLL(os.path.join(d, "plan.so"))


def test_blocks_behind_the_last_tile(plan):
    """Grids are multiples of 8 blocks: those behind the last tile have no rows, also where their first row would be beyond 2^31."""
    for height in (32, 64):
        for rows in (1, height - 1, height, height + 1, 1000, LARGEST - height, LARGEST):
            tiles = -(-rows // height)
            for tile in range(max(0, tiles - 2), (tiles + 7) // 8 * 8):
                assert bool(plan.has_rows(tile, height, rows)) == (tile * height < rows), (tile, height, rows)


def test_slots_behind_a_chunk(plan):
    """Wavefronts ask for row numbers up to 280 slots behind their chunk: they get one that the table holds, eight on from each."""
    for n in (1, 64, 2048):
        for first in (0, 1000, LARGEST - n):
            for base in range(n + 281):
                slot = plan.slot(first, n, base)
                assert slot == first + min(base, n) and first <= slot <= LARGEST  # the table goes on for 8 at least behind the last row
