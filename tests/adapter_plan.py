"""The choice of tiles of projections with adapters (csrc/adapter_plan.h, plain host code, compiled here with g++)."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "adapter_plan.h"
extern "C" int choose(int cus, long rows, int N, int K) { return choose_project(cus, rows, N, K); }
"""


@functools.lru_cache(None)
def library():
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "plan.cpp"), "w").write(SOURCE)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2506_08276_amd", "csrc"),
                               "-o", os.path.join(d, "plan.so"), os.path.join(d, "plan.cpp")])
        return ctypes.CDLL(os.path.join(d, "plan.so"))


def tile(rows, N, K, cus=256):
    """32, 64, 256 or 96 (64 rows)."""
    return (32, 64, 256, 96)[library().choose(cus, ctypes.c_long(rows), N, K)]
