"""Which matrices share bytes (csrc/adapter_plan.h, compiled here with g++), against a set of bytes; and that calls which must not overlap refuse those that do."""
import ctypes
import itertools
import os
import subprocess
import tempfile

import pytest

from gpu_util import say

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "adapter_plan.h"
extern "C" int overlap(uint64_t a, int64_t lda, int64_t ac, uint64_t b, int64_t ldb, int64_t bc, int64_t rows, int size)
{
    return rows_overlap(a, lda, ac, b, ldb, bc, rows, size);
}
"""


@pytest.fixture(scope="module")
def overlap():
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "plan.cpp"), "w").write(SOURCE)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2506_08276_amd", "csrc"),
                               "-o", os.path.join(d, "plan.so"), os.path.join(d, "plan.cpp")])
        f = ctypes.CDLL(os.path.join(d, "plan.so")).overlap
        f.argtypes = [ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
        yield lambda *a: bool(f(*a))


def test_against_sets_of_bytes(overlap):
    span = lambda at, ld, cols, rows: {at + 2 * (i * ld + c) + e for i in range(rows) for c in range(cols) for e in range(2)}
    for rows, lda, ldb in itertools.product((0, 1, 2, 5), (1, 3, 4), (1, 2, 4, 7)):
        for ac, bc in itertools.product(range(1, lda + 1), range(1, ldb + 1)):
            a = span(100, lda, ac, rows)
            for at in range(20, 190):
                assert overlap(100, lda, ac, at, ldb, bc, rows, 2) == bool(a & span(at, ldb, bc, rows)), (rows, lda, ldb, ac, bc, at)


def test_far_addresses(overlap):
    a, ld = 0x7F0000000000, 1 << 40
    assert not overlap(a, ld, 8, a + 16, ld, 8, 1 << 30, 2) and overlap(a, ld, 8, a + 14, ld, 8, 1 << 30, 2)
    assert not overlap(a, 2**63 - 1, 8, a + 16, 2**63 - 1, 8, 1, 2) and overlap(a, 2**63 - 1, 8, a, 2**63 - 1, 8, 1, 2)
    assert overlap(2**64 - 64, 8, 8, 2**64 - 32, 8, 8, 4, 2) and not overlap(2**64 - 64, 8, 8, 64, 8, 8, 4, 2)


@pytest.mark.gpu
def test_refused():
    import torch
    import paper_2506_08276_amd as L
    lib = L.load_library()
    ctx = L.leann_create(dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1), torch.zeros(640, device="cuda:0"))
    g = torch.Generator(device="cuda:0").manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda:0").bfloat16()
    T, n = 100, 64
    wide, down, up = rand(T, 256), rand(1, 8, n), rand(1, n, 8)
    proj = L.leann_projection_create(ctx, rand(n, n), gradient=True)
    rows = L.leann_adapter_rows_create(ctx, [T], [0], [8], [1.0], 8)
    x, dout, apart = wide[:, :n], wide[:, n:2 * n], wide[:, 128:192]
    before = wide.clone()
    for out in (x, wide[:, 56:56 + n], wide.view(-1)[n * 3:n * 3 + T * n].view(T, n)):
        say("out overlaps x", out.stride(), out.storage_offset())
        with pytest.raises(L.LeannError) as e:
            L.leann_adapter_project(ctx, proj, rows, x, down, up, out=out)
        assert e.value.status == -1 and "out overlaps x" in str(e.value)
    low = torch.zeros((T, 8), device="cuda:0")
    ddown, dup = torch.full((1, 8, n), 7.0, device="cuda:0"), torch.full((1, n, 8), 7.0, device="cuda:0")
    back = lambda dx, grads: lib.leann_adapter_project_backward(ctx, proj, rows, dout.data_ptr(), 256, x.data_ptr(), 256, low.data_ptr(), down.data_ptr(),
                                                                up.data_ptr(), dx.data_ptr(), 256, *grads)
    grads = ddown.data_ptr(), dup.data_ptr()
    for dx, what in ((dout, b"dx overlaps dout"), (x, b"dx overlaps x"), (wide[:, 120:184], b"dx overlaps dout")):
        assert back(dx, grads) == -1 and what in lib.leann_last_error(None)
    torch.cuda.synchronize()
    assert torch.equal(wide, before) and bool((ddown == 7).all()) and bool((dup == 7).all())
    # rows between each other's; x is not read without the adapters' gradients
    want = L.leann_adapter_project(ctx, proj, rows, x, down, up)
    assert torch.equal(L.leann_adapter_project(ctx, proj, rows, x, down, up, out=apart), want)
    want = L.leann_adapter_project_backward(ctx, proj, rows, dout, None, None, down, up, need_adapters=False)[0]
    assert back(apart, grads) == 0 and torch.equal(apart, want)
    assert back(x, (None, None)) == 0 and torch.equal(x, want)
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)
    L.leann_destroy(ctx)
