"""The low-rank activations of batches of more than 1024 tiles of 16 rows, a wavefront for 32 rows each, against the plain forms in 64 bits."""
import numpy as np
import pytest

import plain64
import test_gpu_adapter as base
from gpu_util import say
from test_gpu_adapter import ctx  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
# Lengths with tails of every kind behind 32; rows without adapter, an adapter of rank 0, one of a single row; ranks that end inside 16 and 8.
LENGTHS, OF = [7000, 33, 4001, 0, 1, 2999, 16, 4500, 47, 15], [0, 1, 2, 3, 4, -1, 1, 0, 5, 2]
RANKS = {16: [16, 9, 1, 16, 8, 0], 24: [24, 17, 9, 3, 16, 0], 32: [32, 25, 17, 32, 1, 0], 64: [64, 33, 48, 5, 57, 0], 128: [128, 65, 100, 16, 127, 0]}
SHAPES = [(136, 264), (40, 24), (8, 8), (384, 96)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("room", RANKS)
@pytest.mark.parametrize("n_in,n_out", SHAPES)
def test_many_rows(ctx, room, n_in, n_out, dtype):
    import torch
    say("many rows", room, n_in, n_out, dtype)
    base.BATCHES["many more rows"] = LENGTHS, OF, RANKS[room]
    p = base.Problem(ctx, "many more rows", n_in, n_out, dtype, pad=8 if n_in == 40 else 0)
    del base.BATCHES["many more rows"]
    assert p.R == room and p.T > 16384
    want, low64 = plain64.project(p.x64, p.w64, p.bias.double().cpu().numpy(), p.down64, p.up64, *p.plan)
    _, mag, mag_low = base.sizes(p)
    out, low = p.forward(keep=True)
    base.close(low, low64, "float32", base.steps(n_in) * mag_low, "low")
    assert bool((low == 0).cpu().numpy()[mag_low == 0].all())
    base.close(out, want, dtype, (base.steps(n_in) + base.steps(p.R) + 2.0 ** -16) * mag, "out")
    assert bool((p.forward() == out).all())
    a = np.abs
    low64 = low.double().cpu().numpy()
    want = plain64.project_backward(p.dout64, p.x64, low64, p.w64, p.down64, p.up64, *p.plan)
    mag = plain64.project_backward(a(p.dout64), a(p.x64), a(low64), a(p.w64), a(p.down64), a(p.up64), p.lengths, p.of, p.ranks, a(p.plan[3]))
    dx, ddown, dup = p.backward(low)
    base.close(dx, want[0], dtype, (base.steps(n_out) + base.steps(p.R) + 2.0 ** -16) * mag[0], "dx")
    base.close(ddown, want[1], "float32", (base.steps(n_out) + base.steps(p.T) + 2.0 ** -22) * mag[1], "ddown")
    base.close(dup, want[2], "float32", (base.steps(p.T) + 2.0 ** -22) * mag[2], "dup")
    for got, m in ((ddown, mag[1]), (dup, mag[2])):
        assert bool((got == 0).cpu().numpy()[m == 0].all())
    # another request's infinities, in this kernel too
    rest = torch.ones(p.T, dtype=torch.bool, device="cuda:0")
    for o, rows in plain64.request_rows(p.lengths, p.of):
        if o == 0:
            rest[rows] = False
    p.up[0], p.down[0] = float("inf"), float("nan")
    got, got_low = p.forward(keep=True)
    assert bool((got[rest] == out[rest]).all()) and bool((got_low[rest] == low[rest]).all())
    p.close()
