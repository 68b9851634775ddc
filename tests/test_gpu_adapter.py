"""Projections with low-rank adapters and their gradients on the device against the plain forms in 64 bits."""
import numpy as np
import pytest

import plain64
from gpu_util import say

pytestmark = pytest.mark.gpu
EPS32 = 2.0 ** -24
# requests' row counts, their adapters, the adapters' ranks
BATCHES = {
    "one token": ([1], [0], [8]),
    "empty requests": ([0, 1, 0, 5, 0], [0, 1, 1, -1, 2], [16, 3, 8]),
    "single tokens": ([1] * 45, [(7 * i) % 41 - 1 for i in range(45)], [16] * 41),
    "no adapter": ([20, 30], [-1, -1], [8]),
    "rank zero": ([20, 30, 3], [0, 1, 0], [0, 5]),
    "odd ranks": ([33, 31, 64, 1, 129, 16, 0, 77], [2, 0, 1, 2, 3, -1, 4, 0], [1, 17, 24, 7, 23]),
    "large ranks": ([40, 90, 1, 5], [0, 1, 2, 0], [128, 100, 65]),
    "many rows": ([300, 511, 1, 700, 250, 90, 33, 64], [1, 0, 2, 1, -1, 2, 0, 1], [16, 9, 32]),
    "tall": ([2500, 37, 2900, 1111], [1, 0, -1, 1], [12, 16]),
}
SHAPES = [(8, 8), (40, 24), (264, 136), (384, 768), (768, 384), (1000, 776)]


@pytest.fixture(scope="module")
def ctx():
    import torch
    import paper_2506_08276_amd as L
    c = L.leann_create(dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1), torch.zeros(640, device="cuda:0"))
    yield c
    L.leann_destroy(c)


class Problem:
    def __init__(self, ctx, batch, n_in, n_out, dtype, pad=0, seed=0, gradient=True):
        import torch
        import paper_2506_08276_amd as L
        self.lengths, self.of, self.ranks = BATCHES[batch]
        rng = np.random.default_rng(seed + n_in + n_out)
        T, R, n = sum(self.lengths), (max(max(self.ranks), 1) + 7) // 8 * 8, len(self.ranks)
        self.T, self.R, self.n, self.L, self.ctx, self.dtype = T, R, n, L, ctx, dtype
        type_ = getattr(torch, dtype)

        def make(shape, scale, pad=0):
            wide = torch.full(shape[:-1] + (shape[-1] + pad,), float("nan"), dtype=type_, device="cuda:0")
            wide[..., :shape[-1]] = torch.from_numpy(rng.normal(size=shape) * scale).to(type_).to("cuda:0")
            t = wide[..., :shape[-1]]
            return t, t.double().cpu().numpy()

        self.x, self.x64 = make((T, n_in), 1.0, pad)
        self.dout, self.dout64 = make((T, n_out), 0.1, pad)
        self.w, self.w64 = make((n_out, n_in), 0.05)
        self.down, self.down64 = make((n, R, n_in), 1 / np.sqrt(n_in))
        self.up, self.up64 = make((n, n_out, R), 0.05)
        self.bias = torch.from_numpy(rng.normal(size=n_out).astype(np.float32)).to("cuda:0")
        self.scales = (rng.uniform(0.25, 2, size=n) * rng.choice([-1, 1], size=n)).astype(np.float32)
        for a, r in enumerate(self.ranks):  # beyond the rank, and in adapters without rows: anything
            self.down[a, r:], self.up[a, :, r:] = float("nan"), float("inf")
            if not any(m and o == a for m, o in zip(self.lengths, self.of)):
                self.down[a], self.up[a] = float("inf"), float("nan")
        self.proj = L.leann_projection_create(ctx, self.w, self.bias, gradient=gradient)
        self.rows = L.leann_adapter_rows_create(ctx, self.lengths, self.of, self.ranks, self.scales, R)
        self.plan = (self.lengths, self.of, self.ranks, self.scales.astype(np.float64))

    def close(self):
        self.L.leann_projection_free(self.proj)
        self.L.leann_adapter_rows_free(self.rows)

    def forward(self, **kw):
        return self.L.leann_adapter_project(self.ctx, self.proj, self.rows, self.x, self.down, self.up, **kw)

    def backward(self, low, **kw):
        return self.L.leann_adapter_project_backward(self.ctx, self.proj, self.rows, self.dout, self.x, low, self.down, self.up, **kw)


def close(got, want, dtype, error, what):
    """One rounding to dtype of a value that is off by at most `error`."""
    u, tiny = plain64.ROUND[dtype]
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - (error * (1 + u) + u * np.abs(want) + tiny)
    assert (off <= 0).all(), (what, off.max(), np.unravel_index(off.argmax(), off.shape))


def sizes(p, low=None):
    """Sums of magnitudes, which the errors scale with: what plain64 computes from absolute values."""
    a = np.abs
    args = (a(p.down64), a(p.up64), p.lengths, p.of, p.ranks, a(p.plan[3]))
    base = a(p.x64) @ a(p.w64).T
    out, mag_low = plain64.project(a(p.x64), a(p.w64), a(p.bias.double().cpu().numpy()), *args)
    return base, out, mag_low


def steps(n):
    """A bound of the relative error of a sum of n exact products in fp32, added in any order: a rounding of at most 2^-23 each (the
    matrix instructions may cut off instead of rounding), and some for what is done with it."""
    return (n + 16) * 2 * EPS32


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("n_in,n_out", SHAPES)
def test_project(ctx, batch, n_in, n_out, dtype):
    say("project", batch, n_in, n_out, dtype)
    p = Problem(ctx, batch, n_in, n_out, dtype, pad=8 if n_in == 40 else 0)
    want, low64 = plain64.project(p.x64, p.w64, p.bias.double().cpu().numpy(), p.down64, p.up64, *p.plan)
    _, mag, mag_low = sizes(p)
    out, low = p.forward(keep=True)
    close(low, low64, "float32", steps(n_in) * mag_low, "low")
    assert bool((low == 0).cpu().numpy()[mag_low == 0].all())  # rows without adapter, beyond the rank
    # the low-rank activations: their sum's error, 2^-16 for what their two pieces leave out, the second sum's error; the base's sum
    error = (steps(n_in) + steps(p.R) + 2.0 ** -16) * mag
    close(out, want, dtype, error, "out")
    assert bool((p.forward() == out).all())  # without keeping, and twice the same bits
    p.close()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("n_in,n_out", SHAPES)
def test_project_backward(ctx, batch, n_in, n_out, dtype):
    import torch
    say("project backward", batch, n_in, n_out, dtype)
    p = Problem(ctx, batch, n_in, n_out, dtype, pad=16 if n_in == 40 else 0)
    low64 = plain64.project(p.x64, p.w64, 0.0, p.down64, p.up64, *p.plan)[1].astype(np.float32)
    low = torch.from_numpy(low64).to("cuda:0")
    a = np.abs
    want = plain64.project_backward(p.dout64, p.x64, low64.astype(np.float64), p.w64, p.down64, p.up64, *p.plan)
    mag = plain64.project_backward(a(p.dout64), a(p.x64), a(low64.astype(np.float64)), a(p.w64), a(p.down64), a(p.up64), p.lengths, p.of, p.ranks,
                                   a(p.plan[3]))
    dx, ddown, dup = p.backward(low)
    close(dx, want[0], dtype, (steps(n_out) + steps(p.R) + 2.0 ** -16) * mag[0], "dx")
    # a sum over n_out for the low-rank gradients, a sum over the rows; 2^-22 for what three pieces leave out
    close(ddown, want[1], "float32", (steps(n_out) + steps(p.T) + 2.0 ** -22) * mag[1], "ddown")
    close(dup, want[2], "float32", (steps(p.T) + 2.0 ** -22) * mag[2], "dup")
    for got, m in ((ddown, mag[1]), (dup, mag[2])):  # no rows, beyond the rank
        assert bool((got == 0).cpu().numpy()[m == 0].all())
    again = p.backward(low)
    assert all(bool((u == v).all()) for u, v in zip((dx, ddown, dup), again))
    assert bool((p.backward(None, need_adapters=False)[0] == dx).all())
    only = p.backward(low, need_dx=False)
    assert only[0] is None and bool((only[1] == ddown).all()) and bool((only[2] == dup).all())
    p.close()


def test_gradient_against_differences(ctx):
    """The device's gradients against central differences of the 64-bit forward."""
    p = Problem(ctx, "empty requests", 8, 8, "float16")
    _, low = p.forward(keep=True)
    grads = [g.double().cpu().numpy() for g in p.backward(low)]
    down, up = (np.nan_to_num(v, nan=0, posinf=0) for v in (p.down.double().cpu().numpy(), p.up.double().cpu().numpy()))
    values = [p.x64, down, up]
    loss = lambda v: (plain64.project(v[0], p.w64, 0.0, v[1], v[2], *p.plan)[0] * p.dout64).sum()
    for i, g in enumerate(grads):
        for j in np.ndindex(values[i].shape):
            a, b = [v.copy() for v in values], [v.copy() for v in values]
            a[i][j] += 1e-5
            b[i][j] -= 1e-5
            # the loss is linear in each value: differences are off by 1e-15 / 1e-5 x loss; dx is rounded to fp16, the others are sums of 16 terms of order 1
            assert abs((loss(a) - loss(b)) / 2e-5 - g[j]) < 1e-8 + (2.0 ** -11 * abs(g[j]) + 2.0 ** -25 if i == 0 else 0) + 2 * steps(16)
    p.close()


@pytest.mark.parametrize("batch", ["single tokens", "many rows", "tall"])
def test_requests_do_not_touch_each_other(ctx, batch):
    """Infinities and NaN in one request's rows, or in its adapter, stay with it."""
    p = Problem(ctx, batch, 264, 136, "bfloat16")
    out, low = p.forward(keep=True)
    dx, ddown, dup = p.backward(low)
    spans = plain64.request_rows(p.lengths, p.of)
    sick = next(a for a in p.of if a >= 0)
    touched = np.zeros(p.T, bool)
    for a, rows in spans:
        touched[rows] |= a == sick
    import torch
    ok = torch.from_numpy(~touched).to("cuda:0")
    others = [a for a in range(p.n) if a != sick]
    for value in (float("inf"), float("nan")):
        p.down[sick, 0, ::3] = value
        p.up[sick, ::5, 0] = value
        p.x[touched.nonzero()[0][0], 5] = value
        p.dout[touched.nonzero()[0][-1], 7] = value
        out2, low2 = p.forward(keep=True)
        dx2, ddown2, dup2 = p.backward(low2)
        assert bool((out2[ok] == out[ok]).all()) and bool((low2[ok] == low[ok]).all()) and bool((dx2[ok] == dx[ok]).all())
        assert bool((ddown2[others] == ddown[others]).all()) and bool((dup2[others] == dup[others]).all())
        assert not bool(out2[~ok].isfinite().all())
    p.close()


def test_no_rows(ctx):
    import torch
    import paper_2506_08276_amd as L
    BATCHES["none"] = ([0, 0], [0, -1], [8, 8])
    p = Problem(ctx, "none", 40, 24, "bfloat16")
    assert p.forward().shape == (0, 24)
    dx, ddown, dup = p.backward(torch.zeros((0, 8), device="cuda:0"))
    assert dx.shape == (0, 40) and bool((ddown == 0).all()) and bool((dup == 0).all())
    p.close()
    del BATCHES["none"]


def test_rows_far_apart(ctx):
    """Rows whose elements lie beyond 2^32 elements."""
    import torch
    import paper_2506_08276_amd as L
    T, ld = 66000, 65536
    wide = torch.empty((T, ld), dtype=torch.bfloat16, device="cuda:0")  # 8.7 GB
    g = torch.Generator(device="cuda:0").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda:0").bfloat16()
    x, out = wide[:, :64], wide[:, 64:192]
    x.copy_(rand(T, 64))
    w, down, up = rand(128, 64), rand(2, 16, 64), rand(2, 128, 16)
    proj = L.leann_projection_create(ctx, w, gradient=True)
    rows = L.leann_adapter_rows_create(ctx, [30000, 20000, 16000], [1, -1, 0], [16, 9], [0.5, 1.0], 16)
    y, low = L.leann_adapter_project(ctx, proj, rows, x.contiguous(), down, up, keep=True)
    L.leann_adapter_project(ctx, proj, rows, x, down, up, out=out)
    assert bool((out == y).all())
    a = L.leann_adapter_project_backward(ctx, proj, rows, out, x, low, down, up)
    b = L.leann_adapter_project_backward(ctx, proj, rows, y, x.contiguous(), low, down, up)
    assert all(bool((u == v).all()) for u, v in zip(a, b))
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)


def test_refusals(ctx):
    import ctypes as C
    import torch
    import paper_2506_08276_amd as L
    lib = L.load_library()
    EINVAL, ESHAPE = -1, -4

    def refused(status, rc):
        assert rc == status and lib.leann_last_error(None)

    w = torch.zeros((16, 16), dtype=torch.bfloat16, device="cuda:0")
    wp = w.data_ptr()
    out = C.c_void_p()
    P = lib.leann_projection_create
    ok = [ctx, wp, None, 16, 16, 1, 0, C.byref(out)]
    for i, bad, status in [(0, None, EINVAL), (1, None, EINVAL), (3, 0, EINVAL), (4, 0, EINVAL), (5, 0, EINVAL), (5, 3, EINVAL), (7, None, EINVAL),
                           (3, 12, ESHAPE), (4, 4, ESHAPE), (3, 65544, ESHAPE), (4, 65544, ESHAPE)]:
        refused(status, P(*[bad if j == i else a for j, a in enumerate(ok)]))
    ints = lambda *v: (C.c_int32 * len(v))(*v)
    floats = lambda *v: (C.c_float * len(v))(*v)
    A = lib.leann_adapter_rows_create
    ok = [ctx, ints(3, 2), ints(0, -1), 2, ints(8, 4), floats(1, 1), 2, 8, C.byref(out)]
    for i, bad, status in [(0, None, EINVAL), (1, None, EINVAL), (1, ints(3, -1), EINVAL), (2, None, EINVAL), (2, ints(0, 2), EINVAL),
                           (2, ints(0, -2), EINVAL), (3, -1, EINVAL), (4, None, EINVAL), (4, ints(9, 1), EINVAL), (4, ints(-1, 1), EINVAL),
                           (5, None, EINVAL), (5, floats(1, float("inf")), EINVAL), (6, 0, EINVAL), (7, 0, ESHAPE), (7, 12, ESHAPE), (7, 136, ESHAPE),
                           (1, ints(2**31 - 1, 2**31 - 1), ESHAPE), (8, None, EINVAL)]:
        refused(status, A(*[bad if j == i else a for j, a in enumerate(ok)]))
    proj, grad = L.leann_projection_create(ctx, w), L.leann_projection_create(ctx, w, gradient=True)
    rows = L.leann_adapter_rows_create(ctx, [3, 2], [0, -1], [8, 4], [1, 1], 8)
    x = torch.zeros((5, 16), dtype=torch.bfloat16, device="cuda:0")
    xp = x.data_ptr()
    F = lib.leann_adapter_project
    ok = [ctx, proj, rows, xp, 16, wp, wp, xp, 16, None]
    for i, bad, status in [(0, None, EINVAL), (1, None, EINVAL), (2, None, EINVAL), (3, None, EINVAL), (3, xp + 2, EINVAL), (4, 8, ESHAPE),
                           (4, 20, ESHAPE), (5, None, EINVAL), (5, wp + 8, EINVAL), (6, None, EINVAL), (7, None, EINVAL), (7, xp + 2, EINVAL),
                           (8, 8, ESHAPE), (9, xp + 4, EINVAL)]:
        refused(status, F(*[bad if j == i else a for j, a in enumerate(ok)]))
    B = lib.leann_adapter_project_backward
    ok = [ctx, grad, rows, xp, 16, xp, 16, xp, wp, wp, xp, 16, xp, xp]
    for i, bad, status in [(0, None, EINVAL), (1, None, EINVAL), (1, proj, EINVAL), (2, None, EINVAL), (3, None, EINVAL), (4, 8, ESHAPE),
                           (5, None, EINVAL), (6, 12, ESHAPE), (7, None, EINVAL), (8, None, EINVAL), (9, wp + 2, EINVAL), (10, xp + 8, EINVAL),
                           (11, 8, ESHAPE), (12, None, EINVAL), (13, None, EINVAL)]:
        refused(status, B(*[bad if j == i else a for j, a in enumerate(ok)]))
    refused(EINVAL, B(ctx, grad, rows, xp, 16, xp, 16, xp, wp, wp, None, 16, None, None))
    assert bool((x == 0).all()) and bool((w == 0).all())
    for p in (proj, grad):
        L.leann_projection_free(p)
    L.leann_adapter_rows_free(rows)
    L.leann_projection_free(None)
    L.leann_adapter_rows_free(None)


LARGE = {
    # one adapter; runs that end inside every tile; single rows among long requests; rows beyond the last tile
    "one adapter": ([11000], [0], [16]),
    "many runs": ([70, 1, 33, 400, 129, 64] * 18, [(5 * i) % 13 - 1 for i in range(108)], [16, 3, 40, 128, 64, 1, 24, 17, 8, 100, 32, 9]),
    "few adapted": ([9000, 5, 2500, 300], [-1, 0, -1, 1], [8, 33]),
    "between": ([70, 1, 33, 400, 129, 64] * 2, [(5 * i) % 13 - 1 for i in range(12)], [16, 3, 40, 128, 64, 1, 24, 17, 8, 100, 32, 9]),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("batch", LARGE)
@pytest.mark.parametrize("n_in,n_out", [(256, 1000), (776, 768), (768, 1160)])
def test_large_batches(ctx, batch, n_in, n_out, dtype):
    """Tiles of 256 rows, several per block."""
    import torch
    say("large batch", batch, n_in, n_out, dtype)
    BATCHES[batch] = LARGE[batch]
    p = Problem(ctx, batch, n_in, n_out, dtype, pad=8)
    del BATCHES[batch]
    bias = p.bias.double().cpu().numpy()
    want, low64 = plain64.project(p.x64, p.w64, bias, p.down64, p.up64, *p.plan)
    _, mag, mag_low = sizes(p)
    out, low = p.forward(keep=True)
    close(low, low64, "float32", steps(n_in) * mag_low, "low")
    close(out, want, dtype, (steps(n_in) + steps(p.R) + 2.0 ** -16) * mag, "out")
    a = np.abs
    low64 = low.double().cpu().numpy()
    want = plain64.project_backward(p.dout64, p.x64, low64, p.w64, p.down64, p.up64, *p.plan)
    mag = plain64.project_backward(a(p.dout64), a(p.x64), a(low64), a(p.w64), a(p.down64), a(p.up64), p.lengths, p.of, p.ranks, a(p.plan[3]))
    dx, ddown, dup = p.backward(low)
    close(dx, want[0], dtype, (steps(n_out) + steps(p.R) + 2.0 ** -16) * mag[0], "dx")
    close(ddown, want[1], "float32", (steps(n_out) + steps(p.T) + 2.0 ** -22) * mag[1], "ddown")
    close(dup, want[2], "float32", (steps(p.T) + 2.0 ** -22) * mag[2], "dup")
    # another request's infinities
    sick = p.of[0] if p.of[0] >= 0 else p.of[1]
    rest = torch.ones(p.T, dtype=torch.bool, device="cuda:0")
    for o, rows in plain64.request_rows(p.lengths, p.of):
        if o == sick:
            rest[rows] = False
    p.up[sick], p.down[sick] = float("inf"), float("nan")
    assert bool((p.forward()[rest] == out[rest]).all())
    p.close()


@pytest.mark.parametrize("rows", [5, 1000, 1394, 11000])
@pytest.mark.parametrize("n_in", [8, 40, 776])
def test_infinite_weights(ctx, rows, n_in):
    """An infinity of the shared weight is met once by every row, and nothing else meets it."""
    import torch
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(n_in)
    x = torch.from_numpy(rng.uniform(0.5, 1.5, size=(rows, n_in))).bfloat16().to("cuda:0")
    w = torch.from_numpy(rng.normal(size=(768, n_in))).bfloat16().to("cuda:0")
    down, up = (torch.zeros(s, dtype=torch.bfloat16, device="cuda:0") for s in ((1, 8, n_in), (1, 768, 8)))
    table = L.leann_adapter_rows_create(ctx, [rows], [-1], [8], [1.0], 8)
    outs = []
    for bad in (False, True):
        if bad:
            w[7, n_in - 1], w[765, 0] = float("inf"), float("-inf")
        proj = L.leann_projection_create(ctx, w, None, gradient=False)
        outs.append(L.leann_adapter_project(ctx, proj, table, x, down, up))
        L.leann_projection_free(proj)
    L.leann_adapter_rows_free(table)
    want = outs[0].clone()
    want[:, 7], want[:, 765] = float("inf"), float("-inf")
    assert bool((outs[1] == want).all())


def test_rows_far_apart_in_large_batches(ctx):
    """x of more than 4 GB through the tiles of large batches."""
    import torch
    import paper_2506_08276_amd as L
    T, ld, n = 66000, 40960, 256
    wide = torch.empty((T, ld), dtype=torch.bfloat16, device="cuda:0")  # 5.4 GB
    g = torch.Generator(device="cuda:0").manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda:0").bfloat16()
    x, out = wide[:, 128:128 + n], wide[:, 1024:1024 + n]
    x.copy_(rand(T, n))
    w, down, up = rand(n, n), rand(2, 24, n), rand(2, n, 24)
    proj = L.leann_projection_create(ctx, w, gradient=True)
    rows = L.leann_adapter_rows_create(ctx, [30000, 20000, 16000], [1, -1, 0], [24, 9], [0.5, 1.0], 24)
    y, low = L.leann_adapter_project(ctx, proj, rows, x.contiguous(), down, up, keep=True)
    L.leann_adapter_project(ctx, proj, rows, x, down, up, out=out)
    assert bool((out == y).all())
    a = L.leann_adapter_project_backward(ctx, proj, rows, out, x, low, down, up)
    b = L.leann_adapter_project_backward(ctx, proj, rows, y, x.contiguous(), low, down, up)
    assert all(bool((u == v).all()) for u, v in zip(a, b))
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)
