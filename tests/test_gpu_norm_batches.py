"""Dropout, LayerNorm and its gradient in batches: several rows per thread, outputs past the caches, outputs in place of inputs; against the plain forms in 64 bits."""
import ctypes as C

import numpy as np
import pytest

import plain64
import test_gpu_norm as base
from gpu_util import say
from test_gpu_norm import ctx  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
EPS32, EPS = base.EPS32, base.EPS
DTYPES = base.DTYPES


def device_matrix(seed, rows, cols, dtype, pad=0, scale=1.0, shift=0.0):
    """Made on the device, rows cols + pad apart, NaN between them."""
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    wide = torch.full((rows, cols + pad), float("nan"), dtype=getattr(torch, dtype), device="cuda:0")
    wide[:, :cols] = torch.randn((rows, cols), generator=g, device="cuda:0") * scale + shift
    return wide[:, :cols]


def some_rows(rows):
    """Rows to look at: the first and last, and some between."""
    return np.unique(np.concatenate([[0, 1, rows - 2, rows - 1], np.random.default_rng(rows).integers(0, rows, 60)]).clip(0))


def f64(t, at=None):
    import torch
    return (t if at is None else t[torch.from_numpy(at).to("cuda:0")]).double().cpu().numpy()


def dropout_of(x, at, drop):
    """plain64.dropout of the rows `at` of a matrix."""
    if drop is None:
        return x
    p, seed, offset = drop
    below = int(np.rint(np.float32(p) * np.float32(65536)))
    chunks = (x.shape[1] + 7) // 8
    row, chunk = np.meshgrid(at, np.arange(chunks), indexing="ij")
    full = lambda v: np.full(row.shape, v, np.uint64)
    w = plain64.philox([chunk, row, full(offset & 0xFFFFFFFF), full(offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    bits = np.stack([h for v in w for h in (v & np.uint32(0xFFFF), v >> np.uint32(16))], -1).reshape(len(at), chunks * 8)[:, :x.shape[1]]
    return np.where(bits < below, 0.0, x * (65536 / (65536 - below)))


def rows_for(dtype, cols, at_least=96e6):
    """As many rows as make outputs of that many bytes."""
    return int(at_least / cols / {"float32": 4}.get(dtype, 2)) + 33


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(25013, 769), (2_200_001, 1), (2, 9_000_001), (140_003, 72), (None, 769), (None, 1024)])
@pytest.mark.parametrize("with_res", [False, True])
def test_dropout(ctx, dtype, rows, cols, with_res):
    """More accesses than the launch has threads (1 048 576 on 256 units); None: outputs of 96 MB and more, at odd strides."""
    import paper_2506_08276_amd as L
    pad = 3 if rows is None else 0
    rows = rows or rows_for(dtype, cols)
    say("dropout batch", dtype, rows, cols, with_res)
    x = device_matrix(1, rows, cols, dtype, pad)
    res = device_matrix(2, rows, cols, dtype) if with_res else None
    drop = (0.3, 0x123456789ABCDEF0, (3 << 32) + 5)
    out = device_matrix(3, rows, cols, dtype, pad)
    L.leann_dropout(ctx, x, drop, residual=res, out=out)
    at = some_rows(rows)
    want = dropout_of(f64(x, at), at, drop)
    r64 = f64(res, at) if with_res else 0.0
    base.close(out[at.tolist()], want + r64, dtype, 3 * EPS32 * np.abs(want) + EPS32 * np.abs(want + r64), "out")
    if with_res:  # in the residual's place
        L.leann_dropout(ctx, x, drop, residual=res, out=res)
        assert bool((res == out).all())


CASES = [(20011, 768, 0), (20011, 384, 3), (30001, 128, 0), (30001, 200, 5), (9001, 1537, 0), (4999, 3000, 1), (5003, 4100, 0), (4500, 8192, 0), (None, 769, 3), (None, 2048, 0)]


def fits(dtype, rows, cols, pad):
    rows = rows or rows_for(dtype, cols)
    return rows, f"{dtype} {rows} x {cols} + {pad}"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pad", CASES)
@pytest.mark.parametrize("drop", [None, (0.2, 77, 1 << 35)])
def test_layernorm(ctx, dtype, rows, cols, pad, drop):
    import paper_2506_08276_amd as L
    rows, name = fits(dtype, rows, cols, pad)
    say("layernorm batch", name, drop)
    rng = np.random.default_rng(cols)
    x, res = device_matrix(1, rows, cols, dtype, pad, shift=0.5), device_matrix(2, rows, cols, dtype, 0, scale=2.0)
    (gamma, g64), (beta, b64) = base.vector(rng, cols, 1.0), base.vector(rng, cols, 0.0)
    out = device_matrix(3, rows, cols, dtype, pad)
    _, total, mean, rstd = L.leann_layernorm(ctx, x, gamma, beta, EPS, residual=res, drop=drop, keep=True, out=out)
    at = some_rows(rows)
    r64 = f64(res, at)
    t64 = dropout_of(f64(x, at), at, drop) + r64
    want, mean64, rstd64 = plain64.layernorm(t64, g64, b64, EPS)
    mean_error, rel = base.norm_errors(t64, g64, rstd64)
    mean_error = mean_error + 4 * EPS32 * np.abs(t64).max(1)
    error = np.abs(g64) * (mean_error * rstd64)[:, None] + np.abs(want - b64) * rel[:, None] + 4 * EPS32 * (np.abs(want) + np.abs(b64))
    pick = at.tolist()
    base.close(out[pick], want, dtype, error, "out")
    base.close(total[pick], t64, dtype, 4 * EPS32 * (np.abs(t64) + np.abs(r64)), "total")
    base.close(mean[pick], mean64, "float32", mean_error, "mean")
    base.close(rstd[pick], rstd64, "float32", rstd64 * rel, "rstd")
    # all the rows, in calls of a part of them: their bits do not depend on the launch (dropout's row numbers would)
    if drop is None:
        for first in range(0, rows, max(1000, rows // 5)):
            of = slice(first, first + 700)
            part = L.leann_layernorm(ctx, x[of], gamma, beta, EPS, residual=res[of], keep=True)
            assert all(bool((u[of] == v).all()) for u, v in zip((out, total, mean, rstd), part)), first


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pad", CASES)
@pytest.mark.parametrize("drop,extra", [(None, True), ((0.2, 77, 1 << 35), False), ((0.1, 5, 6), True)])
def test_layernorm_backward(ctx, dtype, rows, cols, pad, drop, extra):
    import torch
    import paper_2506_08276_amd as L
    rows, name = fits(dtype, rows, cols, pad)
    say("layernorm backward batch", name, drop, extra)
    rng = np.random.default_rng(cols + 2)
    t, d = device_matrix(1, rows, cols, dtype, pad), device_matrix(2, rows, cols, dtype, 0, scale=0.1)
    e = device_matrix(4, rows, cols, dtype, pad, scale=0.1) if extra else None
    gamma, g64 = base.vector(rng, cols, 1.0)
    wide = t.double()
    mean, rstd = wide.mean(1).float(), (wide.var(1, unbiased=False) + 1e-3).rsqrt().float()
    dres, dx, dgamma, dbeta = L.leann_layernorm_backward(ctx, d, t, mean, rstd, gamma, drop=drop, dtotal=e)
    at = some_rows(rows)
    pick = at.tolist()
    d64, t64, m64, s64 = f64(d, at), f64(t, at), f64(mean, at), f64(rstd, at)
    e64 = f64(e, at) if extra else 0.0
    want = plain64.layernorm_backward(d64, t64, m64, s64, g64)[0]
    xhat = np.abs((t64 - m64[:, None]) * s64[:, None]) + EPS32 * (np.abs(t64) + np.abs(m64[:, None])) * s64[:, None]
    gy = np.abs(d64 * g64)
    error = 100 * EPS32 * s64[:, None] * (gy + gy.mean(1, keepdims=True) + xhat * (gy * xhat).mean(1, keepdims=True))
    error += 4 * EPS32 * (np.abs(want) + np.abs(e64))
    base.close(dres[pick], want + e64, dtype, error, "dresidual")
    if drop is not None:
        factor = 1 / (1 - drop[0])
        base.close(dx[pick], dropout_of(want + e64, at, drop), dtype, (error + 3 * EPS32 * np.abs(want + e64)) * factor * 1.001, "dx")
    # the sums over all rows, in 64 bits on the device
    m, s, dd = mean.double()[:, None], rstd.double()[:, None], d.double()
    depth = 64 + rows / 64
    size = (dd.abs() * ((wide.abs() + m.abs()) * s)).sum(0).cpu().numpy()
    base.close(dgamma, (dd * ((wide - m) * s)).sum(0).cpu().numpy(), "float32", depth * EPS32 * size, "dgamma")
    base.close(dbeta, dd.sum(0).cpu().numpy(), "float32", depth * EPS32 * dd.abs().sum(0).cpu().numpy(), "dbeta")
    del wide, dd
    torch.cuda.empty_cache()


IN_PLACE = [(5, 9), (20011, 768), (30001, 128), (30001, 250), (9001, 1537), (4999, 3000), (5003, 4100)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", IN_PLACE)
def test_layernorm_in_place(ctx, dtype, rows, cols):
    """out is x or the residual, total the other one or a matrix of its own."""
    import paper_2506_08276_amd as L
    say("layernorm in place", dtype, rows, cols)
    lib = L.load_library()
    rng = np.random.default_rng(cols)
    x, res = device_matrix(1, rows, cols, dtype, 3), device_matrix(2, rows, cols, dtype, 5)
    gamma, beta = base.vector(rng, cols, 1.0)[0], base.vector(rng, cols, 0.0)[0]
    code = {"float32": L.LEANN_F32, "bfloat16": L.LEANN_BF16, "float16": L.LEANN_F16}[dtype]
    for drop in (None, (0.25, 9, 10)):
        want = L.leann_layernorm(ctx, x, gamma, beta, EPS, residual=res, drop=drop, keep=True)
        desc = None if drop is None else C.byref(L.binding.DropoutDesc(*drop))
        for out_is, total_is in (("x", "res"), ("res", "x"), ("x", None), ("res", None), (None, "x"), (None, "res")):
            a, b = device_matrix(1, rows, cols, dtype, 3), device_matrix(2, rows, cols, dtype, 5)
            mean, rstd = (gamma.new_empty(rows) for _ in range(2))
            place = {"x": a, "res": b, None: device_matrix(3, rows, cols, dtype)}
            out, total = place[out_is], place[total_is]
            rc = lib.leann_layernorm(ctx, a.data_ptr(), a.stride(0), b.data_ptr(), b.stride(0), rows, cols, code, desc, gamma.data_ptr(), beta.data_ptr(), EPS,
                                     out.data_ptr(), out.stride(0), total.data_ptr(), total.stride(0), mean.data_ptr(), rstd.data_ptr())
            assert rc == 0
            assert all(bool((u == v).all()) for u, v in zip((out, total, mean, rstd), want)), (out_is, total_is)
    without = L.leann_layernorm(ctx, x, gamma, beta, EPS)
    assert L.leann_layernorm(ctx, x, gamma, beta, EPS, out=x) is x and bool((x == without).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", IN_PLACE)
def test_layernorm_backward_in_place(ctx, dtype, rows, cols):
    """dresidual and dx in the places of dout and dtotal."""
    import paper_2506_08276_amd as L
    say("layernorm backward in place", dtype, rows, cols)
    lib = L.load_library()
    rng = np.random.default_rng(cols)
    t, d, e = device_matrix(1, rows, cols, dtype, 3), device_matrix(2, rows, cols, dtype, 1, 0.1), device_matrix(4, rows, cols, dtype, 5, 0.1)
    gamma = base.vector(rng, cols, 1.0)[0]
    wide = t.double()
    mean, rstd = wide.mean(1).float(), (wide.var(1, unbiased=False) + 1e-3).rsqrt().float()
    code = {"float32": L.LEANN_F32, "bfloat16": L.LEANN_BF16, "float16": L.LEANN_F16}[dtype]
    for drop in (None, (0.25, 9, 10)):
        want = L.leann_layernorm_backward(ctx, d, t, mean, rstd, gamma, drop=drop, dtotal=e)
        desc = None if drop is None else C.byref(L.binding.DropoutDesc(*drop))
        for res_is, x_is in (("d", "e"), ("e", "d"), ("d", None), ("e", None), (None, "d"), (None, "e")):
            a, b = device_matrix(2, rows, cols, dtype, 1, 0.1), device_matrix(4, rows, cols, dtype, 5, 0.1)
            place = {"d": a, "e": b, None: device_matrix(3, rows, cols, dtype)}
            dres, dx = place[res_is], place[x_is]
            dgamma, dbeta = gamma.clone(), gamma.clone()
            rc = lib.leann_layernorm_backward(ctx, a.data_ptr(), a.stride(0), t.data_ptr(), t.stride(0), rows, cols, code, gamma.data_ptr(), mean.data_ptr(),
                                              rstd.data_ptr(), b.data_ptr(), b.stride(0), desc, dres.data_ptr(), dres.stride(0), dx.data_ptr(), dx.stride(0),
                                              dgamma.data_ptr(), dbeta.data_ptr())
            assert rc == 0
            got = (dres, dres if drop is None else dx, dgamma, dbeta)
            assert all(bool((u == v).all()) for u, v in zip(got, want)), (res_is, x_is)
