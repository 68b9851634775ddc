"""Dropout, LayerNorm and its gradient on the device against the plain forms in 64 bits."""
import numpy as np
import pytest

import plain64
from gpu_util import say

pytestmark = pytest.mark.gpu
EPS32 = 2.0 ** -24
EPS = 1e-12
DTYPES = ["float32", "bfloat16", "float16"]
COLS = [1, 2, 7, 8, 9, 64, 65, 128, 129, 200, 256, 257, 384, 513, 768, 1021, 1025, 1537, 2047, 2049, 4100, 5001, 8192]


@pytest.fixture(scope="module")
def ctx():
    import torch
    import paper_2506_08276_amd as L
    c = L.leann_create(dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1), torch.zeros(640, device="cuda:0"))
    yield c
    L.leann_destroy(c)


def matrix(rng, rows, cols, dtype, pad=0, scale=1.0, shift=0.0):
    """A device matrix whose rows lie cols + pad apart, NaN between them, and its values in 64 bits."""
    import torch
    wide = torch.full((rows, cols + pad), float("nan"), dtype=getattr(torch, dtype), device="cuda:0")
    wide[:, :cols] = torch.from_numpy(rng.normal(size=(rows, cols)) * scale + shift).to(getattr(torch, dtype)).to("cuda:0")
    t = wide[:, :cols]
    return t, t.double().cpu().numpy()


def vector(rng, cols, at):
    import torch
    v = torch.from_numpy((at + 0.3 * rng.normal(size=cols)).astype(np.float32)).to("cuda:0")
    return v, v.double().cpu().numpy()


def close(got, want, dtype, error, what):
    """One rounding to dtype of a value that is off by at most `error`."""
    u, tiny = plain64.ROUND[dtype]
    got = got.double().cpu().numpy()
    bound = error * (1 + u) + u * np.abs(want) + tiny
    off = np.abs(got - want) - bound
    assert np.isfinite(got).all(), what
    assert (off <= 0).all(), (what, off.max(), np.unravel_index(off.argmax(), off.shape))


def norm_errors(t, gamma, rstd):
    """Bounds of the 32-bit statistics' errors and of the normalised row: sums of n terms added in a tree (a lane's share in order, at most 64 terms).
    mean: 80 roundings of at most max|t|; t - mean: that and its own; rstd: relative, 100 roundings in the sum of squares, the shift of the mean."""
    big = np.abs(t).max(1)
    mean = 80 * EPS32 * big
    rel = 120 * EPS32 + mean * rstd
    return mean, rel


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 7, 8, 64, 769, 3000])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.9, 1.0])
def test_dropout(ctx, dtype, cols, p):
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(cols)
    for rows, pad, with_res in [(1, 0, False), (37, 3, True), (300, 0, False), (300, 8, True)]:
        say("dropout", dtype, rows, cols, p, pad, with_res)
        x, x64 = matrix(rng, rows, cols, dtype, pad)
        res, r64 = matrix(rng, rows, cols, dtype, 1) if with_res else (None, 0.0)
        drop = (p, 0x9876543210FEDCBA, (7 << 32) + rows)
        want = plain64.dropout(x64, drop)
        out = L.leann_dropout(ctx, x, drop, residual=res)
        close(out, want + r64, dtype, 3 * EPS32 * np.abs(want) + EPS32 * np.abs(want + r64), (rows, pad))
        if not with_res:
            assert ((out.cpu().double().numpy() == 0) == (want == 0)).all()
            assert L.leann_dropout(ctx, x, drop, out=x) is x and bool((x == out).all())  # in place


def test_dropout_of_infinities_and_nan(ctx):
    import torch
    import paper_2506_08276_amd as L
    x = torch.full((64, 40), float("inf"), device="cuda:0")
    x[:, ::2] = float("nan")
    out = L.leann_dropout(ctx, x, (0.5, 1, 2)).cpu().numpy()
    gone = plain64.dropout_bits(64, 40, 1, 2) < 32768
    assert (out[gone] == 0).all() and not np.isfinite(out[~gone]).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_layernorm(ctx, dtype, cols):
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(cols + 1)
    for rows, pad, with_res, drop, keep in [(1, 0, False, None, True), (5, 3, True, (0.1, 11, 12), True), (131, 0, True, None, False),
                                            (1030 if cols < 2000 else 67, 8, False, (0.3, 1, 1 << 40), True)]:
        say("layernorm", dtype, rows, cols, pad, with_res, drop, keep)
        x, x64 = matrix(rng, rows, cols, dtype, pad, shift=0.5)
        res, r64 = matrix(rng, rows, cols, dtype, 0, scale=2.0) if with_res else (None, 0.0)
        (gamma, g64), (beta, b64) = vector(rng, cols, 1.0), vector(rng, cols, 0.0)
        t64 = plain64.dropout(x64, drop) + r64
        want, mean64, rstd64 = plain64.layernorm(t64, g64, b64, EPS)
        got = L.leann_layernorm(ctx, x, gamma, beta, EPS, residual=res, drop=drop, keep=keep)
        mean_error, rel = norm_errors(t64, g64, rstd64)
        if cols == 1:  # every row is its own mean: nothing is left but the mean's rounding, times 10^6
            want, rel = np.broadcast_to(b64, want.shape), np.zeros(rows)
        mean_error = mean_error + 4 * EPS32 * np.abs(t64).max(1)  # t itself
        error = np.abs(g64) * (mean_error * rstd64)[:, None] + np.abs(want - b64) * rel[:, None] + 4 * EPS32 * (np.abs(want) + np.abs(b64))
        out = got[0] if keep else got
        close(out, want, dtype, error, "out")
        if keep:
            _, total, mean, rstd = got
            if drop or with_res:
                close(total, t64, dtype, 4 * EPS32 * (np.abs(t64) + np.abs(r64)), "total")
            else:
                assert total is x
            close(mean, mean64, "float32", mean_error, "mean")
            if cols > 1:
                close(rstd, rstd64, "float32", rstd64 * rel, "rstd")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_layernorm_backward(ctx, dtype, cols):
    import torch
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(cols + 2)
    for rows, pad, drop, extra in [(0, 0, None, False), (1, 0, None, True), (5, 3, (0.1, 5, 6), False), (66, 0, (0.5, 5, 6), True),
                                   (4500 if cols < 2000 else 1300 if cols < 5000 else 531, 8, None, False)]:
        say("layernorm backward", dtype, rows, cols, pad, drop, extra)
        t, t64 = matrix(rng, rows, cols, dtype, pad)
        d, d64 = matrix(rng, rows, cols, dtype, pad, scale=0.1)
        e, e64 = matrix(rng, rows, cols, dtype, 0, scale=0.1) if extra else (None, 0.0)
        gamma, g64 = vector(rng, cols, 1.0)
        mean = torch.from_numpy(t64.mean(1).astype(np.float32)).to("cuda:0")
        rstd = torch.from_numpy((1 / np.sqrt(t64.var(1) + 1e-3)).astype(np.float32)).to("cuda:0")
        m64, s64 = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
        want, dgamma64, dbeta64 = plain64.layernorm_backward(d64, t64, m64, s64, g64)
        dres, dx, dgamma, dbeta = L.leann_layernorm_backward(ctx, d, t, mean, rstd, gamma, drop=drop, dtotal=e)
        if rows:
            # each sum: 80 roundings of its terms' mean size; each term: its factors' roundings and its own
            xhat = np.abs((t64 - m64[:, None]) * s64[:, None]) + EPS32 * (np.abs(t64) + np.abs(m64[:, None])) * s64[:, None]
            gy = np.abs(d64 * g64)
            error = 100 * EPS32 * s64[:, None] * (gy + gy.mean(1, keepdims=True) + xhat * (gy * xhat).mean(1, keepdims=True))
            error += 4 * EPS32 * (np.abs(want) + np.abs(e64))
            close(dres, want + e64, dtype, error, "dresidual")
            factor = 1 if drop is None else 1 / (1 - drop[0])
            if drop is None:
                assert dx is dres
            else:
                close(dx, plain64.dropout(want + e64, drop), dtype, (error + 3 * EPS32 * np.abs(want + e64)) * factor * 1.001, "dx")
        # sums over the rows: at most 64 in order per wavefront, then blocks and slices; their terms' roundings
        depth = 64 + rows / 64
        close(dgamma, dgamma64, "float32", depth * EPS32 * (np.abs(d64) * np.abs((np.abs(t64) + np.abs(m64[:, None])) * s64[:, None])).sum(0), "dgamma")
        close(dbeta, dbeta64, "float32", depth * EPS32 * np.abs(d64).sum(0), "dbeta")


def test_layernorm_gradient_against_differences(ctx):
    """The device's gradients of a whole block against central differences of the 64-bit forward."""
    import torch
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(3)
    rows, cols, drop = 4, 13, (0.3, 21, 22)
    x, x64 = matrix(rng, rows, cols, "float32")
    res, r64 = matrix(rng, rows, cols, "float32")
    d, d64 = matrix(rng, rows, cols, "float32")
    (gamma, g64), (beta, b64) = vector(rng, cols, 1.0), vector(rng, cols, 0.0)
    _, total, mean, rstd = L.leann_layernorm(ctx, x, gamma, beta, 1e-3, residual=res, drop=drop, keep=True)
    dres, dx, dgamma, dbeta = L.leann_layernorm_backward(ctx, d, total, mean, rstd, gamma, drop=drop)
    loss = lambda v: (plain64.layernorm(plain64.dropout(v[0], drop) + v[1], v[2], v[3], 1e-3)[0] * d64).sum()
    values = [x64, r64, g64, b64]
    for i, got in enumerate((dx, dres, dgamma, dbeta)):
        got = got.double().cpu().numpy()
        for j in np.ndindex(values[i].shape):
            up, down = [v.copy() for v in values], [v.copy() for v in values]
            up[i][j] += 1e-6
            down[i][j] -= 1e-6
            # differences: 1e-12 x third derivative and 1e-16 / 1e-6 x loss; the kernel: some 100 roundings of terms of order 10
            assert abs((loss(up) - loss(down)) / 2e-6 - got[j]) < 100 * EPS32 * 10 + 1e-8, (i, j)


def test_rows_do_not_touch_each_other(ctx):
    """A row of NaN, one of infinities, a constant one, one of zeros: the others' bits stay, constant rows give beta."""
    import torch
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(4)
    x, _ = matrix(rng, 37, 768, "bfloat16")
    gamma, beta = vector(rng, 768, 1.0)[0], vector(rng, 768, 0.0)[0]
    want = L.leann_layernorm(ctx, x, gamma, beta, EPS)
    bad = x.clone()
    bad[3], bad[9, 5], bad[20], bad[36] = float("nan"), float("inf"), 0.0, 0.5
    got = L.leann_layernorm(ctx, bad, gamma, beta, EPS)
    rest = [i for i in range(37) if i not in (3, 9, 20, 36)]
    assert bool((got[rest] == want[rest]).all())
    assert bool((got[20] == beta.bfloat16()).all()) and bool((got[36] == beta.bfloat16()).all())  # 0.5 * 768 / 768 is exact
    assert bool(got[3].isnan().all())


@pytest.mark.parametrize("cols", [1, 72, 128, 130, 250])
def test_many_narrow_rows(ctx, cols):
    """Several rows per wavefront, each wavefront several times: every row as in a call of a part of them; the sums against 64 bits."""
    import torch
    import paper_2506_08276_amd as L
    rng = np.random.default_rng(cols + 5)
    rows, part = 70003, 2047
    x, x64 = matrix(rng, rows, cols, "bfloat16", 5)
    d, d64 = matrix(rng, rows, cols, "bfloat16")
    (gamma, g64), (beta, _) = vector(rng, cols, 1.0), vector(rng, cols, 0.0)
    out, _, mean, rstd = L.leann_layernorm(ctx, x, gamma, beta, 1e-3, residual=d, keep=True)
    total = (x.float() + d.float()).bfloat16()
    dres, _, dgamma, dbeta = L.leann_layernorm_backward(ctx, d, total, mean, rstd, gamma)
    for at in range(0, rows, 20 * part):
        of = slice(at, at + part)
        want = L.leann_layernorm(ctx, x[of], gamma, beta, 1e-3, residual=d[of], keep=True)
        assert bool((out[of] == want[0]).all()) and bool((mean[of] == want[2]).all()) and bool((rstd[of] == want[3]).all()), at
        assert bool((dres[of] == L.leann_layernorm_backward(ctx, d[of], total[of], mean[of], rstd[of], gamma)[0]).all()), at
    t64, m64, s64 = (v.double().cpu().numpy() for v in (total, mean, rstd))
    _, dgamma64, dbeta64 = plain64.layernorm_backward(d64, t64, m64, s64, g64)
    depth = 64 + rows / 64
    close(dgamma, dgamma64, "float32", depth * EPS32 * (np.abs(d64) * np.abs((np.abs(t64) + np.abs(m64[:, None])) * s64[:, None])).sum(0), "dgamma")
    close(dbeta, dbeta64, "float32", depth * EPS32 * np.abs(d64).sum(0), "dbeta")


def test_same_bits_twice_and_large_offsets(ctx):
    """Rows whose elements lie beyond 2^32 elements; the bits repeat."""
    import torch
    import paper_2506_08276_amd as L
    rows, cols, ld = 70001, 64, 65000
    wide = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda:0")  # 9.1 GB
    x = wide[:, :cols]
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x.copy_(torch.randn((rows, cols), generator=g, device="cuda:0"))
    gamma, beta = torch.ones(cols, device="cuda:0"), torch.zeros(cols, device="cuda:0")
    packed = x.contiguous()
    drop = (0.2, 3, 4)
    out, total, mean, rstd = L.leann_layernorm(ctx, x, gamma, beta, EPS, drop=drop, keep=True)
    out2, total2, mean2, rstd2 = L.leann_layernorm(ctx, packed, gamma, beta, EPS, drop=drop, keep=True)
    assert bool((out == out2).all()) and bool((total == total2).all()) and bool((mean == mean2).all()) and bool((rstd == rstd2).all())
    wide[:, 64:128] = packed
    a = L.leann_layernorm_backward(ctx, wide[:, 64:128], total, mean, rstd, gamma, drop=drop)
    b = L.leann_layernorm_backward(ctx, packed, total, mean, rstd, gamma, drop=drop)
    assert all(bool((u == v).all()) for u, v in zip(a, b))
    assert bool((L.leann_dropout(ctx, x, drop, out=wide[:, 128:192]) == L.leann_dropout(ctx, packed, drop)).all())


def test_context_of_another_stream():
    import torch
    import paper_2506_08276_amd as L
    side = torch.cuda.Stream()
    g = torch.Generator(device="cuda:0").manual_seed(2)
    x = torch.randn((3000, 768), generator=g, device="cuda:0")
    gamma, beta = torch.ones(768, device="cuda:0"), torch.zeros(768, device="cuda:0")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = L.leann_create(dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1), torch.zeros(640, device="cuda:0"))
        y = x * 2  # on the side stream, before the call and after it
        out = L.leann_layernorm(c, y, gamma, beta, 1e-5)
        twice = out * 2
    side.synchronize()
    want = torch.nn.functional.layer_norm(x * 2, (768,), gamma, beta, 1e-5)
    assert float((twice / 2 - want).abs().max()) < 1e-5
    L.leann_destroy(c)


def test_refusals(ctx):
    import torch
    import paper_2506_08276_amd as L
    lib = L.load_library()
    x = torch.zeros((4, 8), device="cuda:0")
    v = torch.ones(8, device="cuda:0")
    p, vp = x.data_ptr(), v.data_ptr()
    from paper_2506_08276_amd.binding import DropoutDesc
    import ctypes as C
    drop = lambda rate: C.byref(DropoutDesc(rate, 1, 2))
    EINVAL, ESHAPE = -1, -4

    def refused(status, rc):
        assert rc == status and lib.leann_last_error(None)

    D = lib.leann_dropout
    refused(EINVAL, D(None, p, 8, None, 0, 4, 8, 0, drop(0.1), p, 8))
    refused(EINVAL, D(ctx, p, 8, None, 0, 4, 8, 0, None, p, 8))
    refused(EINVAL, D(ctx, None, 8, None, 0, 4, 8, 0, drop(0.1), p, 8))
    refused(EINVAL, D(ctx, p, 8, None, 0, 4, 8, 0, drop(0.1), None, 8))
    refused(EINVAL, D(ctx, p, 8, None, 0, -1, 8, 0, drop(0.1), p, 8))
    refused(EINVAL, D(ctx, p, 8, None, 0, 4, 0, 0, drop(0.1), p, 8))
    refused(EINVAL, D(ctx, p, 8, None, 0, 4, 8, 3, drop(0.1), p, 8))
    for rate in (-0.1, 1.1, float("nan")):
        refused(EINVAL, D(ctx, p, 8, None, 0, 4, 8, 0, drop(rate), p, 8))
    refused(ESHAPE, D(ctx, p, 7, None, 0, 4, 8, 0, drop(0.1), p, 8))
    refused(ESHAPE, D(ctx, p, 8, p, 7, 4, 8, 0, drop(0.1), p, 8))
    refused(ESHAPE, D(ctx, p, 8, None, 0, 1 << 31, 8, 0, drop(0.1), p, 8))
    assert D(ctx, None, 8, None, 0, 0, 8, 0, drop(0.1), None, 8) == 0
    N = lib.leann_layernorm
    ok = [ctx, p, 8, None, 0, 4, 8, 0, None, vp, vp, 1e-5, p, 8, None, 0, None, None]
    for i, bad, status in [(0, None, EINVAL), (1, None, EINVAL), (2, 7, ESHAPE), (5, -1, EINVAL), (6, 0, EINVAL), (7, 9, EINVAL),
                           (8, drop(2.0), EINVAL), (9, None, EINVAL), (10, None, EINVAL), (11, 0.0, EINVAL), (11, float("nan"), EINVAL),
                           (12, None, EINVAL), (13, 7, ESHAPE), (16, vp, EINVAL), (17, vp, EINVAL)]:
        refused(status, N(*[bad if j == i else a for j, a in enumerate(ok)]))
    refused(ESHAPE, N(ctx, p, 8193, None, 0, 1, 8193, 0, None, vp, vp, 1e-5, p, 8193, None, 0, None, None))
    refused(ESHAPE, N(ctx, p, 8, p, 7, 4, 8, 0, None, vp, vp, 1e-5, p, 8, None, 0, None, None))
    refused(ESHAPE, N(ctx, p, 8, None, 0, 4, 8, 0, None, vp, vp, 1e-5, p, 8, p, 7, None, None))
    B = lib.leann_layernorm_backward
    ok = [ctx, p, 8, p, 8, 4, 8, 0, vp, vp, vp, None, 0, None, p, 8, None, 0, vp, vp]
    for i, bad, status in [(0, None, EINVAL), (1, None, EINVAL), (2, 7, ESHAPE), (3, None, EINVAL), (4, 7, ESHAPE), (5, -1, EINVAL),
                           (6, 0, EINVAL), (7, -1, EINVAL), (8, None, EINVAL), (9, None, EINVAL), (10, None, EINVAL), (13, drop(0.5), EINVAL),
                           (14, None, EINVAL), (15, 7, ESHAPE), (18, None, EINVAL), (19, None, EINVAL)]:
        refused(status, B(*[bad if j == i else a for j, a in enumerate(ok)]))
    refused(ESHAPE, B(ctx, p, 8, p, 8, 4, 8, 0, vp, vp, vp, p, 7, None, p, 8, None, 0, vp, vp))
    refused(ESHAPE, B(ctx, p, 8193, p, 8193, 1, 8193, 0, vp, vp, vp, None, 0, None, p, 8193, None, 0, vp, vp))
    assert bool((x == 0).all()) and bool((v == 1).all())
