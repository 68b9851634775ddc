"""GELU, its gradient and activations in 8 bits on the GPU against their definitions in 64 bits."""
import math

import pytest

from attention64 import assert_near
from gpu_util import say

pytestmark = pytest.mark.gpu
CTX = dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1)
SIZES = [(1, 1), (1, 128), (3, 129), (12, 768), (7, 127), (5, 8), (33, 1021), (2, 8200), (1500, 384), (70000, 9)]
TYPES = ["float32", "bfloat16", "float16"]


@pytest.fixture(scope="module")
def ctx():
    import torch
    import paper_2506_08276_amd as L
    c = L.leann_create(CTX, torch.zeros(640, device="cuda:0"))
    yield c
    L.leann_destroy(c)


def matrix(rows, cols, dtype, seed=0, pad=0, scale=1.5):
    import torch
    g = torch.Generator("cuda:0").manual_seed(seed)
    t = scale * torch.randn((rows, cols + pad), generator=g, device="cuda:0")
    t[:, ::97] *= 8
    return t.to(getattr(torch, dtype))[:, :cols]


def half_step(t):
    import torch
    return torch.finfo(t.dtype).eps / 2


def blocks(x):
    """Blocks of 128 columns in 64 bits, zeros behind a row's end."""
    import torch
    rows, cols = x.shape
    n = (cols + 127) // 128
    w = torch.zeros((rows, n * 128), dtype=torch.float64, device=x.device)
    w[:, :cols] = x
    return w.view(rows, n, 128)


def stands_for(kept):
    codes, scales = kept
    rows, cols = codes.shape
    return (blocks(codes) * scales.double()[:, :, None]).view(rows, -1)[:, :cols]


def check_codes(x, kept):
    """The codes are the nearest whole numbers of 127 x / max |x|, the scales max |x| / 127."""
    import torch
    codes, scales = kept
    w = blocks(x)
    a = w.abs().amax(2)
    assert_near(scales, a / 127, 2.0 ** -24 * a / 127 + 2.0 ** -150, "scales")
    q = torch.where(a[:, :, None] > 0, 127 * w / a[:, :, None], 0.0).view(len(x), -1)[:, :x.shape[1]]
    want = q.round()  # ties to even
    if x.dtype == torch.float32:  # the product and the quotient in 32 bits: two roundings of 2^-24 of up to 127
        near = (q - q.floor() - 0.5).abs() < 127 * 2.0 ** -23
        assert bool(((codes.double() - want).abs() <= near).all())
    else:
        assert torch.equal(codes.double(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_checkpoint(ctx, rows, cols, dtype):
    import torch
    import paper_2506_08276_amd as L
    say("checkpoint", rows, cols, dtype)
    for pad in (0, 3):
        x = matrix(rows, cols, dtype, seed=rows + cols, pad=pad)
        kept = L.leann_checkpoint(ctx, x)
        check_codes(x, kept)
        for to in (torch.float32, torch.bfloat16, torch.float16):
            got = L.leann_checkpoint_restore(ctx, kept, to)
            assert got.dtype == to
            want = stands_for(kept)
            assert_near(got, want, (2.0 ** -24 + torch.finfo(to).eps / 2) * want.abs() + (2.0 ** -25 if to == torch.float16 else 2.0 ** -140), "restored")


def test_ties_and_ends(ctx):
    """Rows whose largest is 127 steps of a power of two, so that many quotients are ties; zeros; the smallest and largest numbers; one element."""
    import torch
    import paper_2506_08276_amd as L
    say("checkpoint, ties")
    steps = torch.arange(-127, 128, device="cuda:0") / 2
    for dtype, scale in ((torch.bfloat16, 2.0 ** -3), (torch.bfloat16, 2.0 ** 100), (torch.bfloat16, 2.0 ** -120), (torch.float16, 2.0 ** -10), (torch.float16, 2.0 ** 8),
                         (torch.float32, 2.0 ** 118), (torch.float32, 2.0 ** -130), (torch.float32, 1.0)):
        x = torch.zeros((6, 256), device="cuda:0")
        x[0, :255], x[1, 1:] = steps, steps
        x[0, 255], x[0, 0] = 127, -127  # both blocks have their 127
        x[1, 0] = x[1, 255] = 127
        x[2, 3] = 1
        x[3, 200] = -5
        x[4] = 127
        x = (x * scale).to(dtype)
        assert bool(torch.isfinite(x).all())
        kept = L.leann_checkpoint(ctx, x)
        check_codes(x, kept)
        assert not kept[0][5].any() and not kept[1][5].any()
        if dtype != torch.float32 or scale != 2.0 ** -130:  # a scale that is no normal number is off by more
            assert torch.equal(L.leann_checkpoint_restore(ctx, kept, dtype)[4], x[4])


def test_infinities_stay_in_their_block(ctx):
    import torch
    import paper_2506_08276_amd as L
    say("checkpoint, infinities")
    for dtype in TYPES:
        x = matrix(4, 300, dtype)
        clean = L.leann_checkpoint_restore(ctx, L.leann_checkpoint(ctx, x), x.dtype)
        x[0, 5], x[1, 200], x[2, 299] = float("nan"), float("inf"), -float("inf")
        got = L.leann_checkpoint_restore(ctx, L.leann_checkpoint(ctx, x), x.dtype)
        hit = torch.zeros_like(x, dtype=torch.bool)
        hit[0, :128] = hit[1, 128:256] = hit[2, 256:] = True
        assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean[~hit])


def exact(x, kind):
    """(y, dy / dx, bounds of their errors in fp32) in 64 bits.  A reciprocal or an exponential below 2^-126 may come as 0: off by that much before it is multiplied by x."""
    import torch
    x = x.double()
    if kind == "gelu":
        phi = 0.5 * torch.erfc(-x / math.sqrt(2))
        e = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        # Phi: the formula's 7.5e-8, and eight roundings of 2^-23 of a number below 1; the exponential's argument is off by 2^-23 of itself, twice
        off = 7.5e-8 + 8 * 2.0 ** -23
        return x * phi, phi + x * e, off * x.abs(), off + x.abs() * e * (8 + x * x) * 2.0 ** -23
    b = math.sqrt(2 / math.pi)
    u, du = b * (x + 0.044715 * x ** 3), b * (1 + 3 * 0.044715 * x ** 2)
    g = torch.sigmoid(2 * u)
    off = (8 + 8 * u.abs()) * 2.0 ** -23 * g + 2.0 ** -126  # the exponential's argument is off by four roundings
    return x * g, g + 2 * x * g * (1 - g) * du, off * x.abs(), off + x.abs() * 2 * du * (off + 12 * 2.0 ** -23 * g * (1 - g) + 2.0 ** -23 * g) + 2.0 ** -23


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_activation(ctx, rows, cols, kind, dtype):
    import torch
    import paper_2506_08276_amd as L
    say("activation", rows, cols, kind, dtype)
    for pad in (0, 5):
        x = matrix(rows, cols, dtype, seed=rows, pad=pad)
        dout = matrix(rows, cols, dtype, seed=1, scale=0.1)
        h, tiny = half_step(x), 2.0 ** -25 if dtype == "float16" else 2.0 ** -126
        y, kept = L.leann_activation(ctx, x, kind, keep=True)
        want, _, far, _ = exact(x, kind)
        assert_near(y, want, far + h * want.abs() + tiny, "out")
        assert torch.equal(y, L.leann_activation(ctx, x, kind))
        assert all(torch.equal(a, b) for a, b in zip(kept, L.leann_checkpoint(ctx, x)))
        for given, at in ((kept, stands_for(kept)), (x, x)):
            want, slope, far, far_slope = exact(at, kind)
            if given is kept:  # the restored x is rounded to fp32; the slope's own slope is below 1.2
                far, far_slope = far + 2.0 ** -23 * at.abs(), far_slope + 2.0 ** -23 * at.abs()
            dx, again = L.leann_activation_backward(ctx, dout, given, kind, again=True)
            d = dout.double()
            assert_near(again, want, far + h * want.abs() + tiny, "again")
            assert_near(dx, d * slope, d.abs() * far_slope + (h + 2.0 ** -23) * (d * slope).abs() + tiny, "dx")
            assert torch.equal(dx, L.leann_activation_backward(ctx, dout, given, kind))
        inplace = dout.clone()
        L.leann_activation_backward(ctx, inplace, kept, kind, dx=inplace)
        assert torch.equal(inplace, L.leann_activation_backward(ctx, dout, kept, kind))
        z = x.clone()
        L.leann_activation(ctx, z, kind, out=z)
        assert torch.equal(z, y)


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh"])
def test_far_values(ctx, kind):
    """Where the function is 0 or x itself; NaN."""
    import torch
    import paper_2506_08276_amd as L
    say("activation, far values", kind)
    x = torch.tensor([[-3e38, -1e19, -1e4, -50, -0.0, 0.0, 50, 1e4, 1e19, 3e38, float("inf"), float("nan")]], device="cuda:0")
    y = L.leann_activation(ctx, x, kind)
    assert torch.equal(y[0, :6].abs(), torch.zeros(6, device="cuda:0")) and torch.equal(y[0, 6:11], x[0, 6:11]) and bool(y[0, 11].isnan())
    dx = L.leann_activation_backward(ctx, torch.ones_like(x), x, kind)
    assert bool(((dx[0, 4:6] - 0.5).abs() <= 7.5e-8 + 2.0 ** -24).all())  # the formula's own error at 0, half of 1.5e-7, and its last rounding
    assert not dx[0, :4].any() and bool((dx[0, 6:10] == 1).all()) and bool(dx[0, 11].isnan())


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh"])
def test_against_differences(ctx, kind):
    import torch
    import paper_2506_08276_amd as L
    say("activation against differences", kind)
    x = torch.linspace(-6, 6, 4001, device="cuda:0")[None, :]
    h = 2.0 ** -6
    up, down = x + h, x - h
    rise = (L.leann_activation(ctx, up, kind).double() - L.leann_activation(ctx, down, kind).double()) / (up.double() - down.double())
    dx = L.leann_activation_backward(ctx, torch.ones_like(x), x, kind)
    # the third derivative is below 1.6; outputs are off by 1.2e-6 of x (the bound above)
    assert_near(dx, rise, 1.6 / 6 * h * h + 2 * 1.2e-6 * (x.abs().double() + h) / (2 * h) + 2e-6 * (1 + x.abs().double()), "dx")


def test_rows_around_stay(ctx):
    import torch
    import paper_2506_08276_amd as L
    say("activation into a slice")
    x = matrix(9, 130, "bfloat16")
    whole = torch.full((12, 150), 7.0, dtype=x.dtype, device="cuda:0")
    L.leann_activation(ctx, x, out=whole[1:10, 3:133])
    assert torch.equal(whole[1:10, 3:133], L.leann_activation(ctx, x))
    whole[1:10, 3:133] = 7
    assert bool((whole == 7).all())
    kept = L.leann_checkpoint(ctx, x)
    L.leann_checkpoint_restore(ctx, kept, out=whole[1:10, 3:133])
    assert torch.equal(whole[1:10, 3:133], L.leann_checkpoint_restore(ctx, kept, x.dtype))
    whole[1:10, 3:133] = 7
    assert bool((whole == 7).all())


def test_offsets_beyond_32_bits(ctx):
    import torch
    import paper_2506_08276_amd as L
    say("activation over 2.2e9 elements")
    x = torch.zeros((540_000, 4096), dtype=torch.bfloat16, device="cuda:0")
    x[-1] = matrix(1, 4096, "bfloat16")[0]
    y, kept = L.leann_activation(ctx, x, keep=True)
    one, kept_one = L.leann_activation(ctx, x[-1:], keep=True)
    assert torch.equal(y[-1:], one) and not y[:-1].any() and torch.equal(kept[0][-1:], kept_one[0]) and torch.equal(kept[1][-1:], kept_one[1])
    dx = L.leann_activation_backward(ctx, y, kept)
    assert torch.equal(dx[-1:], L.leann_activation_backward(ctx, one, kept_one))


def test_zero_rows_and_refusals(ctx):
    import torch
    import paper_2506_08276_amd as L
    say("activation refusals")
    empty = torch.empty((0, 64), device="cuda:0")
    y, kept = L.leann_activation(ctx, empty, keep=True)
    assert y.shape == (0, 64) and L.leann_activation_backward(ctx, y, kept).shape == (0, 64) and L.leann_checkpoint_restore(ctx, kept, torch.float32).shape == (0, 64)
    x = matrix(4, 64, "float32")
    y, kept = L.leann_activation(ctx, x, keep=True)
    for call in (lambda: L.leann_activation(ctx, x, "relu"), lambda: L.leann_activation(ctx, x.double()), lambda: L.leann_activation(ctx, x.t()),
                 lambda: L.leann_activation(ctx, x, out=y.half()), lambda: L.leann_activation_backward(ctx, y[:3], kept),
                 lambda: L.leann_activation_backward(ctx, y, x.half()), lambda: L.leann_checkpoint_restore(ctx, kept),
                 lambda: L.leann_checkpoint_restore(ctx, (kept[0].float(), kept[1]), torch.float32),
                 lambda: L.leann_checkpoint_restore(ctx, (kept[0], kept[1][:3]), torch.float32), lambda: L.leann_checkpoint(ctx, x[0])):
        with pytest.raises(AssertionError):
            call()
