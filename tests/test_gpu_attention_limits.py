"""Attention and its gradient at the ends of what their header allows: scales of either sign, positions up to 2^30, 1024 heads, rows 2^22 elements apart."""
import pytest

from attention64 import assert_near
from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_backward import NAMES

pytestmark = pytest.mark.gpu


def check_with(c, scale):
    """Forward and backward under `scale` against the definitions."""
    c.scale = scale
    out, lse = c.L.leann_attention(c.ctx, c.plan, c.q, c.k, c.v, scale=scale, bias=c.bias, keep=True)
    want, want_lse, far, far_lse = c.sequences().forward(c.step)
    assert_near(out, want, far, "out")
    assert_near(lse, want_lse, far_lse, "lse")
    got = c.L.leann_attention_backward(c.ctx, c.plan, c.dout, c.q, c.k, c.v, out, lse, scale=scale, bias=c.bias)
    for name, g, (w, f) in zip(NAMES, got, c.sequences().backward(c.dout, out, lse, c.step)):
        if g is not None:
            assert_near(g, w, f, name)


@pytest.mark.parametrize("scale", [0.7, -0.125, -0.03, 2.0 ** -20, -2.0 ** -20])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("plan", [dict(q_rows=[70, 200, 300]), dict(q_rows=[40, 130], dim=128), dict(q_rows=[90, 7], kv_heads=1, window=(30, 10), sinks=3),
                                  dict(q_rows=[2], k_rows=[1500])], ids=["heads of 64", "heads of 128", "window, shared heads", "keys in parts"])
def test_scales(ctx, plan, dtype, scale):  # noqa: F811
    say("attention, scales", plan, dtype, scale)
    for more in (dict(), dict(buckets=16, distance=40)):
        with Case(ctx, heads=2, dtype=dtype, **plan, **more) as c:
            check_with(c, scale)


@pytest.mark.parametrize("scale", [2.0 ** 20, -2.0 ** 20])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_the_largest_scale(ctx, dtype, scale):  # noqa: F811
    """Queries as small as the scale is large."""
    say("attention, the largest scale", dtype, scale)
    with Case(ctx, [70, 300], heads=2, dtype=dtype, buckets=16, distance=40) as c:
        c.q.mul_(2.0 ** -11)
        c.k.mul_(2.0 ** -11)
        check_with(c, scale)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rules", [dict(), dict(window=(-1, 0)), dict(window=(0, -1)), dict(window=(100, 7), sinks=5), dict(window=(1 << 30, 1 << 30)), dict(window=((1 << 30) - 120, 0))],
                         ids=["all", "no keys ahead", "no keys behind", "first keys only", "the widest window", "a window that ends at key 0 and on"])
def test_the_last_positions(ctx, rules, dtype):  # noqa: F811
    """Queries at positions up to 2^30 - 2, the keys where they always are."""
    say("attention, last positions", rules, dtype)
    rows = [200, 3, 130]
    for more in (dict(), dict(buckets=16, distance=40)):
        with Case(ctx, rows, heads=2, dtype=dtype, first=[(1 << 30) - 1 - n for n in rows], **rules, **more) as c:
            check_with(c, c.scale)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("kv_heads", [1024, 1])
def test_many_heads(ctx, kv_heads, dtype):  # noqa: F811
    say("attention, 1024 heads", kv_heads, dtype)
    for more in (dict(), dict(buckets=4, distance=5)):
        with Case(ctx, [3, 40, 66], heads=1024, kv_heads=kv_heads, dim=8, dtype=dtype, **more) as c:
            check_with(c, c.scale)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,dim", [([256], 64), ([100, 156], 64), ([256], 128)])
def test_rows_far_apart(ctx, rows, dim, dtype):  # noqa: F811
    """Slices of one matrix of 2^22 columns: the 256 rows of a block span 2 GiB."""
    import torch
    say("attention, rows far apart", rows, dim, dtype)
    with Case(ctx, rows, heads=2, dim=dim, dtype=dtype, buckets=16, distance=40) as c:
        wide = torch.zeros((256, 1 << 22), dtype=c.q.dtype, device="cuda:0")
        n = 2 * dim
        for i, name in enumerate(("q", "k", "v", "dout")):
            wide[:, i * n:(i + 1) * n] = getattr(c, name)
        near = c.run()
        want = c.L.leann_attention_backward(c.ctx, c.plan, c.dout, c.q, c.k, c.v, *near, bias=c.bias)
        q, k, v, dout, out, dq, dk, dv = (wide[:, i * n:(i + 1) * n] for i in range(8))
        lse = c.L.leann_attention(c.ctx, c.plan, q, k, v, bias=c.bias, keep=True, out=out)[1]
        assert torch.equal(out, near[0]) and torch.equal(lse, near[1])
        got = c.L.leann_attention_backward(c.ctx, c.plan, dout, q, k, v, out, lse, bias=c.bias, dq=dq, dk=dk, dv=dv)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert not wide[:, 8 * n:].any()
