"""The gradient of rows that large finite biases hide altogether, as 1e9 and fp32's lowest value: their log-sum cannot hold the number of keys, and they have none."""
import pytest

from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_backward import backward

pytestmark = pytest.mark.gpu
SIZES = [(8, 2), (32, 2), (40, 2), (64, 2), (128, 2)]


@pytest.mark.parametrize("value", [-3.4e38, -1e20, -1e9, -1e7, 1e9, 3e38])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,heads", SIZES)
def test_all_rows(ctx, dim, heads, dtype, value):  # noqa: F811
    say("attention backward, hidden rows", dim, dtype, value)
    for more in (dict(q_rows=[1, 5, 200, 300]), dict(q_rows=[3], k_rows=[1000], first=[997]), dict(q_rows=[130], window=(40, 0)), dict(q_rows=[100], kv_heads=1)):
        with Case(ctx, heads=heads, dim=dim, dtype=dtype, buckets=16, distance=32, **more) as c:
            c.bias[:] = value
            assert not any(g.any() for g in backward(c, *c.run()))


@pytest.mark.parametrize("value", [-3.4e38, -1e9])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,heads", SIZES)
def test_some_rows(ctx, dim, heads, dtype, value):  # noqa: F811
    """Queries of one sequence stand where they see nothing but far keys; the others' gradients are those of a bias of -inf, to the bit."""
    import torch
    say("attention backward, some rows hidden", dim, dtype, value)
    with Case(ctx, [90, 40, 300], heads=heads, dim=dim, dtype=dtype, buckets=16, distance=32, first=[0, 500, 0]) as c:
        got = []
        for low in (value, -float("inf")):
            c.bias[int(c.table[0])] = c.bias[int(c.table[-1])] = low
            got.append(backward(c, *c.run()))
        for a, b in zip(*got):
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
        assert not any(t[90:130].any() for t in got[0][:3]) and all(t[:90].any() for t in got[0][:3])
