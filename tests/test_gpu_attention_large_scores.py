"""Scores so large that their product with log2 e is rounded by more than fp16's range of weights: biases that hide whole rows, and queries and keys of that size."""
import pytest

from attention64 import assert_near
from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_far_biases import assert_even

pytestmark = pytest.mark.gpu
SIZES = [(8, 2), (32, 2), (40, 2), (64, 2), (96, 1), (128, 2)]


@pytest.mark.parametrize("value", [-3.4e38, -1e20, -1e9, 1e9, 3e38])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,heads", SIZES)
def test_rows_of_one_large_bias(ctx, dim, heads, dtype, value):  # noqa: F811
    """Scores of up to 10 are lost against 1e9 (a step of 64): all that a query sees weighs the same, in one block, in parts, and beyond the last distance."""
    say("attention, rows of one large bias", dim, dtype, value)
    for more in (dict(q_rows=[5, 200]), dict(q_rows=[1, 3], k_rows=[3000, 400], first=[2999, 0]), dict(q_rows=[130], window=(40, 0))):
        with Case(ctx, heads=heads, dim=dim, dtype=dtype, buckets=16, distance=32, **more) as c:
            c.bias[:] = value
            assert_even(c)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,heads", SIZES)
@pytest.mark.parametrize("sign", [1, -1])
def test_large_queries_and_keys(ctx, sign, dim, heads, dtype):  # noqa: F811
    """Scores around 2^30, all of whose products and sums are whole numbers of fp32: one key of a row is above the others by far, or two are alike."""
    import torch
    say("attention, large queries and keys", sign, dim, dtype)
    with Case(ctx, [3, 150], heads=heads, dim=dim, dtype=dtype) as c:
        c.q[:], c.k[:] = 0, 0
        c.q[:, ::dim] = 2.0 ** 15
        g = torch.Generator("cuda:0").manual_seed(3)
        steps = torch.randint(128, 256, (153, heads), generator=g, device="cuda:0")  # numbers of eight bits
        c.k[:, ::dim] = (sign * steps * 128).to(c.k.dtype)
        out, lse = c.run()
        s = c.sequences()
        for rows, keys, see, _ in s.parts():
            for h in range(heads):
                cq, ck = s.columns(h)
                n = sign * steps[keys, h]
                best = (n == n.max()).double()
                want = (best / best.sum()) @ c.v[keys, ck].double()
                size = (best / best.sum()) @ c.v[keys, ck].double().abs()
                assert_near(out[rows, cq], want.expand(rows.stop - rows.start, -1), (c.step * (size * (1 + c.step) + want.abs()) + 2.0 ** -20 * size + 1e-6).expand(rows.stop - rows.start, -1), "out")
                top = float(n.max()) * 128 * 2.0 ** 15 * c.scale
                assert bool(((lse[h, rows].double() - top).abs() <= 2.0 ** -22 * abs(top)).all())
