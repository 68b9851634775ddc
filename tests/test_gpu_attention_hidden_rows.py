"""The gradient of rows of large log-sums, as biases of -1e9 and fp32's lowest value make them that hide a row altogether: exp(s - lse) is all rounding there, and they have none."""
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


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_up_to_the_border(ctx, dim, dtype, sign):  # noqa: F811
    """Scores of queries and keys alone: below 2^21 weights are off by less than a half and within fp16's range, from there on there are none."""
    import torch
    say("attention backward, large log-sums", dim, dtype, sign)
    g = torch.Generator("cuda:0").manual_seed(1)
    for log in [14, 17] + [20 + i / 8 for i in range(25)]:
        with Case(ctx, [3, 90, 300], heads=2, dim=dim, dtype=dtype) as c:
            c.q[:], c.k[:] = 0, 0
            # the sequence's best key has steps of 128 (or 256, the other way round), its score is 2^log in magnitude, up to the rounding of q
            c.q[:, ::dim] = 2.0 ** (log - 14) / c.scale / (1 if sign < 0 else 2)
            steps = torch.randint(129, 255, (393, 2), generator=g, device="cuda:0")
            for at in (0, 3, 93):
                steps[at] = 128 if sign < 0 else 256
            c.k[:, ::dim] = (sign * steps * 128).to(c.k.dtype)
            out, lse = c.run()
            top = lse.abs().max()
            assert float(lse.abs().min()) == float(top) and abs(float(top.log2()) - log) < 2.0 ** -7
            if float(top) < 2.0 ** 21:
                got = backward(c, out, lse)
                want = c.sequences().backward(c.dout, out, lse, c.step)
                for at in (0, 3, 93):  # the best key's weights
                    size = want[2][0][at].abs()
                    assert bool(((got[2][at].double() - want[2][0][at]).abs() <= (0.5 + 2 * c.step) * size + 1e-6).all())
                assert all(bool(torch.isfinite(x).all()) for x in got[:3])
            else:
                assert not any(x.any() for x in backward(c, out, lse)[:3])
