"""How exact few queries over many keys are: their largest weight is 1, which is rounded to nothing, so that only the others' roundings and the result's remain."""
import pytest

from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bits", [("bfloat16", 7), ("float16", 10)])
@pytest.mark.parametrize("plan", [dict(q_rows=[2] * 40, k_rows=[380] * 40), dict(q_rows=[1] * 200, k_rows=[40, 150] * 100), dict(q_rows=[3] * 30, k_rows=[3000] * 30)],
                         ids=["380 keys", "many", "in parts"])
def test_error_of_the_roundings_that_remain(ctx, plan, dtype, bits):  # noqa: F811
    """A rounding to b bits behind the leading one is off by 2^-b of the number's power of two, times a number evenly spread over [-1/2, 1/2], whose square is 1/12 on average."""
    import torch
    say("attention, few queries", dtype, plan["q_rows"][:2])
    with Case(ctx, heads=12, dtype=dtype, buckets=32, distance=128, **plan) as c:
        out = c.run(keep=False)
        s, error, expected, exact_weight = c.sequences(), 0.0, 0.0, 0.0
        want = s.forward(c.step)[0]
        error = float((out.double() - want).square().sum())
        expected = float((want.to(out.dtype).double() - want).square().sum())
        for rows, keys, see, buckets in s.parts():
            for h in range(12):
                cq, ck = s.columns(h)
                scores = s.scores(rows, keys, see, buckets, h)
                p = torch.exp(scores - scores.amax(1, keepdim=True))
                power = torch.exp2(torch.floor(torch.log2(p)).clamp(min=-14 if bits == 10 else -126))
                off = torch.where(p == 1, 0.0, (power * 2.0 ** -bits).square() / 12) @ s.v[keys, ck].double().square()
                expected += float((off / p.sum(1, keepdim=True).square()).sum())
        # the squares of some 10^5 roundings, of which a row's few largest weights count most: their mean is met to 10 %, so 5 % of the error
        assert error ** 0.5 <= 1.05 * expected ** 0.5, (error / expected) ** 0.5
