"""Biases that hide keys farther away than the buckets' last distance, where a tile of keys has one bias for all."""
import pytest

from attention64 import assert_near
from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_backward import backward, check

pytestmark = pytest.mark.gpu
NEVER = -float("inf")
BUCKETS = dict(heads=2, buckets=16, distance=32)
PLANS = {
    "blocks of 128 queries": dict(q_rows=[600, 70]),
    "one tile beyond": dict(q_rows=[400]),
    "no keys ahead": dict(q_rows=[600, 400], window=(-1, 0)),
    "keys in parts": dict(q_rows=[1, 3], k_rows=[3000, 400], first=[2999, 397]),
    "keys in parts, 128 queries": dict(q_rows=[130], k_rows=[3000], first=[2870]),
    "all keys far behind": dict(q_rows=[5, 200], k_rows=[400, 300], first=[3000, 3000]),
    "all keys far ahead": dict(q_rows=[4], k_rows=[3000]),
}


def hide_ends(c, value=NEVER):
    """The buckets of the table's two ends, which hold all that is farther away."""
    c.bias[int(c.table[0])] = c.bias[int(c.table[-1])] = value


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("plan", PLANS)
def test_what_is_far_is_hidden(ctx, plan, dtype):  # noqa: F811
    """Spreads that make hidden scores of 12 and more, whose exponentials fp16 cannot hold, and of 95, beyond bf16's."""
    say("attention, far keys hidden", plan, dtype)
    for spread in (1.3, 3.0, 7.0):
        for value in (NEVER, -3e38):
            with Case(ctx, dtype=dtype, spread=spread, **BUCKETS, **PLANS[plan]) as c:
                hide_ends(c, value)
                if value == NEVER:
                    c.check()
                    if spread < 7.0: check(c)
                else:  # the same bits as with -inf, but for rows that see nothing else
                    out, lse = c.run()
                    hide_ends(c)
                    want, want_lse = c.run()
                    some = want_lse > NEVER
                    assert c.torch.equal(lse[some], want_lse[some])
                    rows = some.t().repeat_interleave(64, 1)
                    assert c.torch.equal(out[rows], want[rows])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("plan", PLANS)
def test_all_hidden(ctx, plan, dtype):  # noqa: F811
    """All biases -inf: nothing is seen.  All of them fp32's lowest: a row is even, on both sides of the table's ends."""
    import torch
    say("attention, all biases hide", plan, dtype)
    with Case(ctx, dtype=dtype, **BUCKETS, **PLANS[plan]) as c:
        c.bias[:] = NEVER
        out, lse = c.run()
        assert not out.any() and bool((lse == NEVER).all())
        assert not any(g.any() for g in backward(c, out, lse))
        c.bias[:] = torch.finfo(torch.float32).min
        assert_even(c)


def assert_even(c):
    """Every row is the mean of the values that it sees, up to the roundings of weights and result and those of a sum in fp32."""
    out, _ = c.run()
    for rows, keys, see, _ in c.sequences().parts():
        n, see = see.sum(1, keepdim=True), see.double()
        for h in range(c.args["heads"]):
            cq, ck = c.sequences().columns(h)
            v = c.v[keys, ck].double()
            mean, size = see @ v / n, see @ v.abs() / n
            assert_near(out[rows, cq], mean, c.step * (size * (1 + c.step) + mean.abs()) + see.shape[1] * 2.0 ** -24 * size + 1e-6, "out")
