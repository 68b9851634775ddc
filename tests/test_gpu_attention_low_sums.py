"""The gradient of attention where all of a query's scores lie far below zero: keys behind a sequence's last one are zeros, whose score of 0 is then far above its log-sum."""
import math

import pytest

from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_backward import check

pytestmark = pytest.mark.gpu
# a short sequence's one kernel takes none of these: fp16, wide or shared heads, windows, long sequences
PLANS = {
    "heads of 32": dict(dim=32),
    "heads of 64": dict(),
    "heads of 40": dict(dim=40),
    "heads of 128": dict(dim=128),
    "shared key heads": dict(kv_heads=1),
    "a window that sees all": dict(window=(400, 400)),
    "a window": dict(window=(70, 70), sinks=2),
    "no keys ahead": dict(window=(-1, 0)),
}


def shift(c, low):
    """Queries around 1 and keys around a negative number, so that log-sums come to about `low`."""
    keys = max(c.q_rows)
    c.q.copy_(1 + c.q.float() / 8)
    c.k.copy_(c.k.float() / 8 + (low - math.log(keys)) / (c.args["head_dim"] * c.scale))


@pytest.mark.parametrize("low", [-10.0, -25.0, -60.0, -100.0])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("plan", PLANS)
def test_keys_behind_the_last_one(ctx, plan, dtype, low):  # noqa: F811
    say("attention backward, low log-sums", plan, dtype, low)
    for rows in ([3], [12, 48], [100, 300]):
        with Case(ctx, rows, heads=2, dtype=dtype, **PLANS[plan]) as c:
            shift(c, low)
            lse = c.run()[1]
            assert bool(((lse - low).abs() < 0.2 * abs(low) + 8).all())
            c.check()
            check(c)
