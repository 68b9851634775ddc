"""The gradient of sequences of a single key: its weight is 1 whatever its score, so queries, keys and biases have none, to the bit."""
import pytest

from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_backward import check

pytestmark = pytest.mark.gpu
PLANS = {
    "single tokens": dict(q_rows=[1, 1, 1]),
    "many single tokens": dict(q_rows=[1] * 90),
    "queries over one key": dict(q_rows=[5, 1, 200, 0, 300], k_rows=[1, 1, 1, 1, 1]),
    "one key far behind": dict(q_rows=[70], k_rows=[1], first=[900]),
    "one key ahead of the first query only": dict(q_rows=[40], k_rows=[1], window=(3, 0)),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", [dict(dim=32), dict(dim=64), dict(dim=96, heads=4, kv_heads=1), dict(dim=128)], ids=lambda s: f"{s['dim']}")
@pytest.mark.parametrize("plan", PLANS)
def test_one_key(ctx, plan, shape, dtype):  # noqa: F811
    say("attention backward, one key", plan, shape, dtype)
    for more in (dict(), dict(buckets=16, distance=32)):
        with Case(ctx, dtype=dtype, **PLANS[plan], **shape, **more) as c:
            dq, dk, dv, dbias = check(c)
            assert not dq.any() and not dk.any() and (dbias is None or not dbias.any())
            assert dv.any()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_beside_others(ctx, dim, dtype):  # noqa: F811
    """A block that has one key of its own, as the last of 65, 129 and 257 have, is not a sequence of one key."""
    say("attention backward, one key beside others", dim, dtype)
    for rows in ([65, 1, 129, 257], [1, 65], [2, 1, 2]):
        with Case(ctx, rows, dim=dim, dtype=dtype, buckets=16, distance=32) as c:
            dq, dk, _, _ = check(c)
            at = 0
            for n in rows:
                assert (n == 1) != bool(dk[at + n - 1].any()) and (n == 1) != bool(dq[at + n - 1].any())
                at += n


@pytest.mark.parametrize("what", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_infinities_stay(ctx, value, what):  # noqa: F811
    import torch
    say("attention backward, one key, infinities", what, value)
    for shape in (dict(dim=64), dict(dim=128), dict(dim=64, dtype="float16")):
        with Case(ctx, [1, 1], heads=2, **shape) as c:
            getattr(c, what)[1] = value
            out, lse = c.run()
            dq, dk, _, _ = c.L.leann_attention_backward(c.ctx, c.plan, c.dout, c.q, c.k, c.v, out, lse)
            assert not dq[0].any() and not dk[0].any()
            if not (what in "qk" and value == float("inf")):  # a score of -inf is a weight of 0
                assert not torch.isfinite(dq[1]).any() and not torch.isfinite(dk[1]).any()
