"""Buckets of the bias that no pair of a sequence is in, but a longer sequence's are: infinities and NaN of theirs do not reach it."""
import pytest

from gpu_util import say
from test_gpu_attention import Case, ctx  # noqa: F401
from test_gpu_attention_backward import backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_short_beside_long(ctx, value, dim, dtype):  # noqa: F811
    """40, 100 and 130 tokens fill no block of 32: where a block goes on behind them, relative positions are as far as 63, 127 and 159."""
    import torch
    say("attention, unreached buckets", value, dim, dtype)
    for short, far in ((40, 46), (100, 116), (130, 150)):
        with Case(ctx, [short, 400, short], heads=2, dim=dim, dtype=dtype, buckets=256, distance=200) as c:
            away = torch.arange(-200, 201)
            reached = torch.as_tensor(c.table, dtype=torch.int64)
            hurt = reached[away.abs() >= far].unique()
            assert not set(hurt.tolist()) & set(reached[away.abs() < short].tolist())
            out, lse = c.run()
            clean = backward(c, out, lse)
            c.bias[hurt.to(c.bias.device)] = value
            again, lse_again = c.run()
            got = backward(c, again, lse_again)
            for rows in (slice(0, short), slice(short + 400, 2 * short + 400)):
                assert torch.equal(again[rows], out[rows]) and torch.equal(lse_again[:, rows], lse[:, rows])
                for a, b in zip(got[:3], clean[:3]):
                    assert torch.equal(a[rows], b[rows])
            assert not torch.isfinite(again[short:short + 400]).all()
