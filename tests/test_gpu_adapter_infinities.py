"""Infinities in an adapter, in the rows that go through it, and in what reaches its gradients: the definition's infinities and nothing else."""
import numpy as np
import pytest

import plain64
import test_gpu_adapter as base
from gpu_util import say
from test_gpu_adapter import ctx  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
# By rows and shape every kernel of the product in both directions, and both of the low-rank activations.
CASES = {
    "odd ranks": (base.BATCHES["odd ranks"], 264, 136),
    "wide, many rows": (base.BATCHES["many rows"], 384, 768),
    "many rows": (base.BATCHES["many rows"], 768, 384),
    "large": (base.LARGE["many runs"], 776, 768),
    "more rows": (([9000, 7, 6000, 3000, 500], [0, 1, -1, 2, 0], [16, 24, 9]), 256, 264),
    "narrow": (([9000, 7, 6000, 3000, 500], [0, 1, -1, 2, 0], [60, 33, 128]), 40, 24),
}
params = pytest.mark.parametrize("dtype,case,value", [(d, c, v) for d in ("bfloat16", "float16") for c in CASES for v in ("inf", "-inf")])


class Positive(base.Problem):
    """Weights, adapters and scales above zero, so that sums of infinities keep their sign; rows of either sign."""

    def __init__(self, ctx, case, dtype):
        import torch
        batch, n_in, n_out = CASES[case]
        base.BATCHES["infinities"] = batch
        super().__init__(ctx, "infinities", n_in, n_out, dtype)
        del base.BATCHES["infinities"]
        self.close()
        type_ = getattr(torch, dtype)
        rng = np.random.default_rng(11)

        def positive(t):
            t.copy_(torch.from_numpy(rng.uniform(0.01, 0.1, size=tuple(t.shape))).to(type_))
            return t.double().cpu().numpy()

        self.w64, self.down64, self.up64 = positive(self.w), positive(self.down), positive(self.up)
        self.scales = np.abs(self.scales)
        self.proj = self.L.leann_projection_create(ctx, self.w, self.bias, gradient=True)
        self.rows = self.L.leann_adapter_rows_create(ctx, self.lengths, self.of, self.ranks, self.scales, self.R)
        self.a = next(a for a, n in zip(self.of, self.lengths) if a >= 0 and n)
        spans = [np.arange(s.start, s.stop) for o, s in plain64.request_rows(self.lengths, self.of) if o == self.a]
        self.mine = np.concatenate(spans)
        self.row, self.rank = int(self.mine[len(self.mine) // 2]), self.ranks[self.a]


def same(got, want, but=()):
    """Equal bits outside `but`, an index."""
    differs = (got != want).cpu().numpy()
    if but:
        differs[but] = False
    assert not differs.any(), np.argwhere(differs)[:4]


def infinite(got, sign, sure=None):
    """Infinities of the given signs (where those are sure)."""
    got = got.double().cpu().numpy()
    assert np.isinf(got).all(), (np.isnan(got).sum(), np.isfinite(got).sum(), got.size)
    right = np.sign(got) == sign
    assert right[... if sure is None else sure].all()


@params
def test_forward(ctx, dtype, case, value):
    say("infinities forward", dtype, case, value)
    p = Positive(ctx, case, dtype)
    v, a, r, n = float(value), p.a, p.rank - 1, p.up.shape[1] - 3
    out, low = p.forward(keep=True)
    p.x[p.row], p.x64[p.row] = 0.0, 0.0
    zero, _ = p.forward(keep=True)
    kept = p.up[a, n, r].item()
    p.up[a, n, r] = v
    got, got_low = p.forward(keep=True)
    rest = p.mine[p.mine != p.row]
    sign = np.sign(low.cpu().numpy()[rest, r])
    assert (sign != 0).all()
    infinite(got[rest, n], np.sign(v) * sign)
    assert bool(got[p.row, n].isnan())  # 0 x infinity
    same(got, zero, (p.mine, n))
    p.up[a, n, r] = kept
    p.x[p.row, 5] = v
    got, got_low = p.forward(keep=True)
    infinite(got[p.row], np.sign(v))
    infinite(got_low[p.row, :p.rank], np.sign(v))
    assert bool((got_low[p.row, p.rank:] == 0).all())
    same(got, out, (p.row,))
    same(got_low, low, (p.row,))
    p.close()


@params
def test_backward(ctx, dtype, case, value):
    say("infinities backward", dtype, case, value)
    p = Positive(ctx, case, dtype)
    v, a, r, n, k = float(value), p.a, p.rank - 1, p.up.shape[1] - 3, 5
    sign = np.sign(v)
    _, low = p.forward(keep=True)
    dx, ddown, dup = p.backward(low)
    grad_low = p.dout64 @ p.up64[a, :, :p.rank]
    sure = np.abs(grad_low) > 1e-3 * (np.abs(p.dout64) @ p.up64[a, :, :p.rank])  # far beyond its sum's error

    kept = p.down[a, r, k].item()
    p.down[a, r, k] = v
    got = p.backward(low)
    infinite(got[0][p.mine, k], sign * np.sign(grad_low[p.mine, r]), sure[p.mine, r])
    same(got[0], dx, (p.mine, k))
    same(got[1], ddown)
    same(got[2], dup)
    p.down[a, r, k] = kept

    kept = p.x[p.row, k].item()
    p.x[p.row, k] = v
    got = p.backward(low)
    infinite(got[1][a, :p.rank, k], sign * np.sign(grad_low[p.row]), sure[p.row])
    same(got[0], dx)
    same(got[1], ddown, (a, slice(0, p.rank), k))
    same(got[2], dup)
    p.x[p.row, k] = kept

    kept = low[p.row, r].item()
    low[p.row, r] = v
    got = p.backward(low)
    infinite(got[2][a, :, r], sign * np.sign(p.dout64[p.row]))
    same(got[0], dx)
    same(got[1], ddown)
    same(got[2], dup, (a, slice(None), r))
    low[p.row, r] = kept

    p.dout[p.row, n] = v
    got = p.backward(low)
    infinite(got[0][p.row], sign)
    infinite(got[1][a, :p.rank], sign * np.sign(p.x64[p.row]))
    infinite(got[2][a, n, :p.rank], sign * np.sign(low[p.row, :p.rank].cpu().numpy()))
    same(got[0], dx, (p.row,))
    same(got[1], ddown, (a, slice(0, p.rank)))
    same(got[2], dup, (a, n, slice(0, p.rank)))
    p.close()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES)
def test_few_bits(ctx, dtype, case):
    """Low-rank activations and elements of one or two bits, which their first piece holds: no other piece of them adds to a finite result, or takes an infinity away."""
    import torch
    say("infinities, few bits", dtype, case)
    p = Positive(ctx, case, dtype)
    p.down.zero_()
    for r in range(p.rank):
        p.down[:, r, r % p.down.shape[2]] = 1.0  # low is an element of x
    p.x.copy_(torch.from_numpy(np.random.default_rng(5).choice([-2.0, -1.0, -0.5, 0.5, 1.0, 2.0], size=tuple(p.x.shape))))
    out, low = p.forward(keep=True)
    n, r = 3, p.rank - 1
    assert bool((low[p.mine, r] == p.x[p.mine, r % p.x.shape[1]].float()).all())
    p.up[p.a, n, r] = float("inf")
    got = p.forward()
    infinite(got[p.mine, n], np.sign(low[p.mine, r].cpu().numpy()))
    same(got, out, (p.mine, n))
    # up of zeros, as training begins: gradients of down that are zeros
    p.up.zero_()
    _, ddown, dup = p.backward(low)
    assert bool((ddown == 0).all()) and not bool((dup == 0).all())
    p.dout.copy_(torch.from_numpy(np.random.default_rng(6).choice([-2.0, -1.0, 1.0], size=tuple(p.dout.shape))))
    dup = p.backward(low)[2]
    low[p.row, r] = float("inf")
    got = p.backward(low)[2]
    infinite(got[p.a, :, r], np.sign(p.dout[p.row].double().cpu().numpy()))
    same(got, dup, (p.a, slice(None), r))
    p.close()
