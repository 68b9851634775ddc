"""A single row is one whatever its tensor says about the distance to the next."""
import pytest

from gpu_util import say
from test_gpu_adapter import ctx  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def single(t, stride, at=0):
    """The row t [1][n] as a tensor with this row stride."""
    import torch
    room = torch.full((at + max(t.shape[1], 1) + 8,), float("nan"), dtype=t.dtype, device=t.device)
    row = room.as_strided((1, t.shape[1]), (stride, 1), at)
    row.copy_(t)
    return row


@pytest.mark.parametrize("stride", [0, 1, 771, 40, 2**33 + 1])
def test_single_rows(ctx, stride):
    import torch
    import paper_2506_08276_amd as L
    say("single row", stride)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda:0").bfloat16()
    n_in, n_out = 40, 24
    x, dout, w, down, up = rand(1, n_in), rand(1, n_out), rand(n_out, n_in), rand(1, 8, n_in), rand(1, n_out, 8)
    proj = L.leann_projection_create(ctx, w, gradient=True)
    rows = L.leann_adapter_rows_create(ctx, [1], [0], [8], [2.0], 8)
    want, low = L.leann_adapter_project(ctx, proj, rows, x, down, up, keep=True)
    out = single(torch.zeros_like(want), stride)
    L.leann_adapter_project(ctx, proj, rows, single(x, stride, 8), down, up, out=out)
    assert torch.equal(out, want)
    for a, b in zip(L.leann_adapter_project_backward(ctx, proj, rows, single(dout, stride), single(x, stride), low, down, up),
                    L.leann_adapter_project_backward(ctx, proj, rows, dout, x, low, down, up)):
        assert torch.equal(a, b)
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)
    gamma, beta, drop = torch.ones(n_in, device="cuda:0"), torch.zeros(n_in, device="cuda:0"), (0.3, 5, 6)
    row, res = rand(1, n_in), rand(1, n_in)
    assert torch.equal(L.leann_dropout(ctx, single(row, stride), drop, residual=single(res, stride)), L.leann_dropout(ctx, row, drop, residual=res))
    want = L.leann_layernorm(ctx, row, gamma, beta, 1e-5, residual=res, drop=drop, keep=True)
    got = L.leann_layernorm(ctx, single(row, stride), gamma, beta, 1e-5, residual=single(res, stride), drop=drop, keep=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    want_back = L.leann_layernorm_backward(ctx, row, *want[1:], gamma, drop=drop, dtotal=res)
    got_back = L.leann_layernorm_backward(ctx, single(row, stride), single(want[1], stride), *want[2:], gamma, drop=drop, dtotal=single(res, stride))
    assert all(torch.equal(a, b) for a, b in zip(got_back, want_back))


@pytest.mark.parametrize("rows", [1, 3])
def test_single_columns(ctx, rows):
    """Rows of one element, in a tensor with any column stride."""
    import torch
    import paper_2506_08276_amd as L
    say("single column", rows)
    x = torch.arange(1, 1 + 6 * rows, dtype=torch.float32, device="cuda:0").as_strided((rows, 1), (6, 5))
    assert torch.equal(L.leann_dropout(ctx, x, (0.0, 1, 2)), x)
