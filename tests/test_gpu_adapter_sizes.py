"""Sizes of projections with adapters beyond what a launch takes: refused before anything is launched."""
import pytest

from gpu_util import say
from test_gpu_adapter import ctx  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
ESHAPE = -4


def test_more_tiles_than_a_launch_takes(ctx):
    """2^20 + 64 rows x 65 536 columns at K of 8 in tiles of 64 x 64: 2^24 + 1024."""
    import torch
    import paper_2506_08276_amd as L
    lib = L.load_library()
    T, n_in, n_out = (1 << 20) + 64, 8, 65536
    x, w = (torch.zeros(s, dtype=torch.bfloat16, device="cuda:0") for s in ((T, n_in), (n_out, n_in)))
    out = torch.zeros(64, dtype=torch.bfloat16, device="cuda:0")  # never written: 137 GB would be
    proj = L.leann_projection_create(ctx, w)
    rows = L.leann_adapter_rows_create(ctx, [T], [-1], [8], [1.0], 8)  # no adapter: nothing but the product to launch
    say("refused", T, n_in, n_out)
    rc = lib.leann_adapter_project(ctx, proj, rows, x.data_ptr(), n_in, w.data_ptr(), w.data_ptr(), out.data_ptr(), n_out, None)
    assert rc == ESHAPE and b"workgroups" in lib.leann_last_error(None)
    torch.cuda.synchronize()
    assert bool((out == 0).all())
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)


def test_more_adapters_than_a_launch_takes(ctx):
    """Gradients of 2049 adapters with 128 ranks at 65 536 columns: 2^24 + 8192 pieces of 32 x 32 to turn."""
    import torch
    import paper_2506_08276_amd as L
    n, n_in, n_out, R = 2049, 8, 65536, 128
    half = dict(dtype=torch.bfloat16, device="cuda:0")
    proj = L.leann_projection_create(ctx, torch.zeros((n_out, n_in), **half), gradient=True)
    rows = L.leann_adapter_rows_create(ctx, [1] * n, list(range(n)), [R] * n, [1.0] * n, R)
    down, up, dout = torch.zeros((n, R, n_in), **half), torch.empty((n, n_out, R), **half), torch.zeros((n, n_out), **half)  # up: 34 GB
    say("refused", n, n_in, n_out, R)
    with pytest.raises(L.LeannError) as e:
        L.leann_adapter_project_backward(ctx, proj, rows, dout, None, None, down, up, need_adapters=False)
    assert e.value.status == ESHAPE and "workgroups" in str(e.value)
    torch.cuda.synchronize()
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)
    del up, dout
    torch.cuda.empty_cache()
