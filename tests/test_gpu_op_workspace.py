"""The operators' workspace makes room for what else the context allocates."""
import numpy as np
import pytest

import leann_inputs as li
from gpu_util import say, to_dev

pytestmark = pytest.mark.gpu
CFG = dict(layers=1, hidden=128, heads=2, ffn=512, vocab=500, max_pos=256, ln_eps=1e-12)
T = 1 << 22  # rows of 128 ranks: 2.1 GB of pieces


@pytest.fixture
def pressed():
    """A context whose operators have taken 2.1 GB, the call that took them, and a way to leave some 300 MB (up to half a gigabyte more has been seen)."""
    import torch
    import paper_2506_08276_amd as L
    ctx = L.leann_create(CFG, to_dev(li.encoder_weights(CFG, 3)))
    half = dict(dtype=torch.bfloat16, device="cuda:0")
    x, w = torch.ones((T, 8), **half), torch.eye(8, **half)
    down, up = torch.full((1, 128, 8), 0.125, **half), torch.full((1, 8, 128), 0.5, **half)
    proj = L.leann_projection_create(ctx, w)
    rows = L.leann_adapter_rows_create(ctx, [T], [0], [128], [1.0], 128)
    call = lambda: L.leann_adapter_project(ctx, proj, rows, x, down, up)

    def with_little_room(use):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        hold = torch.empty(torch.cuda.mem_get_info()[0] - (300 << 20), dtype=torch.uint8, device="cuda:0")
        try:
            return use()
        finally:
            del hold
            torch.cuda.empty_cache()

    before = torch.cuda.mem_get_info()[0]
    out = call()
    assert bool((out == 65).all())  # 1 + 128 x 0.5 x 1
    assert before - torch.cuda.mem_get_info()[0] >= T * 512 - (64 << 20)
    del out
    yield ctx, call, with_little_room
    assert bool((call() == 65).all())  # allocated anew
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)
    L.leann_destroy(ctx)


def test_an_encoder_pass_finds_memory(pressed):
    import torch
    import paper_2506_08276_amd as L
    ctx, _, with_little_room = pressed
    tokens, lengths = li.uniform_chunks(2048, 256, 1, CFG["vocab"], 1, 256, 31)  # 524 288 padded rows: 1.3 GB
    t, l = to_dev(tokens), to_dev(lengths)
    other = L.leann_create(CFG, to_dev(li.encoder_weights(CFG, 3)))
    want = L.leann_embed(other, t, l, hidden=CFG["hidden"])
    L.leann_destroy(other)
    out = torch.empty_like(want)
    say("embed beside the operators' workspace")
    with_little_room(lambda: L.leann_embed(ctx, t, l, hidden=CFG["hidden"], out=out))
    assert torch.equal(out, want)


def test_pq_training_finds_memory(pressed):
    import torch
    import paper_2506_08276_amd as L
    ctx, _, with_little_room = pressed
    emb = torch.randn((65536, 4096), generator=torch.Generator("cuda:0").manual_seed(6), device="cuda:0")  # scratch of 1.1 GB
    say("train beside the operators' workspace")
    pq = with_little_room(lambda: L.leann_build_pq(ctx, emb, 128, 1, 7))
    got = L.leann_pq_export(ctx, pq)
    L.leann_pq_free(pq)
    pq = L.leann_build_pq(ctx, emb, 128, 1, 7)
    assert all(np.array_equal(a, b) for a, b in zip(got, L.leann_pq_export(ctx, pq)))
    L.leann_pq_free(pq)
