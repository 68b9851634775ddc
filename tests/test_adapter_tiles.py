"""Projections with adapters: the choice of tiles where many adapters meet in one (csrc/adapter_plan.h, compiled here with g++), and the large tiles with more than a hundred."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest

import adapter_plan
import plain64
import test_gpu_adapter as gpu
import test_gpu_adapter_many_rows as more
from gpu_util import say

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "adapter_plan.h"
extern "C" int choose(int cus, int64_t rows, int N, int K, int most, int64_t pairs, int64_t sixteens)
{
    AdapterLoad l;
    l.most_pairs = most;
    l.pairs = pairs;
    l.sixteens = sixteens;
    return choose_project(cus, rows, N, K, l);
}
extern "C" int shares_k(int cus, int tiles) { return low_shares_k(cus, tiles); }
extern "C" int pairs(int rank, int pieces) { return segment_pairs(rank, pieces); }
"""
MANY = (2560, 1100, 8, 8192, 4096)  # single tokens, adapters, ranks, n_in, n_out


def many():
    T, n, R, _, _ = MANY
    return [1] * T, list(np.random.default_rng(8).integers(-1, n, T)), [1 + a % R for a in range(n)]


@pytest.fixture(scope="module")
def plan():
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "plan.cpp"), "w").write(SOURCE)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2506_08276_amd", "csrc"),
                               "-o", os.path.join(d, "plan.so"), os.path.join(d, "plan.cpp")])
        lib = ctypes.CDLL(os.path.join(d, "plan.so"))

        def tile(lengths, of, ranks, N, K, pieces=1):
            """(tile, pairs of the busiest one) of a batch."""
            slots = np.concatenate([np.full(n, a) for n, a in sorted(zip(lengths, of), key=lambda p: p[1]) if a >= 0 and ranks[a]] + [np.zeros(0, int)])
            sixteens = sum(-(-int(ranks[int(a)]) // 16) for at in range(0, len(slots), 32) for a in np.unique(slots[at:at + 32]))
            each = [sum(lib.pairs(int(ranks[int(a)]), pieces) for a in np.unique(slots[at:at + 256])) for at in range(0, len(slots), 256)] or [0]
            return (32, 64, 256, 96)[lib.choose(256, ctypes.c_int64(sum(lengths)), N, K, max(each), ctypes.c_int64(sum(each)), ctypes.c_int64(sixteens))], max(each)

        yield tile, lib


def test_pairs_of_a_segment(plan):
    for rank in range(1, 129):
        slabs = -(-rank // 16)
        assert plan[1].pairs(rank, 1) == -(-slabs // 2) and plan[1].pairs(rank, 2) == slabs


@pytest.mark.parametrize("rows,adapters,rank,N,K,pieces,want", [
    (8000, 1024, 16, 768, 768, 1, 64), (8000, 4000, 16, 768, 768, 1, 64), (8000, 1024, 64, 768, 768, 2, 64), (16000, 64, 16, 768, 768, 1, 256),
    (8000, 6, 16, 2304, 768, 1, 256), (8000, 1024, 16, 2304, 768, 1, 64), (8000, 64, 64, 2304, 768, 1, 256), (64000, 4000, 16, 2304, 768, 1, 256),
    (2000, 1024, 16, 2304, 768, 1, 64), (4000, 4000, 16, 2304, 768, 1, 64), (32000, 1024, 64, 2304, 768, 1, 256), (4100, 15, 33, 1536, 384, 1, 256),
    (4100, 64, 64, 1536, 384, 1, 64), (32000, 1024, 64, 1536, 384, 1, 256), (32000, 4000, 16, 1536, 384, 1, 64)])
def test_many_adapters(plan, rows, adapters, rank, N, K, pieces, want):
    """Single tokens with adapters at random: the faster of the tiles as measured, where they differ by more than a twelfth."""
    tile, pairs = plan[0]([1] * rows, np.random.default_rng(1).integers(0, adapters, rows), [rank] * adapters, N, K, pieces)
    assert tile == want, pairs


def test_few_adapters_change_nothing(plan):
    for rows, N, K in [(1, 8, 8), (48, 768, 768), (3391, 384, 1536), (6560, 2304, 768), (82953, 768, 768), (10**6, 2304, 768)]:
        code = plan[1].choose(256, ctypes.c_int64(rows), N, K, 0, ctypes.c_int64(0), ctypes.c_int64(0))
        assert (32, 64, 256, 96)[code] == adapter_plan.tile(rows, N, K)
        code = plan[1].choose(256, ctypes.c_int64(rows), N, K, 2, ctypes.c_int64(2 * (rows + 255) // 256), ctypes.c_int64((rows + 31) // 32))
        assert (32, 64, 256, 96)[code] == adapter_plan.tile(rows, N, K)


def test_gpu_tests_still_reach_all_tiles(plan):
    for pieces in (1, 2):
        reached = {True: set(), False: set()}
        for batches, shapes in ((gpu.BATCHES, gpu.SHAPES), (gpu.LARGE, [(256, 1000), (776, 768), (768, 1160)])):
            for lengths, of, ranks in batches.values():
                for n_in, n_out in shapes:
                    reached[True].add(plan[0](lengths, of, ranks, n_out, n_in, pieces)[0])
                    reached[False].add(plan[0](lengths, of, ranks, n_in, n_out, pieces)[0])
        assert reached[True] == reached[False] == {32, 64, 96, 256}


def test_gpu_tests_reach_both_kernels_of_the_low_rank_activations(plan):
    """For 16, 32, 64 and 128 ranks, in tests that compare with 64 bits."""
    reached = set()
    for lengths, of, ranks in [*gpu.BATCHES.values(), *gpu.LARGE.values(), *((more.LENGTHS, more.OF, r) for r in more.RANKS.values())]:
        rows_of = {}
        for n, a in zip(lengths, of):
            a = a if a >= 0 and ranks[a] else -1
            rows_of[a] = rows_of.get(a, 0) + n
        room = (max(max(ranks), 1) + 7) // 8 * 8
        reached.add((next(r for r in (16, 32, 64, 128) if room <= r), bool(plan[1].shares_k(256, sum(-(-n // 16) for n in rows_of.values())))))
    assert reached == {(r, s) for r in (16, 32, 64, 128) for s in (False, True)}


def test_many_segments_go_through_the_large_tiles(plan):
    _, _, _, n_in, n_out = MANY
    tile, pairs = plan[0](*many(), n_out, n_in)
    assert tile == 256 and pairs > 100
    tile, pairs = plan[0](*many(), n_in, n_out)
    assert tile == 64


@pytest.mark.gpu
def test_a_hundred_adapters_in_a_tile():
    """More than a hundred adapters in every tile of 256 rows, forwards; backwards, a dozen in every 32 rows of the smaller tiles."""
    import torch
    import paper_2506_08276_amd as L
    T, n, R, n_in, n_out = MANY
    lengths, of, ranks = many()
    say("many adapters", *MANY)
    ctx = L.leann_create(dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1), torch.zeros(640, device="cuda:0"))
    g = torch.Generator(device="cuda:0").manual_seed(9)
    rand = lambda scale, *s: (torch.randn(s, generator=g, device="cuda:0") * scale).bfloat16()
    x, dout, w, down, up = rand(1, T, n_in), rand(0.1, T, n_out), rand(0.05, n_out, n_in), rand(n_in ** -0.5, n, R, n_in), rand(0.5, n, n_out, R)
    scales = np.random.default_rng(3).uniform(0.5, 2, n).astype(np.float32)
    proj = L.leann_projection_create(ctx, w, gradient=True)
    rows = L.leann_adapter_rows_create(ctx, lengths, of, ranks, scales, R)
    out, low = L.leann_adapter_project(ctx, proj, rows, x, down, up, keep=True)
    dx = L.leann_adapter_project_backward(ctx, proj, rows, dout, None, None, down, up, need_adapters=False)[0]
    some = np.random.default_rng(4).permutation(T)[:160]  # rows to look at
    at = torch.from_numpy(some).to("cuda:0")
    f64 = lambda t: t.double().cpu().numpy()
    w64, x64, d64 = f64(w), f64(x[at]), f64(dout[at])
    used = sorted({of[i] for i in some if of[i] >= 0})
    number = {a: i for i, a in enumerate(used)}
    pick = torch.tensor(used, device="cuda:0")
    pools = f64(down[pick]), f64(up[pick])
    batch = ([1] * len(some), [number.get(of[i], -1) for i in some], [ranks[a] for a in used], scales[used].astype(np.float64))
    a = np.abs
    want, low64 = plain64.project(x64, w64, 0.0, *pools, *batch)
    mag, mag_low = plain64.project(a(x64), a(w64), 0.0, a(pools[0]), a(pools[1]), *batch)
    gpu.close(low[at], low64, "float32", gpu.steps(n_in) * mag_low, "low")
    gpu.close(out[at], want, "bfloat16", (gpu.steps(n_in) + gpu.steps(R) + 2.0 ** -16) * mag, "out")
    none = np.zeros_like(low64)
    want = plain64.project_backward(d64, x64, none, w64, *pools, *batch)[0]
    mag = plain64.project_backward(a(d64), a(x64), none, a(w64), a(pools[0]), a(pools[1]), *batch)[0]
    gpu.close(dx[at], want, "bfloat16", (gpu.steps(n_out) + gpu.steps(R) + 2.0 ** -16) * mag, "dx")
    L.leann_projection_free(proj)
    L.leann_adapter_rows_free(rows)
    L.leann_destroy(ctx)
