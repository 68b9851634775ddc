"""CPU checks of the tiles that projections with adapters go through, and that the GPU tests reach all of them."""
import itertools

import adapter_plan
import test_gpu_adapter as gpu

ROWS = sorted({int(1.2 ** i) for i in range(70)})


def test_the_rule():
    for N, K in itertools.product((8, 384, 768, 2304, 8192), (8, 128, 256, 768, 4096)):
        last = 32
        for rows in ROWS:
            t = adapter_plan.tile(rows, N, K)
            assert t != 256 or K >= 256  # its pipeline needs four pairs of slabs
            assert (t == 32) == (-(-rows // 32) * -(-N // 32) <= 256)
            assert t != 96 or -(-rows // 64) * -(-N // 96) <= 256 < -(-rows // 64) * -(-N // 64)  # one round instead of two
            if t == 256 and rows * N > 1 << 26:
                last = 256
            assert last != 256 or t == 256 or K < 256  # no way back to small tiles for large products


def test_large_products_take_large_tiles():
    assert adapter_plan.tile(83229, 2304, 768) == adapter_plan.tile(82953, 768, 768) == adapter_plan.tile(6560, 2304, 768) == 256
    assert adapter_plan.tile(48, 768, 768) == 32 and adapter_plan.tile(1000, 768, 768) == 64
    assert adapter_plan.tile(3391, 384, 1536) == 96


def test_gpu_tests_reach_all_tiles_in_both_directions():
    reached = {True: set(), False: set()}
    for batches, shapes in ((gpu.BATCHES, gpu.SHAPES), (gpu.LARGE, [(256, 1000), (776, 768), (768, 1160)])):
        for (lengths, _, _), (n_in, n_out) in itertools.product(batches.values(), shapes):
            reached[True].add(adapter_plan.tile(sum(lengths), n_out, n_in))
            reached[False].add(adapter_plan.tile(sum(lengths), n_in, n_out))
    assert reached[True] == reached[False] == {32, 64, 96, 256}
