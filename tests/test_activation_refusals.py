"""Calls of attention and of activations that are refused before the device is touched."""
import ctypes
import os

import pytest

EINVAL = -1


@pytest.fixture(scope="module")
def lib():
    import paper_2506_08276_amd as L
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libleann.so not built (run __graft_entry__.build())")
    return L.load_library()


def test_null_arguments(lib):
    zeros = [None, 0]
    calls = [
        lambda: lib.leann_attention_create(None, None, None, None, 0, None, None),
        lambda: lib.leann_attention(None, None, None, 0, None, 0, None, 0, 1, 1.0, None, None, 0, None),
        lambda: lib.leann_attention_backward(None, None, *zeros * 5, None, 1, 1.0, None, *zeros * 3, None),
        lambda: lib.leann_checkpoint(None, None, 0, 1, 1, 0, None, 0, None),
        lambda: lib.leann_checkpoint_restore(None, None, 0, None, 1, 1, 0, None, 0),
        lambda: lib.leann_activation(None, None, 0, 1, 1, 0, 0, None, 0, None, 0, None),
        lambda: lib.leann_activation_backward(None, None, 0, None, 0, None, 0, None, 1, 1, 0, 0, None, 0, None, 0),
    ]
    for call in calls:
        assert call() == EINVAL
        assert len(lib.leann_last_error(None)) > 0
    lib.leann_attention_free(None)


def test_position_buckets(lib):
    """The table against whole-number arithmetic, and what it refuses."""
    import numpy as np
    import paper_2506_08276_amd as L
    for buckets, distance, both in [(4, 2, True), (8, 100, True), (32, 128, True), (32, 128, False), (64, 1000, True), (16, 1024, False), (2, 2, False), (128, 33, True)]:
        half = buckets // 2 if both else buckets
        single = half // 2
        got = L.leann_position_buckets(buckets, distance, both)
        assert got.shape == (2 * distance + 1,)
        for d in range(-distance, distance + 1):
            n = -d if d < 0 else d if both else 0
            b = n
            if n >= single:  # the largest b whose lower bound single (distance / single)^((b - single) / (half - single)) is not above n
                b = max(b for b in range(single, half) if n ** (half - single) * single ** (b - single) >= distance ** (b - single) * single ** (half - single))
            assert got[d + distance] == b + (half if both and d > 0 else 0), (buckets, distance, both, d)
    out = np.zeros(5000, np.int32)
    for args in [(1, 5, 0), (3, 5, 1), (32, 8, 1), (32, 1025, 1), (5000, 1024, 0), (32, -1, 1)]:
        assert lib.leann_position_buckets(*args, out.ctypes.data) == EINVAL
    assert lib.leann_position_buckets(32, 128, 1, None) == EINVAL
