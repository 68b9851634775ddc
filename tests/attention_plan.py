"""The host arithmetic of attention (csrc/attention_plan.h, no HIP in it), compiled here with g++."""
import ctypes
import functools
import os
import subprocess
import tempfile

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include <cstring>
#include "attention_plan.h"
typedef std::vector<AttentionTile> Tiles;
extern "C" int plan(int64_t left, int64_t right, int64_t sinks, int n, const int32_t *q, const int32_t *k, const int32_t *first, int keys, int share, int block, int split,
                    const char *left_out, int heads, int32_t *tiles_to, int32_t *joins_to, int32_t *items_to, int32_t *counts)
{
    Tiles tiles;
    std::vector<int32_t> of;
    std::vector<AttentionJoin> joins;
    const std::vector<char> without(left_out, left_out + n);
    att_make_tiles({left, right, sinks}, n, q, k, first, keys != 0, share, block, split, tiles, of, joins, &without);
    const std::vector<AttentionItem> items = att_order(tiles, of, heads, keys ? 1 : share);
    counts[0] = (int32_t)tiles.size(), counts[1] = (int32_t)joins.size(), counts[2] = (int32_t)items.size();
    if (!tiles_to) return 0;
    memcpy(tiles_to, tiles.data(), tiles.size() * sizeof(AttentionTile));
    memcpy(joins_to, joins.data(), joins.size() * sizeof(AttentionJoin));
    memcpy(items_to, items.data(), items.size() * sizeof(AttentionItem));
    return sizeof(AttentionTile);
}
extern "C" int split_of(const int32_t *lengths, int n, int heads, int cus, int blocks, int least)
{
    Tiles tiles(n);
    for (int i = 0; i < n; ++i) tiles[i].begin = 3, tiles[i].end = 3 + lengths[i];
    return att_split(tiles, heads, cus, blocks, least);
}
extern "C" int overlap(uint64_t a, int64_t lda, int64_t ac, int64_t ar, uint64_t b, int64_t ldb, int64_t bc, int64_t br, int size)
{
    return att_overlap(a, lda, ac, ar, b, ldb, bc, br, size);
}
"""
TILE = np.dtype([(name, np.int32) for name in ("row0", "rows", "other0", "others", "at", "first", "sink_tiles", "first_tile", "begin", "end", "slot", "per_head")] +
                [("pad", np.int32, 4)])
JOIN = np.dtype([(name, np.int32) for name in ("row0", "rows", "slot0", "slots")])
ITEM = np.dtype([("tile", np.int32), ("head", np.int32)])


@functools.lru_cache(None)
def library():
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "plan.cpp"), "w").write(SOURCE)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2506_08276_amd", "csrc"),
                               "-o", os.path.join(d, "plan.so"), os.path.join(d, "plan.cpp")])
        lib = ctypes.CDLL(os.path.join(d, "plan.so"))
        u, i = ctypes.c_uint64, ctypes.c_int64
        lib.overlap.argtypes = [u, i, i, i, u, i, i, i, ctypes.c_int]
        return lib


def make(q_rows, k_rows, first, keys, share, block, split, heads, left=-1, right=-1, sinks=0, without=None):
    """Tiles, joins and items of one side."""
    ints = lambda v: np.ascontiguousarray(v, np.int32)
    q, k, f = ints(q_rows), ints(k_rows), ints(first)
    out = np.zeros(len(q), np.int8) if without is None else np.ascontiguousarray(without, np.int8)
    at = lambda v: v.ctypes.data_as(ctypes.c_void_p)
    counts = np.zeros(3, np.int32)
    call = lambda *to: library().plan(ctypes.c_int64(left), ctypes.c_int64(right), ctypes.c_int64(sinks), len(q), at(q), at(k), at(f), int(keys), share, block, split,
                                      at(out), heads, *to, at(counts))
    call(None, None, None)
    tiles, joins, items = np.zeros(counts[0], TILE), np.zeros(counts[1], JOIN), np.zeros(counts[2], ITEM)
    assert call(at(tiles), at(joins), at(items)) == TILE.itemsize
    return tiles, joins, items


def split_of(lengths, heads, cus, blocks, least):
    lengths = np.ascontiguousarray(lengths, np.int32)
    return library().split_of(lengths.ctypes.data_as(ctypes.c_void_p), len(lengths), heads, cus, blocks, least)
