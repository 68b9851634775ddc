"""Which tiles attention's blocks go through, against the rule of which query sees which key; and which matrices share bytes, against sets of bytes."""
import itertools

import numpy as np
import pytest

from attention_plan import library, make, split_of

RAGGED = dict(q_rows=[70, 0, 1, 300, 5, 64], k_rows=[70, 9, 130, 520, 0, 64], first=[0, 0, 129, 220, 7, 0])
RULES = [dict(), dict(left=0, right=0), dict(left=-1, right=0), dict(left=30, right=30), dict(left=64, right=0, sinks=3), dict(left=10, right=0, sinks=200),
         dict(left=5, right=100, sinks=64), dict(left=1 << 30, right=1 << 30)]


def seen(first, lq, lk, left=-1, right=-1, sinks=0):
    """[lq, lk]: the rule itself."""
    p, j = first + np.arange(lq)[:, None], np.arange(lk)[None]
    return ((right < 0) | (j <= p + right)) & ((left < 0) | (j >= p - left) | (j < sinks))


@pytest.mark.parametrize("rules", RULES, ids=str)
@pytest.mark.parametrize("keys,share,heads,block", [(False, 1, 4, 32), (False, 2, 4, 128), (True, 1, 4, 128), (True, 2, 2, 64)])
@pytest.mark.parametrize("split", [0, 2])
def test_tiles_hold_what_is_seen_once(rules, keys, share, heads, block, split):
    q_rows, k_rows, first = RAGGED.values()
    tiles, joins, items = make(q_rows, k_rows, first, keys, share, block, split, heads, **rules)
    q0, k0 = np.cumsum([0] + q_rows), np.cumsum([0] + k_rows)
    own0, other0, own_rows, other_rows = (k0, q0, k_rows, q_rows) if keys else (q0, k0, q_rows, k_rows)
    taken = np.zeros((own0[-1], other0[-1], share if keys else 1), np.int32)
    rows = np.zeros(own0[-1], np.int32)
    parts = {}
    for t in tiles:
        s = next(s for s in range(len(q_rows)) if own0[s] <= t["row0"] < own0[s + 1])
        i = t["row0"] - own0[s]
        assert 0 < t["rows"] <= block and i + t["rows"] <= own_rows[s] and t["other0"] == other0[s] and t["others"] == other_rows[s]
        assert t["first"] == first[s] and t["at"] == (i if keys else first[s] + i)
        assert 0 <= t["begin"] <= t["end"] and (not split or t["end"] - t["begin"] <= split)
        if t["slot"] < 0: rows[t["row0"]:t["row0"] + t["rows"]] += 1
        else: parts[int(t["slot"])] = (int(t["row0"]), int(t["rows"]))
        for u in range(t["begin"], t["end"]):
            head, u = divmod(u, t["per_head"])
            tile = u if u < t["sink_tiles"] else t["first_tile"] + u - t["sink_tiles"]
            at = other0[s] + 64 * tile
            assert tile >= 0 and 64 * tile < other_rows[s] and (keys or head == 0)  # no tile is behind the sequence
            taken[t["row0"]:t["row0"] + t["rows"], at:min(at + 64, other0[s + 1]), head] += 1
    slots = [p for j in joins for p in range(j["slot0"], j["slot0"] + j["slots"])]
    assert sorted(parts) == slots == list(range(len(slots)))
    for j in joins:
        assert j["slots"] > 1 and all(parts[p] == (j["row0"], j["rows"]) for p in range(j["slot0"], j["slot0"] + j["slots"]))
        rows[j["row0"]:j["row0"] + j["rows"]] += 1
    assert (rows == 1).all()  # each row is written by one block or one join
    assert taken.max() <= 1
    for s in range(len(q_rows)):
        see = seen(first[s], q_rows[s], k_rows[s], **rules)
        mine = taken[own0[s]:own0[s + 1], other0[s]:other0[s + 1]]
        assert (mine[see.T if keys else see] == 1).all()
        mine[...] = 0
    assert not taken.any()  # nothing of another sequence
    pairs = [(int(i["tile"]), int(i["head"])) for i in items if i["tile"] >= 0]
    assert sorted(pairs) == list(itertools.product(range(len(tiles)), range(heads)))


def test_a_hidden_stretch_has_no_tiles():
    tiles, _, _ = make([64], [4096], [4000], False, 1, 64, 0, 1, left=63, right=0, sinks=4)
    assert [int(t["end"]) for t in tiles] == [1 + 3]  # the first keys' tile; keys 3937 .. 4063 lie in tiles 61 .. 63
    tiles, _, _ = make([4096], [4096], [0], True, 1, 64, 0, 1, left=63, right=0, sinks=4)
    assert [int(t["end"]) for t in tiles] == [64] + [2] * 62 + [1]


def test_sequences_left_out():
    tiles, _, items = make([40, 50, 60], [40, 50, 60], [0, 0, 0], True, 1, 64, 0, 2, without=[0, 1, 0])
    assert [(int(t["row0"]), int(t["rows"]), int(t["other0"])) for t in tiles] == [(0, 40, 0), (90, 60, 90)]
    assert sorted((int(i["tile"]), int(i["head"])) for i in items if i["tile"] >= 0) == [(0, 0), (0, 1), (1, 0), (1, 1)]


def test_nothing_to_do():
    for q, k in (([], []), ([0, 0], [0, 0])):
        for keys in (False, True):
            tiles, joins, items = make(q, k, [0] * len(q), keys, 1, 64, 0, 4)
            assert not len(tiles) and not len(joins) and not len(items)


def test_splits():
    assert split_of([8] * 1000, 4, 256, 4, 4) == 0  # the units are full
    assert split_of([100], 1, 256, 4, 4) == 4       # one long one: the least part
    assert split_of([4], 1, 256, 4, 4) == 0         # nothing to split
    split = split_of([4096], 8, 256, 4, 4)          # parts that make four blocks per unit
    assert split == 4096 * 8 // 1024 and -(-4096 // split) * 8 == 1024
    assert split_of([], 8, 256, 4, 4) == 0


def test_work_is_spread():
    """Of many alike sequences each eighth of the blocks has its share, and a sequence's blocks are in one eighth."""
    tiles, _, items = make([256] * 64, [256] * 64, [0] * 64, False, 1, 128, 0, 4)
    eighths = [items[x::8] for x in range(8)]
    assert {len(e) for e in eighths} == {64}
    of = {}
    for x, e in enumerate(eighths):
        for i in e: of.setdefault((int(tiles[i["tile"]]["other0"]), int(i["head"])), set()).add(x)
    assert all(len(v) == 1 for v in of.values())


def test_overlap_against_sets_of_bytes():
    f = library().overlap
    span = lambda at, ld, cols, rows: {at + 2 * (i * ld + c) + e for i in range(rows) for c in range(cols) for e in range(2)}
    for ar, br, lda, ldb in itertools.product((0, 1, 2, 4), (0, 1, 3), (1, 3, 4), (1, 2, 4, 7)):
        for ac, bc in itertools.product(range(1, lda + 1), range(1, ldb + 1)):
            a = span(100, lda, ac, ar)
            for at in range(40, 150):
                assert bool(f(100, lda, ac, ar, at, ldb, bc, br, 2)) == bool(a & span(at, ldb, bc, br)), (ar, br, lda, ldb, ac, bc, at)
