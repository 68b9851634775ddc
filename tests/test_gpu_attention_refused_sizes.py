"""Batches of more blocks than a launch has are refused before tables are made of them."""
import resource

import pytest

from gpu_util import say
from test_gpu_attention import ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [dict(q_rows=[(1 << 30) - 1]), dict(q_rows=[0], k_rows=[(1 << 30) - 1]), dict(q_rows=[1 << 28] * 7, kv_heads=1)], ids=["queries", "keys", "several"])
def test_no_tables_of_what_is_refused(ctx, rows):  # noqa: F811
    import paper_2506_08276_amd as L
    say("attention, too many blocks", rows)
    before = resource.getrusage(resource.RUSAGE_SELF).ru_maxrss
    with pytest.raises(L.LeannError) as e:
        L.leann_attention_create(ctx, rows["q_rows"], rows.get("k_rows"), heads=1024, head_dim=8, kv_heads=rows.get("kv_heads"))
    assert e.value.status == -4 and "workgroups" in str(e.value)
    assert resource.getrusage(resource.RUSAGE_SELF).ru_maxrss - before < 1 << 18  # KB: the first of the tables alone would be 512 MB


def test_many_blocks_still_go(ctx):  # noqa: F811
    """Half a million rows of 64 heads: 262 144 blocks."""
    import paper_2506_08276_amd as L
    say("attention, many blocks")
    for rows in (dict(q_rows=[4096] * 128), dict(q_rows=[1] * 4096)):
        L.leann_attention_free(L.leann_attention_create(ctx, rows["q_rows"], heads=64, head_dim=64))
