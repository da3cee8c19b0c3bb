"""Overlaps that the cache's entry points refuse: results in the place of what the same call reads."""
import pytest

import paper_2409_16626_b200 as H
from test_cache_host import APPEND, ATTENTION, COMPACT, FORK, M, READ

CALLS = {"append": (H.hif8_cache_append, APPEND), "read": (H.hif8_cache_read, READ), "attention": (H.hif8_cache_attention, ATTENTION), "fork": (H.hif8_cache_fork, FORK),
         "compact": (H.hif8_cache_compact, COMPACT)}
OVERLAP = 11
CASES = {
    "append": [dict(v_exp=48 * M), dict(v_exp=48 * M + 4 * 15), dict(k_exp=16 * M + 64), dict(v_exp=32 * M), dict(k_exp=51 * M - 4 * 15), dict(v_exp=52 * M + 4),
               dict(k_exp=50 * M + 4), dict(page_table=48 * M), dict(d_lengths=16 * M + 128), dict(d_new_start=32 * M), dict(page_table=32 * M + 16), dict(k_exp=64 * M), dict(v_exp=65 * M + 4)],
    "fork": [dict(table_out=51 * M), dict(table_out=52 * M + 8), dict(table_out=53 * M - 4 * 11), dict(d_lengths_out=50 * M + 4 * 7), dict(d_lengths_out=52 * M), dict(d_lengths_out=53 * M + 8),
             dict(d_lengths_out=54 * M + 4 * 11), dict(table_out=16 * M), dict(table_out=32 * M + 64), dict(table_out=48 * M), dict(d_lengths_out=49 * M + 4 * 15), dict(d_lengths_out=16 * M),
             dict(v_exp=48 * M + 4), dict(v_pages=16 * M), dict(d_parent=48 * M), dict(page_table=16 * M + 64), dict(d_new_page=49 * M + 4)],
    "compact": [dict(d_n_live=51 * M + 4), dict(d_n_live=50 * M), dict(d_free_pages=51 * M), dict(d_free_pages=50 * M + 4 * 7), dict(d_n_live=53 * M + 4 * 7), dict(workspace=50 * M - 512),
                dict(workspace=51 * M), dict(workspace=53 * M), dict(workspace=16 * M), dict(d_free_pages=32 * M), dict(d_free_pages=48 * M), dict(d_n_live=49 * M), dict(page_table=51 * M - 4 * 7),
                dict(page_table=48 * M), dict(v_exp=48 * M + 4 * 15), dict(v_pages=16 * M), dict(d_lengths=16 * M), dict(d_lengths=48 * M)],
    "read": [dict(k=48 * M), dict(v=49 * M + 4), dict(k=50 * M), dict(v=51 * M), dict(k=52 * M - 4)],
    "attention": [dict(out=48 * M), dict(out=49 * M), dict(out=50 * M + 16), dict(out=51 * M), dict(out=52 * M + 4), dict(lse=64 * M), dict(lse=66 * M + 64), dict(lse=16 * M), dict(lse=48 * M),
                  dict(lse=50 * M), dict(lse=51 * M + 4), dict(workspace=64 * M), dict(workspace=66 * M), dict(workspace=67 * M), dict(workspace=50 * M), dict(workspace=16 * M),
                  dict(workspace=52 * M), dict(workspace=48 * M)],
}


@pytest.mark.parametrize("call,change", [(c, x) for c in CASES for x in CASES[c]])
def test_overlaps(call, change):
    fn, good = CALLS[call]
    args = {**good, **change}
    before = H.hif8_launch_count()
    assert fn(**args, stream=0, check=False) == OVERLAP
    assert H.hif8_launch_count() == before
