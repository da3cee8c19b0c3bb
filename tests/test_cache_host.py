"""The refusals of the cache's entry points: found on the host, before anything is launched."""
import pytest

import paper_2409_16626_b200 as H

OK, NULL, DTYPE, ROUND, FLAGS, RANGE, SHAPE, ALIGN, WORKSPACE, OVERLAP = 0, 1, 2, 3, 4, 5, 6, 7, 8, 11
M = 1 << 20
CACHE = dict(k_pages=16 * M, v_pages=32 * M, k_exp=48 * M, v_exp=49 * M, n_pages=8, kv_heads=2, page_tokens=16, head_dim=64, page_table=50 * M, table_stride=4)
APPEND = dict(k=64 * M, v=65 * M, src_dtype=H.BF16, token_stride=128, head_stride=64, d_new_start=51 * M, d_lengths=52 * M, n_seqs=2, n_new=10, **CACHE)
READ = dict(d_first=51 * M, d_out_start=52 * M, n_seqs=2, n_out=10, k=64 * M, v=65 * M, dst_dtype=H.F32, token_stride=128, head_stride=64, **CACHE)
FORK = dict(d_lengths=51 * M, n_seqs=2, d_parent=52 * M, d_new_page=53 * M, n_children=3, table_out=54 * M, table_out_stride=4, d_lengths_out=55 * M, **CACHE)
COMPACT = dict(d_lengths=51 * M, n_seqs=2, move=1, d_n_live=52 * M, d_free_pages=53 * M, workspace=54 * M, workspace_bytes=1 << 16, **CACHE)
ATTENTION = dict(q=64 * M, dtype=H.BF16, q_token_stride=256, q_head_stride=64, d_q_start=51 * M, d_lengths=52 * M, n_seqs=2, n_q=10, max_q=8, max_length=64, heads=4,
                 softmax_scale=0.125, causal=1, window=0, out=66 * M, out_token_stride=256, out_head_stride=64, lse=67 * M, workspace=68 * M, workspace_bytes=1 << 28, **CACHE)
CALLS = {"attention": (H.hif8_cache_attention, ATTENTION), "append": (H.hif8_cache_append, APPEND), "read": (H.hif8_cache_read, READ), "fork": (H.hif8_cache_fork, FORK), "compact": (H.hif8_cache_compact, COMPACT)}

EVERY = [(dict(n_pages=-1), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=129), SHAPE), (dict(page_tokens=48), SHAPE), (dict(page_tokens=256), SHAPE),
         (dict(page_tokens=0), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=512), SHAPE), (dict(table_stride=0), SHAPE), (dict(k_pages=None), NULL), (dict(v_pages=None), NULL),
         (dict(k_exp=None), NULL), (dict(v_exp=None), NULL), (dict(page_table=None), NULL), (dict(k_pages=16 * M + 8), ALIGN), (dict(v_pages=32 * M + 1), ALIGN),
         (dict(k_exp=48 * M + 2), ALIGN), (dict(page_table=50 * M + 1), ALIGN), (dict(n_seqs=-1), SHAPE)]
OWN = {
    "attention": [(dict(dtype=H.F32), DTYPE), (dict(dtype=5), DTYPE), (dict(n_seqs=4097), SHAPE), (dict(n_q=-1), SHAPE), (dict(max_q=-1), SHAPE), (dict(max_length=-1), SHAPE),
                  (dict(window=-1), SHAPE), (dict(heads=3), SHAPE), (dict(heads=0), SHAPE), (dict(heads=130), SHAPE), (dict(q_token_stride=-1), SHAPE),
                  (dict(out_token_stride=0), SHAPE), (dict(out_head_stride=63), SHAPE), (dict(out_token_stride=192), SHAPE), (dict(n_q=1 << 30), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 27), SHAPE),
                  (dict(softmax_scale=0.0), RANGE), (dict(softmax_scale=-1.0), RANGE), (dict(softmax_scale=float("nan")), RANGE), (dict(softmax_scale=float("inf")), RANGE),
                  (dict(q=None), NULL), (dict(out=None), NULL), (dict(d_q_start=None), NULL), (dict(d_lengths=None), NULL), (dict(q=64 * M + 1), ALIGN), (dict(lse=67 * M + 2), ALIGN),
                  (dict(out=64 * M + 64), OVERLAP), (dict(out=16 * M), OVERLAP), (dict(out=32 * M), OVERLAP), (dict(workspace=None), WORKSPACE),
                  (dict(workspace=68 * M + 16), WORKSPACE), (dict(workspace_bytes=1 << 15), WORKSPACE), (dict(d_q_start=51 * M + 2), ALIGN), (dict(n_seqs=2049), SHAPE), (dict(n_q=0), OK), (dict(n_seqs=0), OK)],
    "append": [(dict(src_dtype=3), DTYPE), (dict(rnd=H.RND_SR), ROUND), (dict(rnd=7), ROUND), (dict(flags=4), FLAGS), (dict(target_exp=16), RANGE), (dict(target_exp=-23), RANGE),
               (dict(n_seqs=4097), SHAPE), (dict(n_new=-1), SHAPE), (dict(token_stride=-128), SHAPE), (dict(head_stride=-1), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL),
               (dict(d_new_start=None), NULL), (dict(d_lengths=None), NULL), (dict(k=64 * M + 1), ALIGN), (dict(src_dtype=H.F32, v=65 * M + 2), ALIGN),
               (dict(k=16 * M), OVERLAP), (dict(v=32 * M + 16), OVERLAP), (dict(v_pages=16 * M), OVERLAP), (dict(n_new=0), OK), (dict(n_seqs=0), OK),
               (dict(d_new_start=51 * M + 2), ALIGN), (dict(d_lengths=52 * M + 1), ALIGN), (dict(n_seqs=2049), SHAPE)],
    "read": [(dict(dst_dtype=-1), DTYPE), (dict(n_out=-1), SHAPE), (dict(n_seqs=4097), SHAPE), (dict(token_stride=64), SHAPE), (dict(token_stride=0), SHAPE), (dict(head_stride=63), SHAPE),
             (dict(token_stride=64, head_stride=600), SHAPE), (dict(k=None), NULL), (dict(d_first=None), NULL), (dict(d_out_start=None), NULL), (dict(k=64 * M + 2), ALIGN),
             (dict(k=16 * M + 64), OVERLAP), (dict(k=65 * M), OVERLAP), (dict(n_out=0), OK),
             (dict(v=64 * M + 4), OVERLAP), (dict(v=64 * M + 252), OVERLAP), (dict(v=64 * M + 256), OVERLAP), (dict(v=64 * M - 128 * 9 * 4), OVERLAP), (dict(v=64 * M + 64 * 19 * 4 + 252), OVERLAP),
             (dict(token_stride=256, v=64 * M + 256), OVERLAP), (dict(token_stride=256, v=64 * M - 768), OVERLAP), (dict(token_stride=64, head_stride=700, v=64 * M + 4 * 700), OVERLAP),
             (dict(d_first=51 * M + 1), ALIGN), (dict(d_out_start=52 * M + 2), ALIGN)],
    "fork": [(dict(n_children=-1), SHAPE), (dict(n_children=4097), SHAPE), (dict(table_out_stride=0), SHAPE), (dict(d_lengths=None), NULL), (dict(d_parent=None), NULL),
             (dict(table_out=None), NULL), (dict(d_lengths_out=None), NULL), (dict(table_out=50 * M + 16), OVERLAP), (dict(d_lengths_out=51 * M + 4), OVERLAP), (dict(n_children=0), OK),
             (dict(d_parent=52 * M + 2), ALIGN), (dict(d_new_page=53 * M + 2), ALIGN), (dict(table_out=54 * M + 1), ALIGN), (dict(d_lengths_out=55 * M + 2), ALIGN), (dict(n_children=2049), SHAPE)],
    "compact": [(dict(n_seqs=4097), SHAPE), (dict(d_lengths=None), NULL), (dict(d_n_live=None), NULL), (dict(d_free_pages=None), NULL), (dict(workspace=None), WORKSPACE),
                (dict(workspace_bytes=255), WORKSPACE), (dict(workspace=54 * M + 16), WORKSPACE),
                (dict(d_lengths=51 * M + 2), ALIGN), (dict(d_n_live=52 * M + 2), ALIGN), (dict(d_free_pages=53 * M + 1), ALIGN)],
}


@pytest.mark.parametrize("call,change,status", [(c, *e) for c in CALLS for e in EVERY + OWN[c]])
def test_refusals(call, change, status):
    fn, good = CALLS[call]
    before = H.hif8_launch_count()
    assert fn(**{**good, **change}, stream=0, check=False) == status
    assert H.hif8_launch_count() == before


def test_a_refusal_raises():
    with pytest.raises(H.Hif8Error):
        H.hif8_cache_append(**{**APPEND, "head_dim": 100}, stream=0)


def test_workspace_bytes():
    sizes = [H.hif8_cache_compact_workspace_bytes(n) for n in (-5, 0, 1, 31, 1000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] == sizes[1] and sizes[-1] >= 3 * 4 * (1 << 20)


def test_attention_workspace_bytes():
    size = H.hif8_cache_attention_workspace_bytes
    assert size(4, 4, 1, 1000, 8, 2, 128) > 33000 and size(4, 4, 1, 1000, 8, 3, 128) == 0 and size(4, 4, 1, 1000, 8, 2, 100) == 0 and size(-1, 4, 1, 1000, 8, 2, 128) == 0
    assert size(4, 4, 1, 1000, 8, 2, 128) % 256 == 0


def test_attention_workspace_stays_within_a_device():
    size = H.hif8_cache_attention_workspace_bytes
    assert size(2048, 1 << 20, 1 << 20, 1 << 30, 64, 1, 128) < (16 << 30) + (1 << 28)
    assert size(64, 1024, 16, 131072, 64, 8, 128) < 1 << 28     # 34 GB of tiles: not asked for
    assert size(4, 4096, 1024, 16384, 32, 8, 128) > 4 * 16384 * 8 * 128 * 4
