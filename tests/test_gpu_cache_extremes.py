"""Attention over the HiF8 key/value cache where factors, weights and values lie at the ends of their ranges.

Each case goes through both kernels: few query rows, and chunks (a workspace without room for tiles takes a chunk through the first).
Tolerances are those of test_gpu_cache_attention, derived there."""
import math

import numpy as np
import pytest
import torch

import paper_2409_16626_b200 as H
from cache_util import VALUES, starts
from test_gpu_cache_attention import BF16, F16, attend, close, make, reference

pytestmark = pytest.mark.gpu
FORMS = [([1, 1], False), ([3, 2], False), ([70, 40], True), ([70, 40], False)]  # queries of each sequence, least workspace


@pytest.mark.parametrize("counts,small", FORMS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_exp,k_exp,scale", [(-112, 24, None), (-120, 48, None), (-90, 48, None), (-70, 48, 1e-10), (0, 0, 1e-40), (-60, -48, 1e-40)])
def test_factors_of_scores_that_vanish(counts, small, dim, q_exp, k_exp, scale):
    """Tokens that a row does not see stay unseen however small the factor of its scores is: the result is a plain mean."""
    c, q = make([70, 333], counts, 8, 2, 32, dim, BF16, seed=dim)
    c.h["k_exp"][:] = k_exp
    c.upload()
    out, lse = close(c, (q.float() * 2.0 ** q_exp).bfloat16(), counts, 8, scale=scale, small=small)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("counts,small", FORMS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_exp,k_exp,scale", [(100, 0, None), (120, 48, None), (90, -9, 0.5), (80, 40, 1e10), (120, 48, 1e10)])
def test_factors_of_scores_beyond_the_ordinary(counts, small, dim, q_exp, k_exp, scale):
    """Queries of up to 2^120: the logarithms of the sums are those of the formula on either kernel."""
    c, q = make([70, 333], counts, 8, 2, 32, dim, BF16, seed=dim)
    c.h["k_exp"][:] = k_exp
    c.upload()
    out, lse = close(c, (q.float() * 2.0 ** q_exp).bfloat16(), counts, 8, scale=scale, small=small)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("counts,small", FORMS)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (256, 16)])
@pytest.mark.parametrize("small_v", [-20, -30, -45])
@pytest.mark.parametrize("window", [0, 60])
def test_blocks_of_zeros_beside_small_values(counts, small, dim, page, small_v, window):
    """Blocks of V that hold zeros have exponent 0, as a call of append gives them, and the others values around 2^small_v: the zeros take part in the denominator, and
    do not push the others' weights out of FP16.  Slots behind a sequence's length hold other values."""
    lengths = [70, 333]
    c, q = make(lengths, counts, 8, 2, page, dim, BF16, seed=dim - small_v)
    c.fill(0)
    c.h["v_exp"] += -small_v
    for s, n in enumerate(lengths):
        blocks = -(-n // page)
        for block in {0, 1, blocks // 2, blocks - 1} - {blocks // 2 + 1}:
            p = c.table[s, block]
            c.h["v_exp"][p] = 0
            c.h["v"][p, :, :min(page, n - block * page)] = 0
            c.h["v"][p, :, min(page, n - block * page):] = 0x48
    c.h["v_exp"] = np.clip(c.h["v_exp"], -H.CACHE_EXP_MAX, H.CACHE_EXP_MAX)
    c.upload()
    for scale in (0.05, None):
        close(c, q, counts, 8, window=window, scale=scale, small=small)


def test_zeros_only():
    for counts in ([1, 1], [70, 40]):
        c, q = make([70, 333], counts, 8, 2, 16, 64, BF16)
        c.h["v"][:], c.h["v_exp"][:] = 0, 0
        c.upload()
        out, _ = close(c, q, counts, 8)
        assert (out == 0).all()


def expect_specials(c, q, counts, heads, window, scale, **kw):
    """Where a query sees Inf or NaN among an element's values, the result is that Inf, or NaN of NaN or both signs, whatever the weights are; elsewhere what the other values give."""
    out, lse = attend(c, q, counts, heads, 1, window, scale, **kw)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    stale, c.h["v"] = c.h["v"], np.where(np.isfinite(VALUES[c.h["v"]]), c.h["v"], 0).astype(np.uint8)
    want, norm, tol, tol_lse = reference(c, q, counts, heads // c.shape[1], scale, 1, window)
    c.h["v"] = stale
    _, kv, page, _ = c.shape
    special, at = torch.zeros_like(want, dtype=torch.bool), 0
    for s, (n, m) in enumerate(zip(c.lengths, counts)):
        codes = c.h["v"][c.table[s, :-(-n // page)]].transpose(1, 0, 2, 3).reshape(kv, -1, c.shape[3])[:, :n]
        pos, key = np.arange(n - m, n)[:, None], np.arange(n)
        seen = torch.from_numpy((key <= pos) & ((key > pos - window) if window else True)).cuda().double()
        kinds = [(torch.einsum("qt,htd->qhd", seen, torch.from_numpy(codes == code).cuda().double()) > 0).repeat_interleave(heads // kv, 1) for code in (0x6F, 0xEF, 0x80)]
        rows = slice(at, at + m)
        special[rows] = kinds[0] | kinds[1] | kinds[2]
        value = torch.where(kinds[2] | (kinds[0] & kinds[1]), math.nan, torch.where(kinds[0], math.inf, -math.inf))
        want[rows] = torch.where(special[rows], value, want[rows])
        at += m
    got = out.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    assert ((got - want).abs()[~special] <= tol[~special]).all()
    assert torch.equal(torch.isfinite(norm), torch.isfinite(lse)) and ((lse.double() - norm).abs() <= tol_lse)[torch.isfinite(norm)].all()
    return special


@pytest.mark.parametrize("counts,small", FORMS)
@pytest.mark.parametrize("dim,dtype", [(64, F16), (128, BF16), (256, BF16)])
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("kinds", [[0x6F], [0xEF, 0x6F], [0x80, 0xEF], [0x6F, 0xEF, 0x80]])
def test_inf_and_nan_among_values_whatever_their_weights(counts, small, dim, dtype, window, kinds):
    """Weights from one that takes all down to none that FP32 could hold; specials in tokens that all queries see, that some see, and that none sees any more."""
    lengths = [70, 333]
    c, q = make(lengths, counts, 8, 2, 32, dim, dtype, seed=dim + window)
    c.fill(0)
    rng = np.random.default_rng(dim + len(kinds))
    for s, n in enumerate(lengths):
        for i in range(24):
            t = int(rng.integers(0, n))
            c.h["v"][c.table[s, t // 32], i % 2, t % 32, int(rng.integers(0, dim // 4))] = rng.choice(kinds)
        t = n - 1
        c.h["v"][c.table[s, t // 32], :, t % 32, dim - 1] = kinds[0]
    c.upload()
    for scale in (4.0, 0.02):
        assert expect_specials(c, q, counts, 8, window, scale, small=small).any()


@pytest.mark.parametrize("small", [False, True])
def test_inf_among_values_of_tokens_of_no_weight(small):
    """Every score is -Inf: zeros, and Inf where a value is."""
    for counts in ([1, 1], [70, 40]):
        c, q = make([70, 333], counts, 8, 2, 32, 64, BF16)
        c.fill(0)
        c.h["k"][:, :, :, 3] = 0xEF
        c.h["v"][c.table[1, 2], :, 5, 7] = 0x6F
        c.upload()
        q[:, :, 3] = 1.0
        out, lse = attend(c, q, counts, 8, small=small)
        assert (lse == -math.inf).all()
        want = torch.zeros_like(out)
        want[counts[0]:, :, 7] = math.inf
        assert torch.equal(out, want)


@pytest.mark.parametrize("kinds", [[0x6F], [0x80], [0x6F, 0xEF, 0x80]])
def test_specials_in_a_long_sequence_that_is_shared_out(kinds):
    """Single tokens over sequences that many groups of warps share: what each part and their sums make of Inf."""
    lengths = [20000, 300, 9000]
    c, q = make(lengths, [1, 1, 2], 8, 1, 128, 128, BF16)
    c.fill(0)
    rng = np.random.default_rng(5)
    for s, n in enumerate(lengths):
        for i in range(40):
            t = int(rng.integers(0, n))
            c.h["v"][c.table[s, t // 128], 0, t % 128, int(rng.integers(0, 40))] = rng.choice(kinds)
    c.upload()
    for scale in (2.0, 0.01):
        assert expect_specials(c, q, [1, 1, 2], 8, 0, scale).any()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,m", [(8, 2, 100), (4, 1, 17), (16, 1, 4)])
def test_the_least_workspace_of_a_chunk(dim, heads, kv_heads, m):
    """A chunk with the workspace of single tokens: the same results as with one for its own bounds, within the tolerance; a byte less is refused."""
    lengths, counts = [300, 45], [m, 3]
    c, q = make(lengths, counts, heads, kv_heads, 32, dim, BF16)
    want, norm, tol, tol_lse = reference(c, q, counts, heads // kv_heads, dim ** -0.5, 1, 0)
    size = H.hif8_cache_attention_workspace_bytes(2, len(q), 1, 300, heads, kv_heads, dim)
    assert size < H.hif8_cache_attention_workspace_bytes(2, len(q), m, 300, heads, kv_heads, dim)
    ws = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 9.0), torch.full((len(q), heads), 9.0, device="cuda")

    def call(size):
        return H.hif8_cache_attention(q, BF16, q.stride(0), q.stride(1), starts(counts), c.d_lengths, 2, len(q), m, 300, *c.args(), heads, dim ** -0.5, 1, 0, out, q.stride(0), q.stride(1), lse,
                                      ws, size, check=False)
    assert call(size - 1) == 8 and (out == 9.0).all()
    assert call(size) == 0 and H.hif8_last_device_status() == 0
    assert ((out.double() - want).abs() <= tol).all() and ((lse.double() - norm).abs() <= tol_lse).all()
    assert (ws[size:] == 0xA5).all()


@pytest.mark.parametrize("dim,heads,kv_heads,seqs,shortest,launches", [(256, 64, 4, 16, 20, 1), (256, 128, 8, 16, 20, 2), (256, 128, 8, 16, 70, 1), (256, 128, 8, 40, 70, 2), (128, 128, 4, 16, 20, 1),
                                                                      (128, 128, 4, 32, 20, 2), (64, 16, 4, 30, 20, 1)])
def test_units_are_taken_whole_where_they_fit_the_blocks(dim, heads, kv_heads, seqs, shortest, launches):
    """Single tokens of several row tiles a key head: one launch where the row tiles of all sequences and key heads fit a round of blocks (heads of 256, more than 64 tokens: four), two otherwise."""
    if torch.cuda.get_device_properties(0).multi_processor_count < 148:
        pytest.skip("fewer blocks than the cases assume")
    lengths = [shortest + i for i in range(seqs)]
    c, q = make(lengths, [1] * seqs, heads, kv_heads, 64, dim, BF16)
    close(c, q, [1] * seqs, heads)
    before = H.hif8_launch_count()
    attend(c, q, [1] * seqs, heads)
    assert H.hif8_launch_count() - before == launches


@pytest.mark.parametrize("counts,small", FORMS)
@pytest.mark.parametrize("dim", [64, 256])
def test_infinite_queries_do_not_see_entries_that_name_no_page(counts, small, dim):
    """Every score of such a query is -Inf: zeros, as if the missing pages were not there."""
    c, q = make([100, 333], counts, 8, 2, 16, dim, BF16)
    c.h["k"][:, :, :, 3] = 0xC8
    c.table[0, 1] = c.table[1, 0] = c.table[1, 7] = -1
    c.upload()
    q[::2, :, 3] = math.inf
    out, lse = attend(c, q, counts, 8, small=small)
    assert (out[::2] == 0).all() and (lse[::2] == -math.inf).all()
    assert (out[1::2] != 0).any(-1).all() and torch.isfinite(lse[1::2]).all()
