"""Attention over the HiF8 key/value cache where factors, weights and values lie at the ends of their ranges.

Each case goes through both kernels: few query rows, and chunks (a workspace without room for tiles takes a chunk through the first).
Tolerances are those of test_gpu_cache_attention, derived there."""
import math

import numpy as np
import pytest
import torch

import paper_2409_16626_b200 as H
from cache_util import VALUES
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
