"""Attention over the HiF8 key/value cache against a plain computation in 64 bits.

Tolerances.  Products of codes are exact in the FP32 sums, so a score differs from the exact one by what its sum rounds: (D + 4) additions of at most 2^-23
of the sum of magnitudes each (the tensor core may truncate), E = (D + 4) 2^-23 scale sum_d |q_d k_d|, the largest over the tokens.  That, the error of the
exponential and of its argument (2^-18 together, arguments below 2^5 in magnitude where weights count), the rounding of a weight to FP16 (2^-11 of it) and the
FP32 sums over n tokens ((n / 16 + 20) 2^-23: sixteen tokens a product) apply to every weight, those of score and sums in numerator and denominator:
  |out - ref| <= eps/2 |ref| + (2^-11 + 2 (E + 2^-18 + (n / 16 + 20) 2^-23)) sum_j p_j |v_j|, eps/2 the half step of the result's type (FP16: and 2^-25)
  |lse - ref| <= E + 2^-18 + (n / 16 + 20) 2^-23 + 2^-22 |ref|
"""
import math

import numpy as np
import pytest
import torch

import paper_2409_16626_b200 as H
from cache_util import TORCH, VALUES, Cache, starts

pytestmark = pytest.mark.gpu
BF16, F16 = H.BF16, H.F16


def reference(c, q, counts, group, scale, causal, window):
    """out, lse, and their tolerances, [queries, heads, (dim)] in 64 bits on the device."""
    n_pages, heads, page, dim = c.shape
    table = torch.from_numpy(VALUES).cuda()
    q = q.double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    tol_out, tol_lse = torch.zeros_like(q), torch.zeros_like(lse)
    half = torch.finfo(TORCH[c.dtype]).eps / 2
    at = 0
    for s, m in enumerate(counts):
        n = max(0, min(c.lengths[s], c.table.shape[1] * page))
        if m and n:
            pages = torch.from_numpy(c.table[s, :-(-n // page)].astype(np.int64)).cuda()
            there = ((pages >= 0) & (pages < n_pages)).repeat_interleave(page)[:n]
            pages = pages.clamp(0, n_pages - 1) * there[::page]
            key, pos = torch.arange(n, device="cuda"), torch.arange(n - m, n, device="cuda")[:, None]
            seen = there.expand(m, n).clone()
            if causal:
                seen &= key <= pos
            if window:
                seen &= key > pos - window
            for h in range(heads):
                def rows(name):
                    e = torch.from_numpy(c.h[name + "_exp"]).cuda()[pages, h].double().clamp(-H.CACHE_EXP_MAX, H.CACHE_EXP_MAX)
                    return table[torch.from_numpy(c.h[name]).cuda()[pages, h].reshape(-1, dim)[:n].long()] * torch.pow(2.0, -e).repeat_interleave(page)[:n, None]
                k, v = rows("k"), rows("v")
                for r in range(h * group, (h + 1) * group):
                    x = scale * (q[at:at + m, r] @ k.T)
                    x = torch.where(seen, x, -math.inf)
                    top = x.amax(1, keepdim=True)
                    top = torch.where(top == -math.inf, 0.0, top)
                    p = torch.exp(x - top)
                    total = p.sum(1, keepdim=True)
                    w = torch.where(total == 0, 0.0, p / total)
                    # a token that is not seen takes no part, whatever its value is
                    bad = ~torch.isfinite(v)
                    o = w @ torch.where(bad, 0.0, v)
                    if bad.any():
                        for j, d in bad.nonzero().tolist():
                            o[:, d] = torch.where(seen[:, j], o[:, d] + w[:, j] * v[j, d], o[:, d])
                    out[at:at + m, r] = o
                    lse[at:at + m, r] = torch.where(total == 0, -math.inf, top + total.log())[:, 0]
                    e = ((dim + 4) * 2.0 ** -23 * scale * (q[at:at + m, r].abs() @ torch.where(torch.isfinite(k), k.abs(), 0.0).T) * seen).amax(1, keepdim=True)
                    e = e + 2.0 ** -18 + (n / 16 + 20) * 2.0 ** -23
                    tol_out[at:at + m, r] = half * o.abs() + (2.0 ** -11 + 2 * e) * (w @ torch.where(bad, 0.0, v.abs())) + (2.0 ** -25 if c.dtype == F16 else 0)
                    tol_lse[at:at + m, r] = e[:, 0] + 2.0 ** -22 * lse[at:at + m, r].abs()
        at += m
    return out, lse, tol_out, tol_lse


def attend(c, q, counts, heads, causal=1, window=0, scale=None, out=None, lse=True, stream=None, max_q=None, small=False):
    n = q.shape[0]
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out = torch.full_like(q, 9.0) if out is None else out
    lse = torch.full((n, heads), 9.0, device="cuda") if lse else None
    max_q = max(counts, default=0) if max_q is None else max_q
    longest = max(c.lengths, default=0)
    group = heads // c.shape[1]
    # (small: the least that the call takes, without room for expanded tiles: as much as for fewer than 64 rows of a key head)
    size = H.hif8_cache_attention_workspace_bytes(len(counts), n, min(max_q, 63 // group) if small else max_q, longest, heads, c.shape[1], c.shape[3])
    ws = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    H.hif8_cache_attention(q, c.dtype, q.stride(0), q.stride(1), starts(counts), c.d_lengths, len(counts), n, max_q, longest, *c.args(), heads, scale, causal, window,
                           out, out.stride(0), out.stride(1), lse, ws, size, stream)
    assert H.hif8_last_device_status(stream) == 0
    assert (ws[size:] == 0xA5).all(), "write behind the workspace"
    return out, lse


def make(lengths, counts, heads, kv_heads, page, dim, dtype, seed=0, extra_pages=3, **kw):
    c = Cache(sum(-(-max(0, n) // page) for n in lengths) + extra_pages, kv_heads, page, dim, lengths, [0] * len(lengths), seed=seed, **kw)
    c.dtype = dtype
    c.fill()
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(sum(counts), heads, dim, generator=g) * torch.exp2(torch.randint(-2, 2, (sum(counts), heads, 1), generator=g).float())
    return c, q.to(TORCH[dtype]).cuda()


def close(c, q, counts, heads, causal=1, window=0, scale=None, **kw):
    out, lse = attend(c, q, counts, heads, causal, window, scale, **kw)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    want, norm, tol, tol_lse = reference(c, q, counts, heads // c.shape[1], scale, causal, window)
    got = out.double()
    finite = torch.isfinite(want)
    assert torch.equal(finite, torch.isfinite(got)) and torch.equal(torch.isnan(want), torch.isnan(got))
    assert torch.equal(want[~finite & ~torch.isnan(want)], got[~finite & ~torch.isnan(want)])
    err = torch.where(finite, (got - torch.where(finite, want, 0.0)).abs() - tol, -1.0)
    assert (err <= 0).all(), (float(err.max()), err.argmax())
    if lse is not None:
        same = torch.isfinite(norm)
        assert torch.equal(same, torch.isfinite(lse)) and (lse[~same & ~torch.isnan(norm)] == norm[~same & ~torch.isnan(norm)]).all()
        assert ((lse.double() - norm).abs()[same] <= tol_lse[same]).all()
    return out, lse


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,page", [(64, 16), (64, 128), (128, 32), (128, 64), (256, 16), (256, 128)])
@pytest.mark.parametrize("lengths", [[1], [517], [0, 1, 16, 63, 64, 65, 200], [3000, 5]])
def test_single_tokens(lengths, dim, page, dtype):
    c, q = make(lengths, [1] * len(lengths), 8, 2, page, dim, dtype, seed=dim + page)
    close(c, q, [1] * len(lengths), 8)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (8, 4), (10, 2), (21, 3), (16, 1), (17, 1), (64, 1), (40, 8)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_head_layouts(heads, kv_heads, dim):
    c, q = make([130, 77, 1000], [1, 1, 1], heads, kv_heads, 64, dim, BF16, seed=heads)
    close(c, q, [1, 1, 1], heads)


@pytest.mark.parametrize("counts", [[2, 1, 3], [4, 0, 4], [5, 7, 1], [0, 0, 9], [33, 64, 20]])
@pytest.mark.parametrize("causal,window", [(1, 0), (0, 0), (1, 1), (1, 5), (1, 64), (0, 100), (1, 1000)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (8, 2, 128), (5, 1, 256)])
def test_several_queries(counts, causal, window, heads, kv_heads, dim):
    lengths = [120, 64, 513]
    c, q = make(lengths, counts, heads, kv_heads, 32, dim, F16 if window else BF16, seed=sum(counts) + window)
    close(c, q, counts, heads, causal, window)


@pytest.mark.parametrize("lengths,counts", [([300], [128]), ([129, 64, 1], [129, 64, 1]), ([3000, 0, 700, 40], [300, 0, 700, 33]), ([5000, 260], [65, 260]), ([50, 20], [70, 90])])
@pytest.mark.parametrize("causal,window", [(1, 0), (0, 0), (1, 200), (1, 3), (0, 129)])
@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(8, 2, 128, BF16), (3, 3, 64, F16), (7, 1, 64, BF16), (5, 5, 128, F16), (4, 2, 256, BF16), (7, 1, 256, F16)])
def test_chunks(lengths, counts, causal, window, heads, kv_heads, dim, dtype):
    c, q = make(lengths, counts, heads, kv_heads, 16 if window else 128, dim, dtype, seed=len(lengths) + window)
    close(c, q, counts, heads, causal, window)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_chunks_without_room_for_tiles(dim):
    c, q = make([700, 90], [100, 90], 8, 2, 64, dim, BF16)
    close(c, q, [100, 90], 8)
    close(c, q, [100, 90], 8, small=True)


def test_chunks_of_a_large_head():
    c, q = make([400, 33], [70, 33], 4, 2, 32, 256, BF16)
    close(c, q, [70, 33], 4)


def test_many_short_prompts():
    counts = [(i * 31) % 90 for i in range(60)]
    c, q = make([n + (i % 3) * 40 for i, n in enumerate(counts)], counts, 8, 4, 32, 64, BF16)
    close(c, q, counts, 8)


def test_rows_that_see_nothing():
    # an empty cache, more queries than tokens, and a window that has moved past pages which were given up
    c, q = make([0, 3, 100], [2, 6, 4], 4, 2, 16, 64, BF16)
    out, lse = close(c, q, [2, 6, 4], 4)
    assert (out[:5] == 0).all() and (lse[:5] == -math.inf).all()
    c.table[2, :5] = -1
    c.upload()
    close(c, q, [2, 6, 4], 4, 1, 8)
    c.table[2, :] = -1
    c.upload()
    out, lse = close(c, q, [2, 6, 4], 4)
    assert (out[8:] == 0).all() and (lse[8:] == -math.inf).all()


def test_entries_that_name_no_page_are_not_seen():
    c, q = make([300, 300], [1, 3], 8, 2, 32, 128, BF16)
    c.table[0, 3], c.table[1, 0], c.table[1, 9] = -1, c.shape[0], 2 ** 31 - 1
    c.upload()
    close(c, q, [1, 3], 8)


def test_a_length_beyond_the_row_is_cut():
    c, q = make([64, 40], [1, 2], 4, 2, 16, 64, F16)
    c.table = c.table[:, :4].copy()
    c.lengths = [10 ** 9, 40]
    c.upload()
    close(c, q, [1, 2], 4)


@pytest.mark.parametrize("counts", [[1, 1], [6, 3], [40, 200]])
@pytest.mark.parametrize("causal,window", [(1, 0), (1, 20), (0, 0)])
@pytest.mark.parametrize("small", [False, True])
def test_inf_and_nan_where_they_are_not_seen(counts, causal, window, small):
    """Stale slots behind the length, tokens before the window, and a later query's tokens hold Inf and NaN in K and V; those that a query sees propagate."""
    lengths = [250, 333]
    c, q = make(lengths, counts, 8, 2, 16, 64, BF16, seed=5)
    c.fill(0)  # (weights that do not vanish: what Inf times a weight below the FP16 range gives is another question)
    specials = [0x80, 0x6F, 0xEF]
    rng = np.random.default_rng(1)
    for s, n in enumerate(lengths):
        last = c.table[s, (n - 1) // 16]
        c.h["v"][last, :, (n - 1) % 16 + 1:] = rng.choice(specials, size=c.h["v"][last, :, (n - 1) % 16 + 1:].shape)
        c.h["k"][last, :, (n - 1) % 16 + 1:] = 0x80
        for name, toks in (("v", [n - 1, n - 2, n - counts[s] + 1, n - 21, 40]), ("k", [n - 3, n - 30])):
            for t in toks:
                if t < n:
                    c.h[name][c.table[s, t // 16], t % 2, t % 16, t % 64] = specials[t % 3]
    for p in set(range(c.shape[0] + 1)) - set(c.table[c.table >= 0].tolist()):
        c.h["v"][p] = 0x80
    c.upload()
    close(c, q, counts, 8, causal, window, small=small)


@pytest.mark.parametrize("small", [False, True])
def test_a_later_query_s_values_are_all_special(small):
    """Every value of the last tokens is Inf or NaN: the queries in front of them keep their results."""
    c, q = make([400], [120], 4, 2, 16, 64, F16)
    c.fill(0)
    clean = attend(c, q, [120], 4, small=small)[0]
    rng = np.random.default_rng(3)
    for t in range(330, 400):
        c.h["v"][c.table[0, t // 16], :, t % 16] = rng.choice([0x80, 0x6F, 0xEF], size=(2, 64))
    c.upload()
    out, _ = close(c, q, [120], 4, small=small)
    assert torch.equal(out[:50], clean[:50]) and not torch.isfinite(out[50:]).any()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 90, 7])
@pytest.mark.parametrize("small", [False, True])
def test_scattered_special_values(dim, window, small):
    """Inf, -Inf and NaN, of several kinds in some elements, all over the tokens that only some queries see; and nearly everywhere."""
    counts, lengths = [500, 70], [600, 71]
    c, q = make(lengths, counts, 4, 2, 32, dim, BF16)
    c.fill(0)
    rng = np.random.default_rng(dim + window)
    for s, n in enumerate(lengths):
        for i in range(60):
            t = int(rng.integers(0, n))
            c.h["v"][c.table[s, t // 32], i % 2, t % 32, int(rng.integers(0, dim)) // 5 * 5] = rng.choice([0x80, 0x6F, 0xEF])
    c.upload()
    close(c, q, counts, 4, 1, window, small=small, scale=0.02)
    c.h["v"][:] = 0x80
    c.upload()
    out, _ = attend(c, q, counts, 4, 1, window, small=small)
    assert torch.isnan(out).all()


@pytest.mark.parametrize("counts", [[1, 2], [1, 40]])
def test_scores_and_spreads_at_the_ends(counts):
    """Large scores (one token takes all), queries and blocks of very different magnitudes, exponents beyond the limit."""
    c, q = make([400, 90], counts, 8, 2, 16, 128, BF16, seed=3)
    n = sum(counts)
    q = (q.float() * torch.exp2((torch.arange(n * 8) % 24).view(n, 8, 1).cuda().float() * 2 - 20)).bfloat16()
    close(c, q, counts, 8, scale=0.5)
    rng = np.random.default_rng(2)
    c.h["k_exp"] = rng.integers(-12, 13, size=c.h["k_exp"].shape).astype(np.int32)
    c.h["v_exp"] = rng.integers(-60, 61, size=c.h["v_exp"].shape).astype(np.int32)
    c.upload()
    _, q = make([400, 90], counts, 8, 2, 16, 128, BF16, seed=3)
    close(c, q, counts, 8, scale=0.01)
    zero = torch.zeros_like(q)
    close(c, zero, counts, 8)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("n", [2, 50])
def test_inf_and_nan_queries_stay_in_their_rows(bad, n):
    c, q = make([100], [n], 4, 2, 16, 64, BF16)
    q[0, 1, 3] = bad
    out, lse = attend(c, q, [n], 4)
    clean, _ = attend(c, torch.where(torch.isfinite(q), q, 0.0), [n], 4)
    keep = torch.ones(n, 4, dtype=torch.bool)
    keep[0, 1] = False
    assert torch.isnan(out[0, 1]).all() and torch.equal(out[keep], clean[keep])


@pytest.mark.parametrize("layout", ["fused", "heads_first", "odd"])
@pytest.mark.parametrize("counts", [[1, 1], [3, 70]])
def test_strides(layout, counts):
    heads, dim, n = 6, 64, sum(counts)
    c, q0 = make([50, 141], counts, heads, 2, 16, dim, BF16)
    if layout == "fused":
        big = torch.full((2, n, heads + 4, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        q, out = big[0, :, :heads], big[1, :, :heads]
    elif layout == "heads_first":
        big = torch.full((2, heads, n, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        q, out = big[0].transpose(0, 1), big[1].transpose(0, 1)
    else:
        big = torch.full((2 * n * heads * (dim + 3) + 1,), 7.0, dtype=torch.bfloat16, device="cuda")
        q, out = big[1:1 + n * heads * (dim + 3)].view(n, heads, dim + 3)[..., :dim], big[1 + n * heads * (dim + 3):].view(n, heads, dim + 3)[..., :dim]
    q.copy_(q0)
    plain, _ = attend(c, q0, counts, heads)
    before = big.clone()
    close(c, q, counts, heads, out=out)
    assert torch.equal(out, plain)
    out.fill_(7.0)
    assert torch.equal(big, before)


def test_queries_behind_the_last_sequence_stay():
    c, q = make([50, 141], [1, 2], 4, 2, 16, 64, BF16)
    more = torch.cat([q, q])
    out = torch.full_like(more, 5.0)
    attend(c, more, [1, 2], 4, out=out)
    assert (out[3:] == 5.0).all() and torch.equal(out[:3], attend(c, q, [1, 2], 4)[0])


def test_wrong_bounds_and_starts_stay_inside():
    """Counts beyond max_q, starts out of order or of range: answers for what there is, nothing written elsewhere."""
    c, q = make([50, 141, 30], [3, 2, 4], 4, 2, 16, 64, BF16)
    close(c, q, [3, 2, 4], 4, max_q=1)
    n, size = 9, H.hif8_cache_attention_workspace_bytes(3, 9, 4, 141, 4, 2, 64)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for start in ([0, 7, 3, 9], [-5, 3, 5, 10 ** 9], [9, 9, 9, 9]):
        out = torch.full((n + 2, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        H.hif8_cache_attention(q, BF16, 256, 64, torch.tensor(start, dtype=torch.int32, device="cuda"), c.d_lengths, 3, n, 4, 141, *c.args(), 4, 0.1, 1, 0, out[1:], 256, 64,
                               None, ws, size)
        assert H.hif8_last_device_status() == 0 and (out[0] == 5.0).all() and (out[n + 1] == 5.0).all()


def test_wrong_starts_of_chunks_stay_inside():
    c, q = make([200, 141, 300], [40, 20, 60], 4, 1, 16, 64, BF16)
    n = 120
    for longest in (300, 90):  # the second: lengths beyond what the host was told
        size = H.hif8_cache_attention_workspace_bytes(3, n, 60, longest, 4, 1, 64)
        ws = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        for start in ([0, 70, 30, 120], [-5, 3, 50, 10 ** 9], [120, 120, 120, 120], [0, 120, 0, 120], [119, 0, 3, 120]):
            out = torch.full((n + 2, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
            lse = torch.full((n + 2, 4), 5.0, device="cuda")
            H.hif8_cache_attention(q, BF16, 256, 64, torch.tensor(start, dtype=torch.int32, device="cuda"), c.d_lengths, 3, n, 60, longest, *c.args(), 4, 0.1, 1, 0, out[1:], 256, 64,
                                   lse[1:], ws, size)
            assert H.hif8_last_device_status() == 0 and (out[0] == 5.0).all() and (out[n + 1] == 5.0).all() and (lse[0] == 5.0).all() and (lse[n + 1] == 5.0).all()
            assert (ws[size:] == 0xA5).all()


@pytest.mark.parametrize("counts", [[1, 1], [30, 40]])
@pytest.mark.parametrize("causal", [0, 1])
def test_the_largest_windows_are_none(counts, causal):
    c, q = make([20, 141], counts, 4, 2, 16, 64, BF16)
    want = attend(c, q, counts, 4, causal)
    for window in (2 ** 31 - 1, 2 ** 30, 200):
        got = attend(c, q, counts, 4, causal, window)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("counts", [[1], [3], [40]])
def test_a_pool_beyond_four_gigabytes(counts):
    """The same sequence in a small pool and at the end of one of more than 2^32 bytes."""
    c, q = make([300], counts, 8, 4, 128, 256, BF16)
    want = attend(c, q, counts, 8)
    n_pages = (1 << 32) // (4 * 128 * 256) + 8
    big = {}
    for name in ("k", "v", "k_exp", "v_exp"):
        big[name] = torch.zeros((n_pages,) + c.d[name].shape[1:], dtype=c.d[name].dtype, device="cuda")
        big[name][-c.shape[0]:] = c.d[name][:c.shape[0]]
    c.d, c.d_table, c.shape = big, torch.where(c.d_table >= 0, c.d_table + (n_pages - c.shape[0]), -1).int(), (n_pages,) + c.shape[1:]
    got = attend(c, q, counts, 8)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_calls_at_once_on_two_streams():
    """Each with a workspace of its own; single tokens, and chunks."""
    for counts in ([1, 1, 1], [50, 3, 90]):
        c, q = make([700, 3000, 99], counts, 8, 2, 32, 128, BF16)
        want = attend(c, q, counts, 8)
        torch.cuda.synchronize()
        streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
        size = H.hif8_cache_attention_workspace_bytes(3, len(q), max(counts), 3000, 8, 2, 128)
        ws, st = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)], starts(counts)
        torch.cuda.synchronize()
        for _ in range(20):
            for i, stream in enumerate(streams):
                out, lse = torch.empty_like(q), torch.empty(len(q), 8, device="cuda")
                H.hif8_cache_attention(q, BF16, q.stride(0), q.stride(1), st, c.d_lengths, 3, len(q), max(counts), 3000, *c.args(), 8, 128 ** -0.5, 1, 0, out, q.stride(0), q.stride(1), lse,
                                       ws[i], size, stream)
                got[i].append((out, lse))
        torch.cuda.synchronize()
        for out, lse in got[0] + got[1]:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_many_sequences_and_shared_pages():
    lengths = [(i * 37) % 150 for i in range(700)]
    lengths[0] = lengths[-1] = 130
    c, q = make(lengths, [1] * 700, 4, 1, 16, 64, BF16, share=[(0, 699)])
    close(c, q, [1] * 700, 4)


def test_long_sequences_are_shared_out_and_reproducible():
    c, q = make([70000, 9000, 31], [1, 2, 1], 8, 1, 128, 64, BF16)
    first = close(c, q, [1, 2, 1], 8)
    for _ in range(3):
        again = attend(c, q, [1, 2, 1], 8)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("counts", [[1, 4], [20, 77]])
def test_another_stream_and_a_captured_graph(counts):
    c, q = make([500, 77], counts, 8, 2, 32, 128, BF16)
    n, most = sum(counts), max(counts)
    want, norm = attend(c, q, counts, 8)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out, lse = attend(c, q, counts, 8, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, norm)
    size = H.hif8_cache_attention_workspace_bytes(2, n, most, 500, 8, 2, 128)
    ws, st = torch.empty(size, dtype=torch.uint8, device="cuda"), starts(counts)
    out.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.hif8_cache_attention(q, BF16, q.stride(0), q.stride(1), st, c.d_lengths, 2, n, most, 500, *c.args(), 8, 128 ** -0.5, 1, 0, out, q.stride(0), q.stride(1), lse, ws, size)
    q.neg_()
    want = attend(c, q, counts, 8)[0]
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_without_lse():
    c, q = make([500], [1], 8, 2, 32, 128, BF16)
    assert torch.equal(attend(c, q, [1], 8)[0], attend(c, q, [1], 8, lse=False)[0])


def test_serving_steps_together():
    """A prompt, forked into three samples that each append and attend two more tokens, one freed, the pool compacted: attention gives what the same tokens
    in a cache of their own give."""
    heads, kv, page, dim = 8, 2, 16, 64
    g = torch.Generator().manual_seed(7)
    tok = lambda n, h: torch.randn(n, h, dim, generator=g).bfloat16().cuda()  # noqa: E731
    n_pages, width, prompt = 40, 8, 37
    pool = [torch.randint(0, 256, (n_pages, kv, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.zeros(n_pages, kv, dtype=torch.int32, device="cuda") for _ in range(2)]
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, :3] = ints(31, 5, 18)
    args = lambda t: (*pool, n_pages, kv, page, dim, t, t.stride(0))  # noqa: E731
    k, v = tok(prompt, kv), tok(prompt, kv)
    H.hif8_cache_append(k, v, BF16, kv * dim, dim, ints(0, prompt), ints(0), 1, prompt, *args(table))
    three, lengths = torch.empty(3, width, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    H.hif8_cache_fork(*args(table), ints(prompt), 1, ints(0, 0, 0), ints(-1, 33, 2), 3, three, width, lengths)
    steps = [(tok(3, kv), tok(3, kv)) for _ in range(14)]
    spare = [9, 10, 11]
    for i, (nk, nv) in enumerate(steps):
        if (prompt + i) % page == 0:
            three[:, (prompt + i) // page] = ints(*spare)
        H.hif8_cache_append(nk, nv, BF16, kv * dim, dim, ints(0, 1, 2, 3), lengths, 3, 3, *args(three))
        lengths += 1
    lengths[1] = 0  # the second sample ends
    live, free = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(n_pages, dtype=torch.int32, device="cuda")
    ws = torch.empty(H.hif8_cache_compact_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda")
    H.hif8_cache_compact(*args(three), lengths, 3, 1, live, free, ws, ws.numel())
    assert int(live) == 6 and int(three[[0, 2]].max()) == 5  # two shared pages, and two of each sample's own
    q = tok(2, heads)
    size = H.hif8_cache_attention_workspace_bytes(3, 2, 1, 51, heads, kv, dim)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(2, heads, device="cuda")
    H.hif8_cache_attention(q, BF16, heads * dim, dim, ints(0, 1, 1, 2), lengths, 3, 2, 1, 51, *args(three), heads, 0.125, 1, 0, out, heads * dim, dim, lse, ws, size)
    for row, s in ((0, 0), (1, 2)):
        n = prompt + len(steps)
        c = Cache(8, kv, page, dim, [0], [n], seed=s)
        c.dtype = BF16
        c.append(k, v, BF16, [prompt])
        c.lengths = [prompt]
        for nk, nv in steps:
            c.append(nk[s:s + 1], nv[s:s + 1], BF16, [1])
            c.lengths[0] += 1
        c.upload()
        want, norm = attend(c, q[row:row + 1], [1], heads, scale=0.125)
        assert torch.equal(out[row:row + 1], want) and torch.equal(lse[row:row + 1], norm)


@pytest.mark.parametrize("counts", [1, 9])
def test_as_many_sequences_as_a_call_takes(counts):
    """2048 of them: single tokens, and with 16 heads to a key head as chunks."""
    lengths = [(i * 29) % 47 for i in range(H.CACHE_MAX_SEQS)]
    group = 1 if counts == 1 else 16
    q_counts = [counts if i % 3 else 0 for i in range(H.CACHE_MAX_SEQS)]
    c, q = make(lengths, q_counts, group, 1, 16, 64, BF16)
    out, lse = attend(c, q, q_counts, group)
    pick = list(range(0, 40)) + list(range(H.CACHE_MAX_SEQS - 40, H.CACHE_MAX_SEQS))
    at = np.concatenate([[0], np.cumsum(q_counts)])
    rows = torch.from_numpy(np.concatenate([np.arange(at[s], at[s + 1]) for s in pick])).cuda()
    few = Cache(1, 1, 16, 64, [0], [0], seed=0)
    few.dtype, few.shape, few.h, few.lengths, few.table = BF16, c.shape, c.h, [lengths[s] for s in pick], c.table[pick]
    want, norm, tol, tol_lse = reference(few, q[rows], [q_counts[s] for s in pick], group, 64 ** -0.5, 1, 0)
    assert ((out[rows].double() - want).abs() <= tol).all()
    same = torch.isfinite(norm)
    assert torch.equal(same, torch.isfinite(lse[rows])) and ((lse[rows].double() - norm).abs()[same] <= tol_lse[same]).all()


@pytest.mark.parametrize("m", [1, 40])
def test_a_captured_step_follows_its_inputs(m):
    """Append, attention, fork, append for the children and compaction in one graph, replayed with other tokens, lengths and parents: what the calls one by one give."""
    heads, kv, page, dim, width, n_pages = 8, 2, 32, 128, 8, 40
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    size = H.hif8_cache_attention_workspace_bytes(2, 2 * m, m, width * page, heads, kv, dim)
    compact_size = H.hif8_cache_compact_workspace_bytes(n_pages)

    def fresh():
        s = {name: torch.full(shape, 5, dtype=t, device="cuda") for name, shape, t in (
            ("q", (2 * m, heads, dim), torch.bfloat16), ("k", (2 * m, kv, dim), torch.bfloat16), ("v", (2 * m, kv, dim), torch.bfloat16), ("out", (2 * m, heads, dim), torch.bfloat16),
            ("lse", (2 * m, heads), torch.float32), ("kp", (n_pages, kv, page, dim), torch.uint8), ("vp", (n_pages, kv, page, dim), torch.uint8), ("ke", (n_pages, kv), torch.int32),
            ("ve", (n_pages, kv), torch.int32), ("table", (2, width), torch.int32), ("lengths", (2,), torch.int32), ("after", (2,), torch.int32), ("parent", (3,), torch.int32),
            ("new", (3,), torch.int32), ("children", (3, width), torch.int32), ("child_lengths", (3,), torch.int32), ("live", (1,), torch.int32), ("free", (n_pages,), torch.int32),
            ("ws", (size,), torch.uint8), ("ws2", (compact_size,), torch.uint8))}
        s["start"], s["one"] = ints([0, m, 2 * m]), ints([0, 1, 1, 2])
        return s

    def fill(s, seed):
        g = torch.Generator().manual_seed(seed)
        for name in ("q", "k", "v"):
            s[name].copy_(torch.randn(s[name].shape, generator=g))
        for name in ("kp", "vp"):
            s[name].copy_(torch.randint(0, 0x60, s[name].shape, generator=g))
        lengths = [int(x) for x in torch.randint(0, width * page - m - 1, (2,), generator=g)]
        s["ke"].zero_(), s["ve"].zero_()
        s["table"].copy_(torch.from_numpy(np.random.default_rng(seed).permutation(n_pages)[:2 * width].reshape(2, width)))
        s["lengths"].copy_(ints(lengths)), s["after"].copy_(ints([x + m for x in lengths]))
        s["parent"].copy_(ints([seed % 2, 1, 0]))
        s["new"].copy_(torch.from_numpy(np.setdiff1d(np.arange(n_pages), s["table"].cpu().numpy())[:3]))

    def step(s):
        pool = lambda t: (s["kp"], s["vp"], s["ke"], s["ve"], n_pages, kv, page, dim, t, width)  # noqa: E731
        H.hif8_cache_append(s["k"], s["v"], BF16, kv * dim, dim, s["start"], s["lengths"], 2, 2 * m, *pool(s["table"]))
        H.hif8_cache_attention(s["q"], BF16, heads * dim, dim, s["start"], s["after"], 2, 2 * m, m, width * page, *pool(s["table"]), heads, 0.1, 1, 50, s["out"], heads * dim, dim, s["lse"],
                               s["ws"], size)
        H.hif8_cache_fork(*pool(s["table"]), s["after"], 2, s["parent"], s["new"], 3, s["children"], width, s["child_lengths"])
        H.hif8_cache_append(s["k"], s["v"], BF16, kv * dim, dim, s["one"], s["child_lengths"], 3, 2 * m, *pool(s["children"]))
        H.hif8_cache_compact(*pool(s["children"]), s["child_lengths"], 3, 1, s["live"], s["free"], s["ws2"], compact_size)

    captured, plain = fresh(), fresh()
    fill(captured, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for seed in (2, 3, 4):
        fill(captured, seed), fill(plain, seed)
        graph.replay()
        step(plain)
        torch.cuda.synchronize()
        for name in captured:
            if name not in ("ws", "ws2"):
                assert torch.equal(captured[name], plain[name]), (seed, name)
        assert int(captured["live"]) > 0
