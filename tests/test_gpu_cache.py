"""The key/value cache: append, read, fork and compact against the oracle and a model of the pages in numpy.  Codes, exponents, tables
and untouched bytes are compared exactly."""
import numpy as np
import pytest
import torch

import paper_2409_16626_b200 as H
from oracle import hif8_oracle as O

from cache_util import TORCH, Cache, bits_of, starts

pytestmark = pytest.mark.gpu
DTYPES = [H.F32, H.BF16, H.F16]


def new_tokens(n, heads, dim, dtype, seed, specials=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2, n, heads, dim, generator=g) * torch.exp2(torch.randint(-12, 8, (2, n, heads, 1), generator=g).float())
    if specials and n > 2:
        x[0, 1, 0, 3], x[1, 2, 0, 5], x[0, 0, :, 7], x[1, n - 1] = float("inf"), float("nan"), -float("inf"), 0.0
    x = x.to(TORCH[dtype]).cuda()
    return x[0], x[1]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,dim,heads", [(16, 64, 1), (32, 128, 3), (64, 128, 2), (128, 256, 2), (64, 64, 5)])
@pytest.mark.parametrize("lengths,counts", [([0], [1]), ([5, 0, 64, 127], [1, 1, 1, 1]), ([0, 3, 16, 200, 31], [300, 0, 17, 64, 1]), ([7, 130], [2, 9])])
def test_append_and_read(lengths, counts, page, dim, heads, dtype):
    room = [c for c in counts]
    n_pages = sum(-(-(n + r) // page) for n, r in zip(lengths, room)) + 3
    c = Cache(n_pages, heads, page, dim, lengths, room, seed=page + dim)
    k, v = new_tokens(sum(counts), heads, dim, dtype, seed=sum(counts), specials=True)
    start = starts(counts)
    H.hif8_cache_append(k, v, dtype, k.stride(0), k.stride(1), start, c.d_lengths, len(counts), len(k), *c.args())
    c.append(k, v, dtype, counts)
    c.same()
    # read back: the new tokens, as values rounded to the type
    first = list(lengths)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    H.hif8_cache_read(*c.args(), torch.tensor(first, dtype=torch.int32, device="cuda"), start, len(counts), len(k), ko, vo, dtype, ko.stride(0), ko.stride(1))
    torch.cuda.synchronize()
    for name, got in (("k", ko), ("v", vo)):
        at = 0
        for s, m in enumerate(counts):
            want, there = c.values(s, lengths[s] + m, name)
            want = torch.from_numpy(want[lengths[s]:]).to(TORCH[dtype])
            g = got[at:at + m].cpu()
            assert there[lengths[s]:].all()
            assert torch.equal(torch.isnan(g), torch.isnan(want)) and torch.equal(torch.nan_to_num(g, nan=0.0), torch.nan_to_num(want, nan=0.0)), (name, s)
            at += m


@pytest.mark.parametrize("rnd", [H.RND_TA, H.RND_HR, H.RND_SSR, H.RND_TE])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("flags", [0, H.FLAG_SATURATE | H.FLAG_NAN_TO_ZERO])
def test_append_rounding_methods_and_options(rnd, dtype, flags):
    for counts, lengths in (([70, 40], [0, 9]), ([1, 1], [3, 32])):
        c = Cache(8, 2, 32, 64, lengths, counts, seed=rnd)
        k, v = new_tokens(sum(counts), 2, 64, dtype, seed=9, specials=True)
        H.hif8_cache_append(k, v, dtype, k.stride(0), k.stride(1), starts(counts), c.d_lengths, 2, len(k), *c.args(), 14, rnd, flags)
        c.append(k, v, dtype, counts, 14, rnd, flags)
        c.same()


def test_append_extreme_exponents_are_clamped():
    c = Cache(4, 1, 16, 64, [0], [48], seed=1)
    x = torch.randn(48, 1, 64)
    x[:16] *= 2.0 ** -90
    x[16:32] *= 2.0 ** 80
    x[32:] = 0.0
    x = x.cuda()
    H.hif8_cache_append(x, x, H.F32, 64, 64, starts([48]), c.d_lengths, 1, 48, *c.args())
    c.append(x, x, H.F32, [48])
    c.same()
    assert {48, -48, 0} <= set(c.h["k_exp"].ravel().tolist())


def test_read_takes_exponents_within_the_limits():
    c = Cache(4, 2, 16, 64, [60], [0], seed=1)
    c.fill()
    want = {}
    for limit in (H.CACHE_EXP_MAX, 100):
        for name in ("k_exp", "v_exp"):
            c.h[name][:, 0], c.h[name][:, 1] = limit, -limit
        c.upload()
        k, v = torch.empty(60, 2, 64, device="cuda"), torch.empty(60, 2, 64, device="cuda")
        H.hif8_cache_read(*c.args(), torch.zeros(1, dtype=torch.int32, device="cuda"), starts([60]), 1, 60, k, v, H.F32, 128, 64)
        want[limit] = torch.stack([k, v])
    assert torch.equal(want[100], want[H.CACHE_EXP_MAX]) and torch.isfinite(want[100]).all() and (want[100][:, :, 1].abs().amax() > 2.0 ** 40)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["fused", "heads_first", "odd"])
def test_append_and_read_strides(dtype, layout):
    heads, dim, counts, lengths = 3, 128, [37, 5], [10, 0]
    n = sum(counts)
    c = Cache(8, heads, 16, dim, lengths, counts, seed=4)
    k0, v0 = new_tokens(n, heads, dim, dtype, seed=5)
    if layout == "fused":  # slices of one projection's output
        big = torch.zeros(n, 4 * heads + 2 * heads, dim, dtype=TORCH[dtype], device="cuda")
        k, v = big[:, 4 * heads:5 * heads], big[:, 5 * heads:]
    elif layout == "heads_first":
        big = torch.zeros(2, heads, n, dim, dtype=TORCH[dtype], device="cuda")
        k, v = big[0].transpose(0, 1), big[1].transpose(0, 1)
    else:  # neither pointers nor strides on 16 bytes
        big = torch.zeros(2 * n * heads * (dim + 3) + 1, dtype=TORCH[dtype], device="cuda")
        k = big[1:1 + n * heads * (dim + 3)].view(n, heads, dim + 3)[..., :dim]
        v = big[1 + n * heads * (dim + 3):].view(n, heads, dim + 3)[..., :dim]
    k.copy_(k0)
    v.copy_(v0)
    H.hif8_cache_append(k, v, dtype, k.stride(0), k.stride(1), starts(counts), c.d_lengths, 2, n, *c.args())
    c.append(k0, v0, dtype, counts)
    c.same()
    before = big.clone()
    k.zero_(), v.zero_()
    zeroed = big.clone()
    H.hif8_cache_read(*c.args(), c.d_lengths, starts(counts), 2, n, k, v, dtype, k.stride(0), k.stride(1))
    back = [torch.from_numpy(np.concatenate([c.values(s, lengths[s] + counts[s], name)[0][lengths[s]:] for s in range(2)])).to(TORCH[dtype]).cuda() for name in ("k", "v")]
    assert torch.equal(k, back[0]) and torch.equal(v, back[1])
    k.copy_(k0), v.copy_(v0)
    assert torch.equal(big, before) and not torch.equal(zeroed, before)  # nothing beside the rows was written


def test_entries_that_name_no_page():
    """Tokens of such an entry are not written and read as zeros; a length beyond the row is cut."""
    c = Cache(9, 2, 16, 64, [20, 3], [30, 30], seed=8)
    c.table[0, 2] = -1
    c.table[1, 0] = 9  # one behind the last
    c.table[1, 1] = 0x7FFFFFFF
    c.upload()
    k, v = new_tokens(60, 2, 64, H.BF16, seed=2)
    H.hif8_cache_append(k, v, H.BF16, 128, 64, starts([30, 30]), c.d_lengths, 2, 60, *c.args())
    c.append(k, v, H.BF16, [30, 30])
    c.same()
    ko, vo = torch.full((60, 2, 64), 5.0, device="cuda"), torch.full((60, 2, 64), 5.0, device="cuda")
    H.hif8_cache_read(*c.args(), c.d_lengths, starts([30, 30]), 2, 60, ko, vo, H.F32, 128, 64)
    for name, got in (("k", ko), ("v", vo)):
        want = np.concatenate([c.values(s, c.lengths[s] + 30, name)[0][c.lengths[s]:] for s in range(2)])
        assert np.array_equal(got.cpu().numpy(), want.astype(np.float32))


@pytest.mark.parametrize("case", ["falling", "negative", "beyond"])
def test_starts_and_lengths_out_of_order_stay_inside(case):
    """Wrong device contents give wrong tokens, but nothing outside the pages named and the rows given is touched."""
    c = Cache(12, 1, 16, 64, [4, 4, 4], [20, 20, 20], seed=3)
    start = {"falling": [0, 40, 10, 60], "negative": [-100, 20, 40, 60], "beyond": [0, 20, 40, 10 ** 9]}[case]
    lengths = {"falling": [4, 4, 4], "negative": [-7, 4, 4], "beyond": [4, 2 ** 31 - 1, 4]}[case]
    k, v = new_tokens(60, 1, 64, H.F32, seed=6)
    st, ln = torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    H.hif8_cache_append(k, v, H.F32, 64, 64, st, ln, 3, 60, *c.args())
    named = set(c.table[c.table >= 0].tolist())
    torch.cuda.synchronize()
    for name in ("k", "v"):
        got = c.d[name].cpu().numpy()
        for p in range(13):
            if p not in named:
                assert np.array_equal(got[p], c.h[name][p])
    out = torch.full((62, 64), 3.0, device="cuda")
    H.hif8_cache_read(*c.args(), ln, st, 3, 60, out[1:61], out[1:61].clone(), H.F32, 64, 64)
    assert (out[0] == 3).all() and (out[61] == 3).all()


def test_more_sequences_than_a_search_round():
    lengths = [i % 37 for i in range(1500)]
    counts = [(i * 7) % 3 for i in range(1500)]
    c = Cache(1500 * 3, 1, 16, 64, lengths, counts, seed=12)
    k, v = new_tokens(sum(counts), 1, 64, H.BF16, seed=3)
    H.hif8_cache_append(k, v, H.BF16, 64, 64, starts(counts), c.d_lengths, 1500, len(k), *c.args())
    c.append(k, v, H.BF16, counts)
    c.same()


def forked(c, parent, new_page, width):
    """The model of hif8_cache_fork."""
    page = c.shape[2]
    table, lengths, taken = np.full((len(parent), width), -1, dtype=np.int32), np.zeros(len(parent), dtype=np.int32), set()
    for i, p in enumerate(parent):
        if not 0 <= p < len(c.lengths):
            if new_page is not None:
                taken.add(new_page[i])
            continue
        n = max(0, min(c.lengths[p], c.table.shape[1] * page, width * page))
        used = -(-n // page)
        table[i, :used], lengths[i] = c.table[p, :used], n
        src = table[i, used - 1] if used else -1
        new = new_page[i] if new_page is not None else -1
        if n % page and 0 <= new < c.shape[0] and 0 <= src < c.shape[0] and new != src and new not in taken:
            for k in c.h:
                c.h[k][new] = c.h[k][src]
            table[i, used - 1] = new
        taken.add(new)
    return table, lengths


@pytest.mark.parametrize("page,dim,heads", [(16, 64, 1), (64, 128, 8), (128, 256, 3)])
def test_fork(page, dim, heads):
    lengths = [0, 1, page, page + 1, 3 * page - 1, 5 * page]
    c = Cache(40, heads, page, dim, lengths, [0] * 6, seed=page)
    parent = [4, 4, 3, 0, 1, 5, 2, 4, -1, 6, 3]
    new = c.spare[:len(parent)].copy()
    new[1] = -1                       # keeps the parent's page
    new[7] = new[0]                   # named twice: the first child gets it
    out = torch.full((len(parent), 7), 99, dtype=torch.int32, device="cuda")
    ln = torch.full((len(parent),), 99, dtype=torch.int32, device="cuda")
    H.hif8_cache_fork(*c.args(), c.d_lengths, 6, torch.tensor(parent, dtype=torch.int32, device="cuda"), torch.from_numpy(new).cuda(), len(parent), out, 7, ln)
    table, want = forked(c, parent, new, 7)
    c.same()
    assert np.array_equal(out.cpu().numpy(), table) and np.array_equal(ln.cpu().numpy(), want)
    # without new pages, and with rows too narrow for the longest
    out = torch.full((len(parent), 2), 99, dtype=torch.int32, device="cuda")
    H.hif8_cache_fork(*c.args(), c.d_lengths, 6, torch.tensor(parent, dtype=torch.int32, device="cuda"), None, len(parent), out, 2, ln)
    table, want = forked(c, parent, None, 2)
    c.same()
    assert np.array_equal(out.cpu().numpy(), table) and np.array_equal(ln.cpu().numpy(), want)


def compacted(c, move):
    """The model of hif8_cache_compact."""
    n_pages, _, page, _ = c.shape
    entries = [(s, i) for s, n in enumerate(c.lengths) for i in range(min(c.table.shape[1], -(-max(0, n) // page))) if 0 <= c.table[s, i] < n_pages]
    live = sorted({int(c.table[e]) for e in entries})
    if move:
        movers, holes = [p for p in live if p >= len(live)], [p for p in range(len(live)) if p not in set(live)]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            for k in c.h:
                c.h[k][b] = c.h[k][a]
        for e in entries:
            c.table[e] = to.get(int(c.table[e]), c.table[e])
        live = list(range(len(live)))
    free = [p for p in range(n_pages) if p not in set(live)]
    return len(live), np.array(free + [-1] * (n_pages - len(free)), dtype=np.int32)


@pytest.mark.parametrize("move", [0, 1])
@pytest.mark.parametrize("n_pages,seqs", [(1, 1), (31, 3), (64, 5), (700, 40), (9000, 600)])
def test_compact(n_pages, seqs, move):
    rng = np.random.default_rng(n_pages)
    most = max(1, n_pages // (2 * seqs)) * 16
    lengths = [int(x) for x in rng.integers(0, most + 1, size=seqs)]
    c = Cache(n_pages, 1, 16, 64, lengths, [0] * seqs, seed=seqs, share=[(0, seqs - 1)] if seqs > 1 else [])
    if seqs > 3:
        c.lengths[2] = 0              # freed: its row stays
        c.table[1, 0] = -1            # names no page
        c.lengths[3] = 10 ** 9        # cut at the row's end, whose last entries are -1
        c.upload()
    if n_pages == 9000:               # a wide table: marked by many blocks
        c.table = np.concatenate([c.table, np.full((seqs, 120), -1, dtype=np.int32)], axis=1)
        c.upload()
    n = H.hif8_cache_compact_workspace_bytes(n_pages)
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
    live, free = torch.full((1,), 77, dtype=torch.int32, device="cuda"), torch.full((n_pages,), 77, dtype=torch.int32, device="cuda")
    for _ in range(2):                # the second time there is nothing to move
        H.hif8_cache_compact(*c.args(), c.d_lengths, seqs, move, live, free, ws, n)
        want, listed = compacted(c, move)
        c.same()
        assert int(live) == want and np.array_equal(free.cpu().numpy(), listed)
        assert np.array_equal(c.d_table.cpu().numpy(), c.table)


def test_compact_nothing():
    ws = torch.empty(H.hif8_cache_compact_workspace_bytes(5), dtype=torch.uint8, device="cuda")
    c = Cache(5, 1, 16, 64, [0, 0], [0, 0], seed=1)
    live, free = torch.full((1,), 7, dtype=torch.int32, device="cuda"), torch.full((5,), 7, dtype=torch.int32, device="cuda")
    H.hif8_cache_compact(*c.args(), c.d_lengths, 2, 1, live, free, ws, ws.numel())
    assert int(live) == 0 and free.tolist() == [0, 1, 2, 3, 4]
    H.hif8_cache_compact(*c.args(), None, 0, 1, live, free, ws, ws.numel())  # no sequences
    assert int(live) == 0 and free.tolist() == [0, 1, 2, 3, 4]
    c.same()


def test_empty_calls_change_nothing():
    c = Cache(4, 1, 16, 64, [5], [20], seed=2)
    before = H.hif8_launch_count()
    H.hif8_cache_append(None, None, H.F32, 64, 64, None, None, 1, 0, *c.args())
    H.hif8_cache_read(*c.args(), None, None, 0, 0, None, None, H.F32, 64, 64)
    H.hif8_cache_fork(*c.args(), c.d_lengths, 1, None, None, 0, None, 1, None)
    assert H.hif8_launch_count() == before
    c.same()


def test_pages_beyond_four_gigabytes():
    """A pool of more than 2^32 bytes: the last pages are written, read, copied and moved."""
    heads, page, dim = 8, 128, 256
    n_pages = (1 << 32) // (heads * page * dim) + 20
    k = torch.zeros(n_pages, heads, page, dim, dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ke, ve = torch.zeros(n_pages, heads, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, heads, dtype=torch.int32, device="cuda")
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device="cuda")
    args = [k, v, ke, ve, n_pages, heads, page, dim, table, 2]
    x, y = new_tokens(200, heads, dim, H.BF16, seed=1)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    H.hif8_cache_append(x, y, H.BF16, x.stride(0), x.stride(1), starts([200]), zero, 1, 200, *args)
    assert int(k[:n_pages - 3].count_nonzero()) == 0 and int(k[n_pages - 2].count_nonzero()) == 0 and int(k[n_pages - 1].count_nonzero()) > 0
    first, again = torch.empty_like(x), torch.empty_like(x)
    H.hif8_cache_read(*args, zero, starts([200]), 1, 200, first, again, H.BF16, x.stride(0), x.stride(1))
    kept = (first.clone(), again.clone())
    out, ln = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([200], dtype=torch.int32, device="cuda")
    H.hif8_cache_fork(*args, lengths, 1, zero, torch.tensor([n_pages - 2], dtype=torch.int32, device="cuda"), 1, out, 2, ln)
    assert out.tolist() == [[n_pages - 1, n_pages - 2]] and torch.equal(k[n_pages - 2], k[n_pages - 3]) and torch.equal(v[n_pages - 2], v[n_pages - 3])
    live, free = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ws = torch.empty(H.hif8_cache_compact_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda")
    args[8] = out
    H.hif8_cache_compact(*args, lengths, 1, 1, live, free, ws, ws.numel())
    assert out.tolist() == [[1, 0]] and int(live) == 2
    H.hif8_cache_read(*args, zero, starts([200]), 1, 200, first, again, H.BF16, x.stride(0), x.stride(1))
    assert torch.equal(first, kept[0]) and torch.equal(again, kept[1])
