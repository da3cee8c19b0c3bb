"""A key/value cache for the tests: its pages on the device and, in numpy, what they ought to hold."""
import numpy as np
import torch

import paper_2409_16626_b200 as H
from oracle import hif8_oracle as O

TORCH = {H.F32: torch.float32, H.BF16: torch.bfloat16, H.F16: torch.float16}
VALUES = np.array([O.value(c) for c in range(256)])


def bits_of(x):
    """The raw encodings of a tensor, as the oracle takes them."""
    x = x.cpu().contiguous()
    return x.view(torch.int32).numpy().view(np.uint32) if x.dtype == torch.float32 else x.view(torch.int16).numpy().view(np.uint16)


class Cache:
    """Pages that no row of the table names, slots behind a sequence's length and a guard page behind the pool hold stale bytes."""

    def __init__(self, n_pages, heads, page, dim, lengths, room, seed, share=()):
        rng = np.random.default_rng(seed)
        self.rng, self.shape, self.lengths = rng, (n_pages, heads, page, dim), list(lengths)
        codes = [rng.integers(0, 256, size=(n_pages + 1, heads, page, dim)).astype(np.uint8) for _ in range(2)]
        exps = [rng.integers(-6, 7, size=(n_pages + 1, heads)).astype(np.int32) for _ in range(2)]
        need = [-(-(n + r) // page) for n, r in zip(lengths, room)]
        order = rng.permutation(n_pages)
        width = max(need, default=0) + 2
        table, at = np.full((len(need), width), -1, dtype=np.int32), 0
        for s, k in enumerate(need):
            table[s, :k] = order[at:at + k]
            at += k
        for a, b in share:  # sequence b's full pages are a's
            k = min(lengths[a], lengths[b]) // page
            table[b, :k] = table[a, :k]
        self.spare = order[at:].astype(np.int32)
        self.h = {"k": codes[0], "v": codes[1], "k_exp": exps[0], "v_exp": exps[1]}
        self.table = table
        self.upload()

    def upload(self):
        self.d = {k: torch.from_numpy(v.copy()).cuda() for k, v in self.h.items()}
        self.d_table = torch.from_numpy(self.table.copy()).cuda()
        self.d_lengths = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def args(self, table=None):
        n, heads, page, dim = self.shape
        t = self.d_table if table is None else table
        return self.d["k"], self.d["v"], self.d["k_exp"], self.d["v_exp"], n, heads, page, dim, t, t.stride(0)

    def fill(self, spread=6):
        """Every token of every sequence a value of the normal kind: finite codes, a few at the ends of the format."""
        n, heads, page, dim = self.shape
        for name in ("k", "v"):
            x = self.rng.standard_normal((n + 1, heads, page, dim)).astype(np.float32)
            x *= np.exp2(self.rng.integers(-spread, spread + 1, size=(n + 1, heads, 1, 1))).astype(np.float32)
            e = self.h[name + "_exp"]
            for p in range(n + 1):
                for h in range(heads):
                    _, se = O.amax_scale(x[p, h].ravel(), O.F32, 3)
                    e[p, h] = se
                    self.h[name][p, h] = O.encode(x[p, h].ravel(), O.F32, se, O.TA, 0, quick=True).reshape(page, dim)
        self.upload()

    def same(self, pages=None):
        """The device's pages are the expected ones, to the last byte, the guard page too."""
        torch.cuda.synchronize()
        for k in ("k", "v", "k_exp", "v_exp"):
            got = self.d[k].cpu().numpy()
            assert np.array_equal(got, self.h[k]), k

    def values(self, seq, n, name):
        """Values [n tokens, heads, dim] of a sequence's first n tokens, in 64 bits; tokens of no page are None in the mask returned."""
        _, heads, page, dim = self.shape
        out, there = np.zeros((n, heads, dim)), np.zeros(n, dtype=bool)
        for t in range(n):
            p = self.table[seq, t // page] if t // page < self.table.shape[1] else -1
            if 0 <= p < self.shape[0]:
                there[t] = True
                out[t] = VALUES[self.h[name][p, :, t % page]] * np.exp2(-self.h[name + "_exp"][p].astype(np.float64))[:, None]
        return out, there

    def append(self, k, v, dtype, counts, target=3, rnd=H.RND_TA, flags=0):
        """What hif8_cache_append of k, v [tokens, heads, dim] ought to do to the pages."""
        _, heads, page, dim = self.shape
        at = 0
        for s, m in enumerate(counts):
            i = 0
            while i < m:
                pos = self.lengths[s] + i
                n = min(m - i, page - pos % page)
                p = self.table[s, pos // page] if pos // page < self.table.shape[1] else -1
                if 0 <= p < self.shape[0]:
                    for name, x in (("k", k), ("v", v)):
                        for h in range(heads):
                            block = bits_of(x[at + i:at + i + n, h]).ravel()
                            if pos % page == 0:
                                _, se = O.amax_scale(block, dtype, target)
                                self.h[name + "_exp"][p, h] = np.clip(se, -H.CACHE_EXP_MAX, H.CACHE_EXP_MAX)
                            se = int(np.clip(self.h[name + "_exp"][p, h], -H.CACHE_EXP_MAX, H.CACHE_EXP_MAX))
                            self.h[name][p, h, pos % page:pos % page + n] = O.encode(block, dtype, se, rnd, flags, quick=True).reshape(n, dim)
                i += n
            at += m


def starts(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), device="cuda")
