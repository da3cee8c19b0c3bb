"""The operators of the HiF8 key/value cache as measurable cases: new tokens written into its pages and read back, attention over
it, sequences forked, pages compacted.

The cache is paged: K and V each [pages, kv_heads, page_tokens, head_dim] bytes, and one power-of-two scale exponent for each
block of tokens (page) and head; a row of the page table lists a sequence's pages.  A case is a dict of plain values.  Which
lengths its sequences have follows from the case alone, what they hold from the seed.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TARGET = 3  # exponent of a block's largest magnitude: it and what lies down to 1/128 of it keep three mantissa bits

LARGEST_CACHE = 8 * 131072 * 8 * 128 * 2  # bytes
LARGEST_SCORES = 32 * 2048 * 16461


def listed():
    gqa = {"heads": 32, "kv_heads": 8, "dim": 128}
    return [
        # one user's next token in a short conversation: latency
        {"name": "decode_one", "op": "attention", "seqs": 1, "ctx": 517, "q": 1, "window": 0, "page": 64, "dtype": "bf16", **gqa},
        # a serving batch's next tokens, ragged contexts
        {"name": "decode_batch", "op": "attention", "seqs": 64, "ctx": 4096, "q": 1, "window": 0, "page": 64, "dtype": "bf16", **gqa},
        # few users with very long contexts, eight query heads to a key head: the largest cache
        {"name": "decode_long", "op": "attention", "seqs": 8, "ctx": 131072, "q": 1, "window": 0, "page": 128, "dtype": "f16", "heads": 64, "kv_heads": 8, "dim": 128},
        # four drafted tokens a sequence checked at once, small heads without sharing, a sliding window
        {"name": "verify_window", "op": "attention", "seqs": 16, "ctx": 8190, "q": 4, "window": 1024, "page": 32, "dtype": "f16", "heads": 16, "kv_heads": 16, "dim": 64},
        # a chunk of a long prompt against all that is cached of it: the most arithmetic
        {"name": "prefill_chunk", "op": "attention", "seqs": 1, "ctx": 16461, "q": 2048, "window": 0, "page": 64, "dtype": "bf16", **gqa},
        # whole short prompts of ragged lengths
        {"name": "prefill_ragged", "op": "attention", "seqs": 12, "ctx": 2047, "q": 2047, "window": 700, "page": 16, "dtype": "f16", "heads": 16, "kv_heads": 4, "dim": 64},
        # a serving batch's new tokens written to the cache and read back as the layer's own K and V
        {"name": "append_tokens", "op": "append", "seqs": 128, "ctx": 3000, "new": 1, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # ragged prompts written to the cache and read back
        {"name": "append_prompts", "op": "append", "seqs": 5, "ctx": 100, "new": 8190, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # beam search: a step's survivors continue from their parents' pages
        {"name": "fork_beams", "op": "fork", "seqs": 32, "ctx": 600, "children": 32, "kv_heads": 8, "dim": 128, "page": 16},
        # many samples of a few long prompts
        {"name": "fork_samples", "op": "fork", "seqs": 16, "ctx": 9000, "children": 512, "kv_heads": 8, "dim": 128, "page": 128},
        # a small pool after a few sequences have ended
        {"name": "compact_small", "op": "compact", "seqs": 24, "ctx": 500, "kv_heads": 4, "dim": 64, "page": 16},
        # a large pool, half of it free and scattered
        {"name": "compact_large", "op": "compact", "seqs": 96, "ctx": 9000, "kv_heads": 8, "dim": 128, "page": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "fork", "compact"])
    dim, page = rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    kv = rng.choice([1, 2, 4, 8, 16])
    if op == "attention":
        while True:
            kind = rng.choice(["decode", "decode", "verify", "prefill"])
            c = {"op": op, "seqs": _log(rng, 1, 256), "ctx": _log(rng, 1, 131072), "q": 1, "window": 0, "page": page, "dtype": rng.choice(["bf16", "f16"]),
                 "heads": kv * rng.choice([1, 2, 4, 5, 7, 8, 16]), "kv_heads": kv, "dim": dim}
            if kind == "verify":
                c["q"] = rng.randint(2, 8)
            if kind == "prefill":
                c["seqs"], c["q"] = _log(rng, 1, 16), _log(rng, 16, 4096)
            if rng.random() < 0.25:
                c["window"] = _log(rng, 16, 8192)
            cache = c["seqs"] * c["ctx"] * kv * dim * 2
            if cache <= LARGEST_CACHE // 2 and c["seqs"] * c["heads"] * c["q"] * c["ctx"] <= LARGEST_SCORES // 2 and c["heads"] <= 128:
                return c
    if op == "append":
        new = rng.choice([1, _log(rng, 2, 8192)])
        return {"op": op, "seqs": _log(rng, 1, 256) if new == 1 else _log(rng, 1, 8), "ctx": _log(rng, 1, 4096), "new": new, "kv_heads": kv, "dim": dim, "page": page,
                "dtype": rng.choice(["bf16", "f16", "f32"])}
    if op == "fork":
        return {"op": op, "seqs": _log(rng, 1, 64), "ctx": _log(rng, 1, 8192), "children": _log(rng, 1, 512), "kv_heads": kv, "dim": dim, "page": page}
    return {"op": op, "seqs": _log(rng, 2, 96), "ctx": _log(rng, 16, 8192), "kv_heads": kv, "dim": dim, "page": page}


def _lengths(c):
    """Tokens that each sequence has in the cache: the longest has ctx, the others are spread below it."""
    rng = random.Random("%s %d %d" % (c["op"], c["seqs"], c["ctx"]))
    n = [max(1, int(c["ctx"] * (0.1 + 0.9 * rng.random()))) for _ in range(c["seqs"])]
    n[rng.randrange(c["seqs"])] = c["ctx"]
    return n


def _counts(c):
    """New tokens, or queries, of each sequence; none of them more than it has tokens (attention)."""
    if c["op"] == "append":
        rng = random.Random("new %d %d" % (c["seqs"], c["new"]))
        return [c["new"] if i == 0 else max(1, int(c["new"] * rng.random())) for i in range(c["seqs"])]
    return [min(c["q"], n) for n in _lengths(c)]


def _visible(c):
    """Over all queries of all sequences: the tokens that each may look at."""
    w, total = c["window"] or 1 << 40, 0
    for n, q in zip(_lengths(c), _counts(c)):
        total += sum(min(w, n - q + i + 1) for i in range(q))
    return total


def work(c):
    token = 2 * c["kv_heads"] * c["dim"]  # bytes of one token in the cache
    page = token * c["page"] + 8 * c["kv_heads"]
    if c["op"] == "attention":
        w = c["window"] or 1 << 40
        cached = sum(min(n, w + q - 1) for n, q in zip(_lengths(c), _counts(c)))
        return {"bytes": cached * token + sum(_counts(c)) * c["heads"] * (c["dim"] * 4 + 4), "flops": 4 * _visible(c) * c["heads"] * c["dim"]}
    if c["op"] == "append":  # the source, the codes written and read, the values read back
        size = 4 if c["dtype"] == "f32" else 2
        return {"bytes": sum(_counts(c)) * token * (2 * size + 2), "flops": 0}
    if c["op"] == "fork":
        lengths, parents = _lengths(c), _parents(c)
        rows = sum(-(-lengths[p] // c["page"]) for p in parents)
        partial = [p for p in parents if lengths[p] % c["page"]]
        return {"bytes": len(partial) * page + len(set(partial)) * page + 8 * rows, "flops": 0}
    live, moved, pages = _pool(c)
    return {"bytes": 2 * moved * page + 8 * live + 4 * pages, "flops": 0}


def _parents(c):
    rng = random.Random("parents %d %d" % (c["seqs"], c["children"]))
    return [rng.randrange(c["seqs"]) for _ in range(c["children"])]


def _pool(c):
    """Live pages, those beyond the live count (which have to move), and pages of a compaction case's pool."""
    live, pages, table = _compact_table(c)
    return live, sum(p >= live for row in table for p in row), pages


def _compact_table(c):
    need = [-(-n // c["page"]) for n in _lengths(c)]
    live = sum(need)
    pages = 2 * live
    rng = random.Random("pool %d" % pages)
    places = rng.sample(range(pages), live)
    table, at = [], 0
    for k in need:
        table.append(places[at:at + k])
        at += k
    return live, pages, table


# ---------------------------------------------------------------------------------------------------------------------
# HiF8 in elementary operations
# ---------------------------------------------------------------------------------------------------------------------
def _code_values():
    """The value of each of the 256 codes (sign, prefix-coded dot field, sign-magnitude exponent, 3/2/1-bit mantissa)."""
    m = torch.arange(128)
    region = torch.bucketize(m, torch.tensor([8, 16, 32, 64, 96]), right=True)  # 0: denormal, 1..5: D = 0..4
    width = torch.tensor([3, 3, 3, 3, 2, 1])[region]
    low = torch.tensor([0, 0, 1, 2, 4, 8])[region]           # smallest magnitude of the exponent
    d = torch.tensor([0, 0, 1, 2, 3, 4])[region]             # bits of the exponent field, its sign on top
    mantissa = (m & ((1 << width) - 1)).float() / (1 << width).float()
    field = (m >> width) & ((1 << d) - 1)
    bits = torch.clamp(d - 1, min=0)
    e = low + (field & ((1 << bits) - 1))
    e = torch.where((d > 0) & ((field >> bits) == 1), -e, e)
    v = torch.where(region == 0, torch.exp2((m - 23).float()), torch.exp2(e.float()) * (1 + mantissa))
    v[0], v[0x6F] = 0.0, math.inf
    v = torch.cat([v, -v])
    v[128] = math.nan
    return v


def _rounded(y):
    """Nearest HiF8 values of y, halves away from zero."""
    a = y.abs()
    e = torch.clamp(torch.frexp(a)[1] - 1, min=-22)
    mag = e.abs()
    width = torch.where(mag <= 3, 3, torch.where(mag <= 7, 2, torch.where(e > -16, 1, 0)))
    step = torch.ldexp(torch.ones_like(y), e - width)
    x = a / step
    low = torch.floor(x)
    r = (low + (x - low >= 0.5)) * step
    return torch.where(r >= 49152.0, math.inf, r) * torch.sign(y)


def _codes(v):
    """The codes of finite HiF8 values."""
    a = v.abs()
    e = torch.frexp(a)[1] - 1
    mag, neg = e.abs(), (e < 0).int()
    width = torch.where(mag <= 3, 3, torch.where(mag <= 7, 2, 1))
    m = torch.ldexp(torch.ldexp(a, -e) - 1, width).int()
    c = torch.where(mag == 0, 0x08 | m, torch.where(mag == 1, 0x10 | neg << 3 | m, torch.where(mag <= 3, 0x20 | neg << 4 | (mag & 1) << 3 | m, torch.where(
        mag <= 7, 0x40 | neg << 4 | (mag & 3) << 2 | m, 0x60 | neg << 4 | (mag & 7) << 1 | m))))
    c = torch.where(e <= -16, e + 23, c)
    return torch.where(a == 0, 0, c + 128 * (v < 0)).to(torch.uint8)


def _block_exponent(amax):
    """Exponent that brings a block's largest magnitude to the binade of 2^TARGET; 0 for a block of zeros."""
    return torch.where(amax > 0, torch.clamp(TARGET - (torch.frexp(amax)[1] - 1), -48, 48), 0).int()


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _start(counts):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


def _filled(pages, c, g):
    """Codes and exponents of a pool of pages: bell-shaped values, blocks of different spread, a few channels with outliers."""
    shape = (pages, c["kv_heads"], c["page"], c["dim"])
    codes = torch.empty(shape, dtype=torch.uint8, device="cuda")
    exps = torch.empty(shape[:2], dtype=torch.int32, device="cuda")
    step = max(1, (1 << 27) // (c["kv_heads"] * c["page"] * c["dim"]))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        x = torch.randn((n,) + shape[1:], generator=g, device="cuda")
        x *= torch.exp2(torch.randint(-1, 2, (n, c["kv_heads"], 1, 1), generator=g, device="cuda").float())
        x[..., 5::37] *= 4
        e = _block_exponent(x.abs().amax((2, 3)))
        exps[p:p + n] = e
        codes[p:p + n] = _codes(_rounded(torch.ldexp(x, e[:, :, None, None])))
    return codes, exps


def prepare(c, seed):
    g = _generator(seed)
    s = {"case": c, "values": _code_values().cuda()}
    lengths = _lengths(c)
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if c["op"] == "compact":
        _, pages, rows = _compact_table(c)
    else:
        new = _counts(c) if c["op"] == "append" else [0] * c["seqs"]
        need = [-(-(n + k) // c["page"]) for n, k in zip(lengths, new)]
        pages = sum(need) + (c["children"] if c["op"] == "fork" else 3)
        order = torch.randperm(pages, generator=g, device="cuda").tolist()
        rows, at = [], 0
        for k in need:
            rows.append(order[at:at + k])
            at += k
        s["spare"] = torch.tensor(order[at:], dtype=torch.int32, device="cuda")
    width = max(len(r) for r in rows) + 1
    s["table"] = torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32, device="cuda")
    (s["k"], s["k_exp"]), (s["v"], s["v_exp"]) = _filled(pages, c, g), _filled(pages, c, g)
    if c["op"] == "attention":
        counts = _counts(c)
        n, shape = sum(counts), (sum(counts), c["heads"], c["dim"])
        s["q"] = torch.randn(shape, generator=g, device="cuda").to(TORCH[c["dtype"]])
        s["q_start"], s["n"], s["max_q"], s["max_length"] = _start(counts), n, max(counts), max(lengths)
        s["out"] = torch.empty(shape, dtype=TORCH[c["dtype"]], device="cuda")
        s["lse"] = torch.empty(n, c["heads"], device="cuda")
        s["rows"] = _padded_rows(counts)
        s["ws"] = {}
    if c["op"] == "append":
        counts = _counts(c)
        shape = (2, sum(counts), c["kv_heads"], c["dim"])
        x = torch.randn(shape, generator=g, device="cuda")
        x[..., 5::37] *= 4
        s["new"] = x.to(TORCH[c["dtype"]])
        s["start"], s["n"] = _start(counts), sum(counts)
        s["back"] = torch.empty(shape, dtype=TORCH[c["dtype"]], device="cuda")
    if c["op"] == "fork":
        s["parent"] = torch.tensor(_parents(c), dtype=torch.int32, device="cuda")
        s["table_out"] = torch.full((c["children"], width), -1, dtype=torch.int32, device="cuda")
        s["lengths_out"] = torch.zeros(c["children"], dtype=torch.int32, device="cuda")
    if c["op"] == "compact":
        s["free"] = torch.empty(pages, dtype=torch.int32, device="cuda")
        s["live"] = torch.empty(1, dtype=torch.int32, device="cuda")
        s["moved_table"] = torch.empty_like(s["table"])
        s["ws"] = {}
    return s


def _padded_rows(counts):
    """For each query its sequence and its place among that sequence's."""
    seq = [i for i, n in enumerate(counts) for _ in range(n)]
    place = [j for n in counts for j in range(n)]
    return torch.tensor(seq, device="cuda"), torch.tensor(place, device="cuda")


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return {"attention": _attention_own, "append": _append_own, "fork": _fork_own, "compact": _compact_own}[op](s)
    return {"attention": _attention, "append": _append, "fork": _fork, "compact": _compact}[op](s)


def _workspace(s, n):
    """A workspace of that many bytes, kept from call to call as a program keeps it."""
    if s["ws"].get("n") != n:
        s["ws"] = {"n": n, "t": torch.empty(n, dtype=torch.uint8, device="cuda")}
    return s["ws"]["t"]


def _cache_args(s):
    c = s["case"]
    return s["k"], s["v"], s["k_exp"], s["v_exp"], s["k"].shape[0], c["kv_heads"], c["page"], c["dim"], s["table"], s["table"].stride(0)


def _attention_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    n = H.hif8_cache_attention_workspace_bytes(c["seqs"], s["n"], s["max_q"], s["max_length"], c["heads"], c["kv_heads"], c["dim"])
    ws = _workspace(s, n)
    H.hif8_cache_attention(s["q"], H.F16 if c["dtype"] == "f16" else H.BF16, s["q"].stride(0), s["q"].stride(1), s["q_start"], s["lengths"], c["seqs"], s["n"], s["max_q"],
                           s["max_length"], *_cache_args(s), c["heads"], c["dim"] ** -0.5, 1, c["window"], s["out"], s["out"].stride(0), s["out"].stride(1), s["lse"], ws, n)
    return {"out": s["out"], "lse": s["lse"]}


def _append_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    dtype = {"f32": H.F32, "bf16": H.BF16, "f16": H.F16}[c["dtype"]]
    k, v = s["new"][0], s["new"][1]
    H.hif8_cache_append(k, v, dtype, k.stride(0), k.stride(1), s["start"], s["lengths"], c["seqs"], s["n"], *_cache_args(s), TARGET, H.RND_TA, 0)
    H.hif8_cache_read(*_cache_args(s), s["lengths"], s["start"], c["seqs"], s["n"], s["back"][0], s["back"][1], dtype, k.stride(0), k.stride(1))
    return {"k": s["back"][0], "v": s["back"][1], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def _fork_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    H.hif8_cache_fork(*_cache_args(s), s["lengths"], c["seqs"], s["parent"], s["spare"], c["children"], s["table_out"], s["table_out"].stride(0), s["lengths_out"])
    return {"table": s["table_out"], "lengths": s["lengths_out"], "k": s["k"], "v": s["v"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def _compact_own(s):
    import paper_2409_16626_b200 as H

    n = H.hif8_cache_compact_workspace_bytes(s["k"].shape[0])
    ws = _workspace(s, n)
    s["moved_table"].copy_(s["table"])  # the call rewrites the table in place; the next pass starts from the same one
    a = list(_cache_args(s))
    a[8] = s["moved_table"]
    H.hif8_cache_compact(*a, s["lengths"], s["case"]["seqs"], 1, s["live"], s["free"], ws, n)
    return {"table": s["moved_table"], "live": s["live"], "free": s["free"], "k": s["k"], "v": s["v"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def _sequences(codes, exps, table, values):
    """All sequences' values, padded to the widest: [seqs, kv_heads, tokens, dim]."""
    t = table.clamp(min=0).long()
    x = torch.ldexp(values[codes[t].int()], -exps[t][..., None, None])  # [seqs, pages, heads, page, dim]
    return x.transpose(1, 2).flatten(2, 3)


def _attention(s):
    c = s["case"]
    b, h, d, group = c["seqs"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    seq, place = s["rows"]
    used = -(-s["max_length"] // c["page"])
    table = s["table"][:, :used]
    q = torch.zeros(b, s["max_q"], c["heads"], d, device="cuda")
    q[seq, place] = s["q"].float()
    q = q.view(b, s["max_q"], h, group, d).permute(0, 2, 1, 3, 4).reshape(b, h, s["max_q"] * group, d)
    k = _sequences(s["k"], s["k_exp"], table, s["values"])
    scores = torch.matmul(q, k.transpose(2, 3)).mul_(d ** -0.5).view(b, h, s["max_q"], group, -1)
    del k
    j = torch.arange(scores.shape[-1], device="cuda")
    at = (s["lengths"] - (s["q_start"][1:] - s["q_start"][:-1]))[:, None] + torch.arange(s["max_q"], device="cuda")  # the queries' own positions
    hidden = (j > at[..., None]) | (j >= s["lengths"][:, None, None])
    if c["window"]:
        hidden |= j <= at[..., None] - c["window"]
    scores.masked_fill_(hidden[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    v = _sequences(s["v"], s["v_exp"], table, s["values"])
    v = v.masked_fill_((j >= s["lengths"][:, None])[:, None, :, None], 0.0)
    out = torch.matmul(scores.view(b, h, s["max_q"] * group, -1), v).view(b, h, s["max_q"], group, d) / total
    lse = (top + total.log()).squeeze(-1)
    out = out.permute(0, 2, 1, 3, 4).reshape(b, s["max_q"], c["heads"], d)[seq, place]
    return {"out": out.to(TORCH[c["dtype"]]), "lse": lse.permute(0, 2, 1, 3).reshape(b, s["max_q"], c["heads"])[seq, place]}


def _append(s):
    c, p = s["case"], s["case"]["page"]
    counts = s["start"][1:] - s["start"][:-1]
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), counts.long(), output_size=s["n"])
    at = torch.arange(s["n"], device="cuda") - s["start"][:-1].long()[seq] + s["lengths"].long()[seq]  # positions of the new tokens
    page, slot = s["table"].long()[seq, at // p], at % p
    started = (s["lengths"].long()[seq] // p == at // p) & (s["lengths"].long()[seq] % p > 0)  # on a page that had tokens before
    pages = s["k"].shape[0]
    answer = {}
    for x, codes, exps, name in ((s["new"][0], s["k"], s["k_exp"], "k"), (s["new"][1], s["v"], s["v_exp"], "v")):
        x = x.float()
        amax = torch.zeros(pages, c["kv_heads"], device="cuda").index_reduce_(0, page, x.abs().amax(-1), "amax")
        fresh = torch.zeros(pages, dtype=torch.bool, device="cuda").index_fill_(0, page, True)
        fresh = fresh & ~torch.zeros(pages, device="cuda").index_add_(0, page, started.float()).bool()
        exps.copy_(torch.where(fresh[:, None], _block_exponent(amax), exps))
        e = exps[page][..., None]
        r = _rounded(torch.ldexp(x, e))
        codes[page, :, slot] = _codes(r)
        answer[name] = torch.ldexp(r, -e).to(TORCH[c["dtype"]])
        answer[name + "_exp"] = exps
    return answer


def _fork(s):
    p = s["case"]["page"]
    parent = s["parent"].long()
    lengths = s["lengths"][parent]
    table = s["table"][parent]
    used = (lengths + p - 1) // p
    table = torch.where(torch.arange(table.shape[1], device="cuda") < used[:, None], table, -1)
    last = (used - 1).clamp(min=0).long()
    copied = lengths % p != 0
    i = torch.arange(len(parent), device="cuda")
    source = table[i, last].long()
    new = torch.where(copied, s["spare"].long(), source)
    for x in (s["k"], s["v"], s["k_exp"], s["v_exp"]):
        x[new] = x[source]
    table[i, last] = new.int()
    return {"table": table, "lengths": lengths, "k": s["k"], "v": s["v"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def _compact(s):
    p, pages = s["case"]["page"], s["k"].shape[0]
    used = torch.arange(s["table"].shape[1], device="cuda") < ((s["lengths"] + p - 1) // p)[:, None]
    page = torch.arange(pages, device="cuda")
    live = torch.zeros(pages, dtype=torch.bool, device="cuda")
    live[s["table"][used].long()] = True
    n = live.sum()
    movers, holes = (live & (page >= n)).nonzero()[:, 0], (~live & (page < n)).nonzero()[:, 0]
    for x in (s["k"], s["v"], s["k_exp"], s["v_exp"]):
        x[holes] = x[movers]
    to = page.clone()
    to[movers] = holes
    table = torch.where(used, to[s["table"].clamp(min=0).long()].int(), s["table"])
    free = torch.where(page < pages - n, page + n, -1).int()
    return {"table": table, "live": n.int().view(1), "free": free, "k": s["k"], "v": s["v"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _value_of_code(c):
    """One code's value, read field by field."""
    bits, sign = format(c & 127, "07b"), -1.0 if c & 128 else 1.0
    if c in (0, 128):
        return 0.0 if c == 0 else math.nan
    if c & 127 == 0x6F:
        return sign * math.inf
    for prefix, d in (("11", 4), ("10", 3), ("01", 2), ("001", 1), ("0001", 0)):
        if bits.startswith(prefix):
            rest = bits[len(prefix):]
            exponent, mantissa = rest[:d], rest[d:]
            magnitude = int("1" + exponent[1:], 2) if d else 0
            e = -magnitude if d and exponent[0] == "1" else magnitude
            return sign * 2.0 ** e * (1 + int(mantissa, 2) / 2 ** len(mantissa))
    return sign * 2.0 ** (int(bits[4:], 2) - 23)


def exact(c, seed):
    if c["op"] not in ("attention", "append"):
        return None  # pages and whole numbers, copied as they are
    s = prepare(c, seed)
    finite = torch.tensor([_value_of_code(i) for i in range(256)], dtype=torch.float64, device="cuda")
    lengths, counts = _lengths(c), _counts(c)
    if c["op"] == "append":
        return _exact_append(c, s, finite, lengths, counts)
    d, group, at = c["dim"], c["heads"] // c["kv_heads"], 0
    out = torch.zeros(s["n"], c["heads"], d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["n"], c["heads"], dtype=torch.float64, device="cuda")
    for i, (n, m) in enumerate(zip(lengths, counts)):
        pages = s["table"][i, :-(-n // c["page"])].long()
        key = torch.arange(n, device="cuda")
        pos = torch.arange(n - m, n, device="cuda")
        seen = key[None, :] <= pos[:, None]
        if c["window"]:
            seen &= key[None, :] > pos[:, None] - c["window"]
        for h in range(c["kv_heads"]):
            scale = lambda e: torch.pow(2.0, -e[pages, h].double()).repeat_interleave(c["page"])[:n, None]  # noqa: E731
            k = finite[s["k"][pages, h].reshape(-1, d)[:n].int()] * scale(s["k_exp"])
            v = finite[s["v"][pages, h].reshape(-1, d)[:n].int()] * scale(s["v_exp"])
            for r in range(h * group, (h + 1) * group):
                x = (s["q"][at:at + m, r].double() @ k.T) / math.sqrt(d)
                x[~seen] = -math.inf
                norm = torch.logsumexp(x, 1)
                out[at:at + m, r] = torch.exp(x - norm[:, None]) @ v
                lse[at:at + m, r] = norm
        at += m
    return {"out": out, "lse": lse}


def _exact_append(c, s, finite, lengths, counts):
    grid = torch.sort(finite[:128][torch.isfinite(finite[:128])])[0]  # magnitudes, 0 among them
    answer = {"k_exp": None, "v_exp": None}
    for x, exps, name in ((s["new"][0], s["k_exp"], "k"), (s["new"][1], s["v_exp"], "v")):
        x, at = x.double(), 0
        got = torch.zeros_like(x)
        for i, (n, m) in enumerate(zip(lengths, counts)):
            first = 0
            while first < m:
                page = (n + first) // c["page"]
                last = min(m, (page + 1) * c["page"] - n)
                block = x[at + first:at + last]  # [tokens, heads, dim]
                e = exps[s["table"][i, page].long()].double()
                if (n + first) % c["page"] == 0:
                    top = block.abs().amax((0, 2))
                    e = torch.where(top > 0, TARGET - torch.floor(torch.log2(top)), 0.0).clamp(-48, 48)
                f = torch.pow(2.0, e)[None, :, None]
                y = block.abs() * f
                k = torch.searchsorted(grid, y.contiguous()).clamp(1, len(grid) - 1)
                low, high = grid[k - 1], grid[k]
                r = torch.where(high - y <= y - low, high, low)
                got[at + first:at + last] = torch.sign(block) * r / f
                first = last
            at += m
        answer[name] = got
    return answer
