"""The operators of a transformer layer whose products are in HiF8 with a scale for each block of 128, as measurable cases: the norm in front
of a product and its gradient, the product and its gradients, the clipping of all gradients in front of an optimizer's step.

A matrix of codes has one power-of-two exponent e for each block, and a code stands for value(code) * 2^-e: blocks of 1 x 128 for activations
and their gradients, of 128 x 128 for weights.  A case is a dict of plain values; what its tensors hold follows from the seed.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TARGET = 3     # exponent of a block's largest magnitude: it and what lies down to 1/128 of it keep three mantissa bits
LIMIT = 96     # exponents of blocks lie within -LIMIT .. LIMIT
EPS = 1e-5     # of the norm

LARGEST_ROWS = 16381 * 8192
LARGEST_PRODUCT = 8192 * 8192 * 28672
LARGEST_GRADIENTS = 440_000_000


def listed():
    return [
        # one user's next token: latency
        {"name": "norm_one", "op": "norm", "rows": 1, "cols": 4096, "dtype": "bf16"},
        # the tokens of a batch of long prompts, not a multiple of anything: memory
        {"name": "norm_prompts", "op": "norm", "rows": 16381, "cols": 8192, "dtype": "bf16"},
        # a short batch of a small model trained in FP16, an odd width
        {"name": "norm_backward_small", "op": "norm_backward", "rows": 301, "cols": 1001, "dtype": "f16", "residual": False},
        # a training batch, the residual stream's gradient added
        {"name": "norm_backward_large", "op": "norm_backward", "rows": 16384, "cols": 8192, "dtype": "bf16", "residual": True},
        # the next token of one user through a feed-forward layer's weight
        {"name": "linear_one", "op": "linear", "tokens": 1, "inner": 4096, "outer": 14336, "dtype": "bf16", "out": "bf16"},
        # the next tokens of a serving batch
        {"name": "linear_batch", "op": "linear", "tokens": 48, "inner": 8192, "outer": 8192, "dtype": "bf16", "out": "bf16"},
        # a chunk of a prompt onto a vocabulary of an odd size, results in FP32
        {"name": "linear_logits", "op": "linear", "tokens": 333, "inner": 4096, "outer": 32003, "dtype": "f16", "out": "f32"},
        # a training batch through the widest layer: the most arithmetic
        {"name": "linear_large", "op": "linear", "tokens": 8192, "inner": 8192, "outer": 28672, "dtype": "bf16", "out": "bf16"},
        # a small layer's gradients from a ragged batch
        {"name": "linear_backward_small", "op": "linear_backward", "tokens": 777, "inner": 768, "outer": 1536, "dtype": "f32"},
        # a large layer's gradients, the weight's added to those of the micro-batches before
        {"name": "linear_backward_large", "op": "linear_backward", "tokens": 4096, "inner": 4096, "outer": 14336, "dtype": "bf16"},
        # all gradients of a small model
        {"name": "clip_small", "op": "clip", "hidden": 250, "ffn": 700, "layers": 4, "dtype": "f32", "max_norm": 1.0},
        # those of two layers of a large one: more than the caches hold
        {"name": "clip_large", "op": "clip", "hidden": 4096, "ffn": 14336, "layers": 2, "dtype": "bf16", "max_norm": 1.0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "linear", "linear", "linear_backward", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_backward"):
        while True:
            c = {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 64, 16384), "dtype": dtype}
            if rng.random() < 0.6:
                c["cols"] = max(64, c["cols"] // 64 * 64)
            if op == "norm_backward":
                c["residual"] = rng.random() < 0.7
            if c["rows"] * c["cols"] * (2 if dtype == "f32" else 1) <= LARGEST_ROWS:
                return c
    if op in ("linear", "linear_backward"):
        while True:
            least = 1 if op == "linear" else 16
            c = {"op": op, "tokens": _log(rng, least, 8192), "inner": _log(rng, 64, 16384), "outer": _log(rng, 64, 28672), "dtype": dtype}
            if rng.random() < 0.6:
                c["inner"], c["outer"] = max(64, c["inner"] // 64 * 64), max(64, c["outer"] // 64 * 64)
            if op == "linear":
                c["out"] = rng.choice(["bf16", "bf16", "f32"])
            if c["tokens"] * c["inner"] * c["outer"] <= LARGEST_PRODUCT // 8:
                return c
    while True:
        c = {"op": op, "hidden": _log(rng, 16, 4096), "ffn": _log(rng, 16, 14336), "layers": _log(rng, 1, 32), "dtype": dtype, "max_norm": rng.choice([1.0, 1.0, 1e6])}
        if sum(sum(s) for s in _sizes(c)) * (2 if dtype == "f32" else 1) <= LARGEST_GRADIENTS:
            return c


def _sizes(c):
    """Elements of the gradients: of the matrices, in the case's type, and of the norms' weights, in FP32."""
    h, f = c["hidden"], c["ffn"]
    layer = [h * h, h * (h // 4 + 1), h * (h // 4 + 1), h * h, h * f, h * f, f * h]
    return layer * c["layers"], [h, h] * c["layers"] + [h]


def _blocks(n):
    return -(-n // 128)


def work(c):
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "norm":  # x, the residual, their sum, the codes with their exponents, the values that these stand for
        n = c["rows"] * c["cols"]
        return {"bytes": n * (3 * size + 1 + 2) + c["rows"] * (4 * _blocks(c["cols"]) + 4) + size * c["cols"], "flops": 0}
    if c["op"] == "norm_backward":
        return {"bytes": c["rows"] * (c["cols"] * size * (4 if c["residual"] else 3) + 4) + c["cols"] * (size + 4), "flops": 0}
    if c["op"] == "clip":
        matrices, norms = _sizes(c)
        return {"bytes": 2 * (size * sum(matrices) + 4 * sum(norms)), "flops": 0}
    m, k, n = c["tokens"], c["inner"], c["outer"]
    if c["op"] == "linear":
        return {"bytes": m * k * size + n * k + 4 * _blocks(n) * _blocks(k) + m * n * (4 if c["out"] == "f32" else 2), "flops": 2 * m * n * k}
    return {"bytes": m * n * size + m * k * 1 + n * k * 1 + 4 * (_blocks(n) + m) * _blocks(k) + m * k * 2 + n * k * 8, "flops": 4 * m * n * k}


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
    return torch.where(amax > 0, torch.clamp(TARGET - (torch.frexp(amax)[1] - 1), -LIMIT, LIMIT), 0).int()


def _in_blocks(x, block_rows):
    """[blocks down, block rows, blocks across, 128], filled up with zeros."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % block_rows))
    return x.view(x.shape[0] // block_rows, block_rows, -1, 128)


def _quantized(x, block_rows):
    """HiF8 values of x * 2^e, and the blocks' exponents e."""
    b = _in_blocks(x, block_rows)
    e = _block_exponent(b.abs().amax((1, 3)))
    r = _rounded(torch.ldexp(b, e[:, None, :, None]))
    return r.reshape(r.shape[0] * block_rows, -1)[:x.shape[0], :x.shape[1]], e


def _spread(e, block_rows, rows, cols):
    """The exponent of each element's block."""
    return e.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def _values(codes, e, block_rows, cols, table):
    """What codes stand for, in 32 bits."""
    x = table[codes[:, :cols].int()]
    return torch.ldexp(x, -_spread(e, block_rows, *x.shape))


def _through(x):
    """What is left of x, [rows, cols], in codes with a scale for each 1 x 128."""
    r, e = _quantized(x.float(), 1)
    return torch.ldexp(r, -_spread(e, 1, *x.shape))


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _bell(g, rows, cols, spread=1.0):
    """Bell-shaped values, a few channels with outliers."""
    x = torch.randn(rows, cols, generator=g, device="cuda").mul_(spread)
    x[:, 5::97] *= 12
    return x


def _padded(n, multiple):
    return -(-n // multiple) * multiple


def _stored(g, rows, cols, block_rows, spread):
    """Codes, their rows a multiple of 16 bytes apart, and exponents."""
    codes = torch.zeros(rows, _padded(cols, 16), dtype=torch.uint8, device="cuda")
    exps = torch.empty(-(-rows // block_rows), _blocks(cols), dtype=torch.int32, device="cuda")
    step = max(128, (1 << 26) // cols // 128 * 128)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        x = torch.randn(n, cols, generator=g, device="cuda").mul_(spread)
        x *= torch.exp2(torch.randint(-2, 3, (1, _blocks(cols)), generator=g, device="cuda").float()).repeat_interleave(128, 1)[:, :cols]
        q, e = _quantized(x, block_rows)
        codes[r:r + n, :cols] = _codes(q)
        exps[r // block_rows:r // block_rows + e.shape[0]] = e
    return codes, exps


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c, "values": _code_values().cuda(), "ws": {}}
    t = TORCH[c["dtype"]]
    if c["op"] in ("norm", "norm_backward"):
        rows, cols = c["rows"], c["cols"]
        s["weight"] = torch.randn(cols, generator=g, device="cuda").mul_(0.2).add_(1.0).to(t)
        if c["op"] == "norm":
            s["x"], s["residual"] = _bell(g, rows, cols, 0.3).to(t), _bell(g, rows, cols).to(t)
            s["h"], s["rstd"] = torch.empty_like(s["x"]), torch.empty(rows, device="cuda")
            s["q"] = torch.empty(rows, _padded(cols, 16), dtype=torch.uint8, device="cuda")
            s["e"] = torch.empty(rows, _blocks(cols), dtype=torch.int32, device="cuda")
            s["back"] = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
        else:
            s["h"], s["dy"] = _bell(g, rows, cols, 1.5).to(t), torch.randn(rows, cols, generator=g, device="cuda").mul_(0.05).to(t)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
            s["dh"] = torch.randn(rows, cols, generator=g, device="cuda").mul_(0.05).to(t) if c["residual"] else None
            s["dx"], s["dweight"] = torch.empty_like(s["h"]), torch.empty(cols, device="cuda")
        return s
    if c["op"] == "clip":
        matrices, norms = _sizes(c)
        s["scale_exp"] = torch.full((1,), 10, dtype=torch.int32, device="cuda")
        s["src"], s["dst"], src, dst, dtypes = [], [], [], [], []
        for sizes, kind, code in ((matrices, t, {"f32": 0, "bf16": 1, "f16": 2}[c["dtype"]]), (norms, torch.float32, 0)):
            n = sum(_padded(k, 8) for k in sizes)
            flat, at = torch.zeros(n, dtype=kind, device="cuda"), 0
            for k in sizes:
                flat[at:at + k] = torch.randn(k, generator=g, device="cuda").mul_(2.0).to(kind)
                src.append(flat.data_ptr() + at * flat.element_size())
                dtypes.append(code)
                at += _padded(k, 8)
            out = torch.zeros_like(flat)
            dst += [p - flat.data_ptr() + out.data_ptr() for p in src[len(dst):]]
            s["src"].append(flat)
            s["dst"].append(out)
        sizes = matrices + norms
        s["from"], s["to"] = torch.tensor(src, device="cuda"), torch.tensor(dst, device="cuda")
        s["dtypes"], s["n"] = torch.tensor(dtypes, dtype=torch.int32, device="cuda"), sum(sizes)
        s["start"] = torch.tensor([0] + sizes, device="cuda").cumsum(0)
        s["norm"], s["found"] = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        return s
    m, k, n = c["tokens"], c["inner"], c["outer"]
    s["w"], s["we"] = _stored(g, n, k, 128, k ** -0.5)
    if c["op"] == "linear":
        out = TORCH[c["out"]]
        s["x"] = _bell(g, m, k).to(t)
        if m > 4:
            s["x"][m // 2] = 0  # a padded token
        s["xq"] = torch.empty(m, _padded(k, 16), dtype=torch.uint8, device="cuda")
        s["xe"] = torch.empty(m, _blocks(k), dtype=torch.int32, device="cuda")
        s["y"] = torch.empty(m, _padded(n, 8), dtype=out, device="cuda")
        return s
    s["xq"], s["xe"] = _stored(g, m, k, 1, 1.0)
    s["dy"] = torch.randn(m, n, generator=g, device="cuda").mul_(0.01).to(t)
    s["dyq"] = torch.empty(m, _padded(n, 16), dtype=torch.uint8, device="cuda")
    s["dye"] = torch.empty(m, _blocks(n), dtype=torch.int32, device="cuda")
    s["dx"] = torch.empty(m, _padded(k, 8), dtype=torch.bfloat16, device="cuda")
    s["dw"] = torch.zeros(n, _padded(k, 8), device="cuda")
    s["dw"][:, :k] = torch.randn(n, k, generator=g, device="cuda").mul_(0.3)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _norm_own, "norm_backward": _norm_backward_own, "linear": _linear_own, "linear_backward": _linear_backward_own, "clip": _clip_own}[op](s)
    return {"norm": _norm, "norm_backward": _norm_backward, "linear": _linear, "linear_backward": _linear_backward, "clip": _clip}[op](s)


def _workspace(s, n):
    """A workspace of that many bytes or more, kept from call to call as a program keeps it."""
    if s["ws"].get("n", -1) < n:
        s["ws"] = {"n": n, "t": torch.empty(n, dtype=torch.uint8, device="cuda")}
    return s["ws"]["t"]


def _dtype(H, name):
    return {"f32": H.F32, "bf16": H.BF16, "f16": H.F16}[name]


def _norm_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    rows, cols, q, e = c["rows"], c["cols"], s["q"], s["e"]
    H.hif8_rmsnorm_encode(s["x"], cols, s["residual"], cols, _dtype(H, c["dtype"]), s["weight"], EPS, rows, cols, s["h"], cols, s["rstd"],
                          q, q.stride(0), e, e.stride(0), TARGET, H.RND_TA, 0)
    H.hif8_block_decode(q, q.stride(0), e, e.stride(0), rows, cols, 1, s["back"], H.BF16, cols)
    return {"h": s["h"], "rstd": s["rstd"], "values": s["back"]}


def _norm_backward_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    rows, cols = c["rows"], c["cols"]
    n = H.hif8_rmsnorm_backward_workspace_bytes(rows, cols)
    H.hif8_rmsnorm_backward(s["dy"], cols, s["h"], cols, s["dh"], cols, _dtype(H, c["dtype"]), s["weight"], s["rstd"], rows, cols, s["dx"], cols, s["dweight"], 0,
                            _workspace(s, n), n)
    return {"dx": s["dx"], "dweight": s["dweight"]}


def _linear_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    m, k, n = c["tokens"], c["inner"], c["outer"]
    x, q, e, w, we, y = s["x"], s["xq"], s["xe"], s["w"], s["we"], s["y"]
    H.hif8_block_encode(x, _dtype(H, c["dtype"]), k, m, k, 1, q, q.stride(0), e, e.stride(0), TARGET, H.RND_TA, 0, 0)
    size = H.hif8_gemm_block_workspace_bytes(m, n, k, 0, 1, 128)
    H.hif8_gemm_block(q, q.stride(0), 0, e, e.stride(0), 1, w, w.stride(0), 1, we, we.stride(0), 128, y, y.stride(0), _dtype(H, c["out"]), m, n, k, 0, _workspace(s, size), size)
    return y[:, :n]


def _linear_backward_own(s):
    import paper_2409_16626_b200 as H

    c = s["case"]
    m, k, n = c["tokens"], c["inner"], c["outer"]
    q, e, w, we, x, xe, dx, dw = s["dyq"], s["dye"], s["w"], s["we"], s["xq"], s["xe"], s["dx"], s["dw"]
    H.hif8_block_encode(s["dy"], _dtype(H, c["dtype"]), n, m, n, 1, q, q.stride(0), e, e.stride(0), TARGET, H.RND_TA, 0, 0)
    size = max(H.hif8_gemm_block_workspace_bytes(m, k, n, 0, 0, 128), H.hif8_gemm_block_workspace_bytes(n, k, m, 1, 0, 1))
    ws = _workspace(s, size)
    H.hif8_gemm_block(q, q.stride(0), 0, e, e.stride(0), 1, w, w.stride(0), 0, we, we.stride(0), 128, dx, dx.stride(0), H.BF16, m, k, n, 0, ws, size)  # dX = dY W
    H.hif8_gemm_block(q, q.stride(0), 1, e, e.stride(0), 1, x, x.stride(0), 0, xe, xe.stride(0), 1, dw, dw.stride(0), H.F32, n, k, m, 1, ws, size)     # dW += dY^T X
    return {"dx": dx[:, :k], "dw": dw[:, :k]}


def _clip_own(s):
    import paper_2409_16626_b200 as H

    n = H.hif8_grad_clip_workspace_bytes()
    H.hif8_grad_clip(s["from"], s["to"], s["dtypes"], s["start"], s["dtypes"].numel(), s["n"], s["scale_exp"], s["case"]["max_norm"], s["norm"], s["found"], _workspace(s, n), n)
    return {"gradients": s["dst"], "norm": s["norm"], "found": s["found"]}


def _norm(s):
    h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
    return {"h": h, "rstd": rstd, "values": _through(h.float() * rstd[:, None] * s["weight"].float()).bfloat16()}


def _norm_backward(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    unit = s["h"].float() * rstd
    wdy = dy * s["weight"].float()
    dx = rstd * (wdy - unit * (wdy * unit).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["h"].dtype), "dweight": (dy * unit).sum(0)}


def _linear(s):
    c = s["case"]
    w = _values(s["w"], s["we"], 128, c["inner"], s["values"])
    return (_through(s["x"]) @ w.T).to(s["y"].dtype)


def _linear_backward(s):
    c = s["case"]
    k = c["inner"]
    dy = _through(s["dy"])
    s["dw"][:, :k] += dy.T @ _values(s["xq"], s["xe"], 1, k, s["values"])
    return {"dx": (dy @ _values(s["w"], s["we"], 128, k, s["values"])).bfloat16(), "dw": s["dw"][:, :k]}


def _clip(s):
    a, b = (x.float() for x in s["src"])
    total = a.square().sum(dtype=torch.float64) + b.square().sum(dtype=torch.float64)
    bad = ~torch.isfinite(total)
    norm = torch.ldexp(total.sqrt(), -s["scale_exp"][0])
    limit = s["case"]["max_norm"]
    factor = torch.ldexp(torch.where(norm > limit, limit / norm, 1.0), -s["scale_exp"][0]).float()
    s["found"].bitwise_or_(bad.int())
    return {"gradients": [torch.where(bad, out.float(), x * factor).to(out.dtype) for x, out in ((a, s["dst"][0]), (b, s["dst"][1]))],
            "norm": torch.where(bad, math.inf, norm).float().view(1), "found": s["found"]}


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


def _nearest(x):
    """Each row's blocks of 128 scaled to the target's binade and moved to the nearest of the format's magnitudes, the larger of two equally near."""
    table = torch.tensor(sorted(v for v in map(_value_of_code, range(128)) if math.isfinite(v)), dtype=torch.float64, device=x.device)
    out = torch.empty_like(x)
    step = max(1, (1 << 25) // max(1, x.shape[0]) // 128) * 128
    for at in range(0, x.shape[1], step):
        part = x[:, at:at + step]
        for j in range(0, part.shape[1], 128):
            b = part[:, j:j + 128]
            top = b.abs().amax(1, keepdim=True)
            e = torch.where(top > 0, TARGET - torch.floor(torch.log2(top)), 0.0).clamp(-LIMIT, LIMIT)
            y = (b.abs() * torch.pow(2.0, e)).contiguous()
            i = torch.searchsorted(table, y).clamp(1, len(table) - 1)
            low, high = table[i - 1], table[i]
            out[:, at + j:at + j + b.shape[1]] = torch.sign(b) * torch.where(high - y <= y - low, high, low) * torch.pow(2.0, -e)
    return out


def _meant(codes, e, block_rows, cols):
    """What stored codes stand for, in 64 bits."""
    table = torch.tensor([_value_of_code(i) for i in range(256)], dtype=torch.float64, device=codes.device)
    out = table[codes[:, :cols].int()]
    factor = torch.pow(2.0, -e.double())
    row = torch.arange(out.shape[0], device=codes.device) // block_rows
    col = torch.arange(cols, device=codes.device) // 128
    return out.mul_(factor[row][:, col])


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "norm":
        h = (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
        d = h.double()
        rstd = 1.0 / torch.sqrt((d * d).sum(1) / c["cols"] + EPS)
        return {"h": h, "rstd": rstd, "values": _nearest(d.mul_(rstd[:, None]).mul_(s["weight"].double()))}
    if c["op"] == "norm_backward":
        n, dweight, out = c["cols"], torch.zeros(c["cols"], dtype=torch.float64, device="cuda"), []
        for at in range(0, c["rows"], 2048):
            rows = slice(at, at + 2048)
            dy, h, r = s["dy"][rows].double(), s["h"][rows].double(), s["rstd"][rows].double()[:, None]
            dweight += torch.einsum("ij,ij,i->j", dy, h, r[:, 0])
            dy *= s["weight"].double()
            dx = r * dy - h * r ** 3 * ((dy * h).sum(1, keepdim=True) / n)
            out.append(dx if s["dh"] is None else dx + s["dh"][rows].double())
        return {"dx": torch.cat(out), "dweight": dweight}
    if c["op"] == "clip":
        a, b = s["src"]
        total = sum(float((x[at:at + (1 << 26)].double() ** 2).sum()) for x in (a, b) for at in range(0, x.numel(), 1 << 26))
        unscale = 2.0 ** -int(s["scale_exp"])
        norm = math.sqrt(total) * unscale
        f = unscale * min(1.0, c["max_norm"] / norm)
        return {"gradients": [a.double() * f, b.double() * f], "norm": torch.tensor([norm], dtype=torch.float64), "found": None}
    m, k, n = c["tokens"], c["inner"], c["outer"]
    w = _meant(s["w"], s["we"], 128, k)
    if c["op"] == "linear":
        return torch.einsum("mk,nk->mn", _nearest(s["x"].double()), w)
    dy = _nearest(s["dy"].double())
    return {"dx": torch.einsum("mn,nk->mk", dy, w), "dw": s["dw"][:, :k].double() + torch.einsum("mn,mk->nk", dy, _meant(s["xq"], s["xe"], 1, k))}
