"""Plain implementations in 64 bits of the operators on block-scaled matrices, on the CPU: matrices of codes with a scale for each 1 x 128 or
128 x 128 elements, products of them, the norm in front of them and its gradient, clipping."""
import numpy as np
import torch

import paper_2409_16626_b200 as H
from oracle import hif8_oracle as O

TORCH = {H.F32: torch.float32, H.BF16: torch.bfloat16, H.F16: torch.float16}
VALUES = np.array([O.value(c) for c in range(256)])
GRID = np.unique(np.abs(VALUES[np.isfinite(VALUES)]))  # the format's finite magnitudes
U32 = 2.0 ** -24                                        # half a step of FP32, relative


def bits(t):
    """A CPU tensor's encodings, as the oracle takes them."""
    t = t.contiguous()
    return t.numpy() if t.dtype == torch.float32 else t.view(torch.int16).numpy().view(np.uint16)


def blocks_of(rows, cols, block_rows):
    for i in range(0, rows, block_rows):
        for j in range(0, cols, 128):
            yield i // block_rows, j // 128, slice(i, min(rows, i + block_rows)), slice(j, min(cols, j + 128))


def encode(x, dtype, block_rows, target=3, rnd=O.TA, flags=0, seed=0):
    """(codes, exponents) of a CPU tensor [rows, cols], by the oracle block by block."""
    rows, cols = x.shape
    codes = np.zeros((rows, cols), np.uint8)
    exps = np.zeros((-(-rows // block_rows), -(-cols // 128)), np.int32)
    flat = np.arange(rows * cols, dtype=np.uint64).reshape(rows, cols)
    for i, j, r, c in blocks_of(rows, cols, block_rows):
        b = bits(x[r, c])
        e = max(-H.BLOCK_EXP_MAX, min(H.BLOCK_EXP_MAX, O.amax_scale(b.ravel(), dtype, target)[1]))
        exps[i, j] = e
        codes[r, c] = O.encode_at(b.ravel(), dtype, flat[r, c].ravel(), e, rnd, flags, seed, quick=True).reshape(b.shape)
    return codes, exps


def meant(codes, exps, block_rows):
    """What codes stand for, in 64 bits."""
    rows, cols = codes.shape
    e = np.clip(exps, -H.BLOCK_EXP_MAX, H.BLOCK_EXP_MAX).astype(np.float64)
    return VALUES[codes] * 2.0 ** -np.repeat(np.repeat(e, block_rows, 0)[:rows], 128, 1)[:, :cols]


def nearest(y):
    """Nearest of the format's values, halves away from zero (finite y below 1.5 * 2^15)."""
    a = np.abs(y)
    k = np.clip(np.searchsorted(GRID, a), 1, len(GRID) - 1)
    low, high = GRID[k - 1], GRID[k]
    return np.sign(y) * np.where(high - a <= a - low, high, low)


def norm(x, residual, weight, eps, dtype):
    """(h as a tensor of its type, r, h * r * weight in 64 bits)"""
    h = x if residual is None else (x.float() + residual.float()).to(TORCH[dtype])
    d = h.double().numpy()
    r = 1.0 / np.sqrt((d * d).mean(1) + float(np.float32(eps)))
    return h, r, d * r[:, None] * weight.double().numpy()


def norm_backward(dy, h, dh, weight, r):
    """(dx, its rounding's scale, dweight, its scale) in 64 bits; r as given."""
    dy, u, w = dy.double().numpy(), h.double().numpy() * r[:, None], weight.double().numpy()
    wdy = dy * w
    dx = r[:, None] * (wdy - u * (wdy * u).mean(1, keepdims=True))
    scale = r[:, None] * (np.abs(wdy) + np.abs(u) * np.abs(wdy * u).mean(1, keepdims=True))
    if dh is not None:
        dx, scale = dx + dh.double().numpy(), scale + np.abs(dh.double().numpy())
    return dx, scale, (dy * u).sum(0), np.abs(dy * u).sum(0)


class Guarded:
    """A [rows, cols] CUDA tensor whose rows lie `ld` elements apart, `offset` elements into a buffer that is filled with a pattern: what lies between and around the rows has to stay."""

    def __init__(self, rows, cols, dtype, ld=None, offset=0, values=None):
        self.ld = cols if ld is None else ld
        n = offset + max(0, rows - 1) * self.ld + cols + 16
        self.raw = torch.full((n * torch.empty(0, dtype=dtype).element_size(),), 0xA5, dtype=torch.uint8, device="cuda")
        self.flat = self.raw.view(dtype)
        self.t = torch.as_strided(self.flat, (rows, cols), (self.ld, 1), offset)
        if values is not None:
            self.t.copy_(values)
        self.before = self.raw.clone()

    @property
    def ptr(self):
        return self.t.data_ptr()

    def check(self):
        """Nothing but the matrix has changed."""
        mask = torch.ones_like(self.flat, dtype=torch.bool)
        torch.as_strided(mask, self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(False)
        was = self.before.view(self.flat.dtype)
        size = self.flat.element_size()
        bytes_of = lambda t: t[mask].contiguous().view(torch.uint8) if size > 1 else t[mask]  # noqa: E731
        assert torch.equal(bytes_of(self.flat), bytes_of(was)), "write outside the matrix"


def encoded(x, dtype, block_rows, ld=None, rnd=H.RND_TA, target=3):
    """(codes, exponents) tensors of a CUDA matrix, by the library."""
    rows, cols = x.shape
    q = torch.empty(rows, ld or -(-cols // 16) * 16, dtype=torch.uint8, device="cuda")
    e = torch.empty(-(-rows // block_rows), -(-cols // 128), dtype=torch.int32, device="cuda")
    H.hif8_block_encode(x, dtype, x.stride(0), rows, cols, block_rows, q, q.stride(0), e, e.stride(0), target, rnd)
    return q, e


def product(q, e, a_is_km, qb, w, we, w_is_nk, wb, M, N, K, c_dtype=H.F32, C=None, accumulate=0, ws=None):
    """A block-scaled product into C (its rows padded to 16 bytes)."""
    if C is None:
        C = torch.empty(M, -(-N // 8) * 8, dtype=TORCH[c_dtype], device="cuda")
    n = H.hif8_gemm_block_workspace_bytes(M, N, K, a_is_km, w_is_nk, wb)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if ws is None else ws
    H.hif8_gemm_block(q, q.stride(0), a_is_km, e, e.stride(0), qb, w, w.stride(0), w_is_nk, we, we.stride(0), wb, C, C.stride(0), c_dtype, M, N, K, accumulate, ws, n)
    return C
