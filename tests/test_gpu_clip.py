"""The global norm of a list of gradients under a loss scale, and clipping, against 64 bits."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H

pytestmark = pytest.mark.gpu
SHIFT = {H.F32: 4, H.BF16: 2, H.F16: 2}


class Gradients:
    """Tensors in two buffers (gradients, results), each `gaps` elements behind the one before; bytes between them are a pattern."""

    def __init__(self, sizes, dtypes, seed, spread=1.0, gap=8, offset=0, values=None):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.dtypes, at = sizes, dtypes, 64 + 4 * offset
        self.host, where = [], []
        for i, (n, d) in enumerate(zip(sizes, dtypes)):
            x = (torch.randn(n, generator=g) * spread).to(B.TORCH[d])
            if values and i in values:
                x[values[i][0]] = values[i][1]
            self.host.append(x)
            where.append(at)
            at += -(-(n * SHIFT[d] + SHIFT[d] * gap) // 4) * 4 if gap % 8 else (n * SHIFT[d] + 31) // 16 * 16
        self.src, self.dst = torch.full((at + 64,), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((at + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        self.where = where
        for x, t in zip(self.host, self.views(self.src)):
            t.copy_(x)
        ints = lambda v, t: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
        self.d_src, self.d_dst = (ints([b.data_ptr() + w for w in where], torch.int64) for b in (self.src, self.dst))
        self.d_dtype = ints(dtypes, torch.int32)
        self.d_start = ints([0] + list(np.cumsum(sizes)), torch.int64)
        self.n = int(sum(sizes))
        self.norm, self.found = torch.full((1,), -1.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = torch.full((H.hif8_grad_clip_workspace_bytes(),), 0xFF, dtype=torch.uint8, device="cuda")

    def views(self, buffer):
        return [buffer[w:w + n * SHIFT[d]].view(B.TORCH[d]) for w, n, d in zip(self.where, self.sizes, self.dtypes)]

    def call(self, max_norm, scale_exp=None, in_place=False, null_dst=False):
        se = None if scale_exp is None else torch.tensor([scale_exp], dtype=torch.int32, device="cuda")
        H.hif8_grad_clip(self.d_src, None if null_dst else self.d_src if in_place else self.d_dst, self.d_dtype, self.d_start, len(self.sizes), self.n, se, max_norm, self.norm, self.found,
                         self.ws, self.ws.numel())
        torch.cuda.synchronize()

    def untouched(self, buffer):
        mask = torch.ones(buffer.numel(), dtype=torch.bool)
        for w, n, d in zip(self.where, self.sizes, self.dtypes):
            mask[w:w + n * SHIFT[d]] = False
        assert bool((buffer.cpu()[mask] == 0xA5).all())

    def check(self, max_norm, scale_exp=0, buffer=None):
        with np.errstate(over="ignore"):
            total = sum(float((x.double() ** 2).sum()) for x in self.host)
        norm = np.sqrt(total) * 2.0 ** -scale_exp
        # FP32 sums over four or eight squares (each rounding halved by the root), the norm rounded once; the factor and its product once each
        if norm > torch.finfo(torch.float32).max:
            assert float(self.norm) == float("inf")
        else:
            assert abs(float(self.norm) - norm) <= 6 * B.U32 * norm + 2.0 ** -150
        assert int(self.found) == 0
        f = 2.0 ** -scale_exp * (max_norm / norm if norm > max_norm else 1.0)
        for x, got, d in zip(self.host, self.views(self.dst if buffer is None else buffer), self.dtypes):
            want = x.double() * f
            half = torch.finfo(B.TORCH[d]).eps / 2
            tiny = {H.F32: 2.0 ** -149, H.BF16: 2.0 ** -134, H.F16: 2.0 ** -25}[d]
            assert bool(((got.cpu().double() - want).abs() <= (half + 8 * B.U32) * want.abs() + tiny).all())
        self.untouched(self.dst if buffer is None else buffer)


ALL = [H.F32, H.BF16, H.F16]


@pytest.mark.parametrize("sizes,dtypes", [([1], [H.F32]), ([7], [H.BF16]), ([0, 5, 0, 0, 3000, 1, 0], [H.F16, H.F32, H.BF16, H.F32, H.BF16, H.F16, H.F32]), ([100000], [H.F16]), ([3_000_001, 17, 123457], ALL),
                                          ([64] * 300, ALL * 100), ([1] * 5000, [H.F32] * 5000), ([2048, 2048, 4096, 1], [H.BF16] * 4)])
@pytest.mark.parametrize("max_norm,scale_exp", [(1.0, None), (1.0, 12), (1e9, 5), (float("inf"), -3), (1e-3, 0)])
def test_norm_and_results(sizes, dtypes, max_norm, scale_exp):
    g = Gradients(sizes, dtypes, len(sizes))
    g.call(max_norm, scale_exp)
    g.check(max_norm, scale_exp or 0)
    g.untouched(g.src)
    for x, t in zip(g.host, g.views(g.src)):
        assert torch.equal(t.cpu(), x)


@pytest.mark.parametrize("null_dst", [False, True])
@pytest.mark.parametrize("max_norm,scale_exp", [(1.0, 3), (1e9, 0)])
def test_in_place(max_norm, scale_exp, null_dst):
    g = Gradients([1000, 70000, 3, 5001], [H.F32, H.BF16, H.F16, H.F16], 3)
    g.call(max_norm, scale_exp, in_place=True, null_dst=null_dst)
    g.check(max_norm, scale_exp, g.src)
    assert bool((g.dst == 0xA5).all())
    if scale_exp == 0:                                   # nothing to clip and nothing to unscale: the same bits
        assert all(torch.equal(t.cpu(), x) for x, t in zip(g.host, g.views(g.src)))


@pytest.mark.parametrize("gap,offset", [(3, 0), (5, 1), (8, 1)])
def test_alignments(gap, offset):
    g = Gradients([1001, 70003, 3, 5001], [H.F32, H.BF16, H.F16, H.F32], 5, gap=gap, offset=offset)
    g.call(1.0, 2)
    g.check(1.0, 2)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("tensor,at", [(0, 0), (1, 69999), (2, 2), (3, 4999)])
def test_not_finite(tensor, at, value):
    g = Gradients([1000, 70000, 3, 5000], [H.F32, H.BF16, H.F16, H.F32], 7, values={tensor: (at, value)})
    g.found.fill_(2)
    g.call(1.0, 4)
    assert float(g.norm) == float("inf") and int(g.found) == 3 and bool((g.dst == 0xA5).all())


@pytest.mark.parametrize("spread", [1e-30, 1e-41, 1e19, 1e37])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16])
def test_squares_beyond_32_bits(dtype, spread):
    g = Gradients([5000, 333], [dtype, H.F32], 9, spread=spread)
    g.call(float(np.float32(spread)), 0)
    g.check(float(np.float32(spread)))
    g.call(float("inf"), 20 if spread > 1 else -20)
    g.check(float("inf"), 20 if spread > 1 else -20)


def test_zeros_and_nothing():
    g = Gradients([1000, 50], [H.F32, H.BF16], 11, spread=0.0)
    g.call(1.0, 3)
    assert float(g.norm) == 0 and int(g.found) == 0 and all(bool((t == 0).all()) for t in g.views(g.dst))
    for n, total in ((0, 0), (2, 0)):
        g.norm.fill_(-1)
        H.hif8_grad_clip(g.d_src, g.d_dst, g.d_dtype, torch.zeros(3, dtype=torch.int64, device="cuda"), n, total, None, 1.0, g.norm, None, g.ws, g.ws.numel())
        assert float(g.norm) == 0


@pytest.mark.parametrize("what", ["format", "address", "no address", "no result"])
def test_what_is_no_tensor_is_left_out(what):
    g = Gradients([1000, 50, 70], [H.F32, H.BF16, H.F32], 13)
    if what == "format":
        g.d_dtype[0] = 9
    elif what == "address":
        g.d_src[0] += 2
    elif what == "no address":
        g.d_src[0] = 0
    else:
        g.d_dst[0] = 0
    g.call(1e9)
    want = np.sqrt(sum(float((x.double() ** 2).sum()) for x in g.host[1:]))
    assert abs(float(g.norm) - want) < 1e-5 * want and bool((g.dst[:g.where[1]] == 0xA5).all())


def test_loss_scale_state_and_controller():
    """The scale is the controller's first int; what it finds is what the controller takes."""
    state, g = torch.empty(H.ALS_STATE_BYTES, dtype=torch.uint8, device="cuda"), Gradients([4000, 300], [H.F32, H.BF16], 15)
    H.hif8_als_state_init(state, 7, 0)
    scale = state.view(torch.int32)[:1]
    H.hif8_grad_clip(g.d_src, g.d_dst, g.d_dtype, g.d_start, 2, g.n, scale, 0.25, g.norm, g.found, g.ws, g.ws.numel())
    g.check(0.25, 7)
    g.views(g.src)[0][5] = float("inf")
    H.hif8_grad_clip(g.d_src, g.d_dst, g.d_dtype, g.d_start, 2, g.n, scale, 0.25, g.norm, g.found, g.ws, g.ws.numel())
    H.hif8_als_update(state, g.found)
    assert int(scale) == 6 and int(g.found) == 0


def test_captured_and_reproducible():
    g = Gradients([300001, 17, 5000], ALL, 17)
    g.call(1.0, 2)
    first, norm = g.dst.clone(), float(g.norm)
    graph = torch.cuda.CUDAGraph()
    se = torch.tensor([2], dtype=torch.int32, device="cuda")
    with torch.cuda.graph(graph):
        H.hif8_grad_clip(g.d_src, g.d_dst, g.d_dtype, g.d_start, 3, g.n, se, 1.0, g.norm, g.found, g.ws, g.ws.numel())
    g.dst.fill_(0xA5)
    g.ws.fill_(0xFF)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g.dst, first) and float(g.norm) == norm


@pytest.mark.parametrize("sizes,dtypes", [([45_000_003], [H.BF16]), ([13_000_001, 9_000_000, 77], ALL)])
@pytest.mark.parametrize("in_place", [False, True])
def test_long_shares(sizes, dtypes, in_place):
    g = Gradients(sizes, dtypes, 9)
    g.call(1.0, 4, in_place=in_place)
    g.check(1.0, 4, g.src if in_place else None)
