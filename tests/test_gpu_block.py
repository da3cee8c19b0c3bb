"""Conversion to codes with a scale for each 1 x 128 or 128 x 128 elements, and back: the oracle's codes, exponents and values to the last bit."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from oracle import hif8_oracle as O

pytestmark = pytest.mark.gpu
MODES = {H.RND_TA: O.TA, H.RND_HR: O.HR, H.RND_SSR: O.SSR, H.RND_TE: O.TE, H.RND_SR: O.SR}


def matrix(rows, cols, dtype, seed, spread=6):
    """Bell-shaped values, blocks of columns of different spread, a few zeros."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (1, cols), generator=g).float())
    x[torch.rand(rows, cols, generator=g) < 0.02] = 0
    return x.to(B.TORCH[dtype])


def check(x, dtype, block_rows, ld=None, offset=0, ld_q=None, q_offset=0, exp_pad=0, target=3, rnd=H.RND_TA, flags=0, seed=0):
    rows, cols = x.shape
    src = B.Guarded(rows, cols, B.TORCH[dtype], ld, offset, x.cuda())
    q = B.Guarded(rows, cols, torch.uint8, ld_q, q_offset)
    e = B.Guarded(-(-rows // block_rows), -(-cols // 128), torch.int32, -(-cols // 128) + exp_pad)
    H.hif8_block_encode(src.ptr, dtype, src.ld, rows, cols, block_rows, q.ptr, q.ld, e.ptr, e.ld, target, rnd, flags, seed)
    codes, exps = B.encode(x, dtype, block_rows, target, MODES[rnd], flags, seed)
    assert np.array_equal(e.t.cpu().numpy(), exps)
    got = q.t.cpu().numpy()
    assert np.array_equal(got, codes), (np.argwhere(got != codes)[:5], got[got != codes][:5], codes[got != codes][:5])
    q.check()
    e.check()
    for dst in (H.F32, H.BF16, H.F16):
        back = B.Guarded(rows, cols, B.TORCH[dst], ld, offset)
        H.hif8_block_decode(q.ptr, q.ld, e.ptr, e.ld, rows, cols, block_rows, back.ptr, dst, back.ld)
        want = torch.from_numpy(B.meant(codes, exps, block_rows)).to(B.TORCH[dst])
        assert torch.equal(back.t.cpu().nan_to_num(nan=77.0), want.nan_to_num(nan=77.0))
        back.check()


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (1, 4096), (3, 129), (129, 8), (130, 1000), (257, 390)])
def test_codes_exponents_and_values(rows, cols, dtype, block_rows):
    check(matrix(rows, cols, dtype, rows + cols), dtype, block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rnd", list(MODES))
def test_roundings(rnd, dtype, block_rows):
    check(matrix(131, 262, dtype, 5), dtype, block_rows, target=6, rnd=rnd, seed=0x1234567890)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("ld,offset,ld_q,q_offset", [(264, 0, 272, 8), (257, 1, 259, 3), (272, 4, 264, 0), (256, 0, 257, 0)])
def test_strides_and_alignments(ld, offset, ld_q, q_offset, dtype, block_rows):
    check(matrix(140, 256, dtype, 7), dtype, block_rows, ld, offset, ld_q, q_offset, exp_pad=3)


@pytest.mark.parametrize("flags", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
def test_inf_nan_and_zeros(dtype, flags):
    x = matrix(136, 300, dtype, 9)
    x[3, 5], x[3, 140], x[4, 200], x[130, 0] = float("inf"), float("-inf"), float("nan"), float("nan")
    x[7] = 0
    x[8, :128] = float("nan")            # a block without a finite value
    x[128:, 128:256] = 0                 # a tile of zeros
    for block_rows in (1, 128):
        check(x, dtype, block_rows, flags=flags)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16])
def test_exponents_end_at_their_limits(dtype):
    x = matrix(4, 640, dtype, 11)
    x *= torch.exp2(torch.tensor([-149.0 + 30, -100.0, 0.0, 90.0, 110.0])).repeat_interleave(128).to(x.dtype)
    for block_rows in (1, 128):
        for target in (-22, 3, 15):
            check(x, dtype, block_rows, target=target)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
def test_many_blocks(dtype):
    """More blocks than are taken at once: tiles and rows in several rounds."""
    g = torch.Generator().manual_seed(13)
    x = torch.randn(1500, 16000, generator=g).to(B.TORCH[dtype]).cuda()
    for block_rows in (1, 128):
        q, e = B.encoded(x, dtype, block_rows)
        top = torch.nn.functional.pad(x.float().abs(), (0, 0, 0, -1500 % block_rows)).view(-1, block_rows, 125, 128).amax((1, 3))
        assert torch.equal(e, (3 - (torch.frexp(top)[1] - 1)).int())
        back = torch.empty(1500, 16000, device="cuda")
        H.hif8_block_decode(q, q.stride(0), e, e.stride(0), 1500, 16000, block_rows, back, H.F32, 16000)
        up = e.repeat_interleave(block_rows, 0)[:1500].repeat_interleave(128, 1)
        scaled = torch.ldexp(x.float(), up)
        grid = torch.from_numpy(B.GRID).cuda()
        k = torch.searchsorted(grid, scaled.double().abs()).clamp(1, len(grid) - 1)
        low, high, a = grid[k - 1], grid[k], scaled.double().abs()
        want = torch.where(high - a <= a - low, high, low) * torch.sign(scaled)
        assert torch.equal(torch.ldexp(back, up).double(), want)


def test_on_another_stream_and_in_a_graph():
    x = matrix(200, 500, H.BF16, 15).cuda()
    want, we = B.encoded(x, H.BF16, 1)
    q, e, back = torch.zeros_like(want), torch.zeros_like(we), torch.zeros(200, 500, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def both(stream):
        H.hif8_block_encode(x, H.BF16, 500, 200, 500, 1, q, q.stride(0), e, e.stride(0), 3, H.RND_TA, 0, 0, stream)
        H.hif8_block_decode(q, q.stride(0), e, e.stride(0), 200, 500, 1, back, H.F32, 500, stream)

    both(side)
    torch.cuda.synchronize()
    assert torch.equal(q[:, :500], want[:, :500]) and torch.equal(e, we)
    first = back.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(None)
    for t in (q, e, back):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q[:, :500], want[:, :500]) and torch.equal(e, we) and torch.equal(back, first)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_rows_far_apart(block_rows):
    """Offsets beyond 32 bits: 2^31 elements of the source, 2^32 bytes of codes and 2^30 exponents between rows."""
    x = matrix(3, 200, H.BF16, 17)
    src = torch.zeros(2 * 2 ** 31 + 200, dtype=torch.bfloat16, device="cuda")
    torch.as_strided(src, (3, 200), (2 ** 31, 1)).copy_(x)
    q, e = torch.zeros(2 * 2 ** 32 + 200, dtype=torch.uint8, device="cuda"), torch.zeros(2 * 2 ** 30 + 2, dtype=torch.int32, device="cuda")
    H.hif8_block_encode(src, H.BF16, 2 ** 31, 3, 200, block_rows, q, 2 ** 32, e, 2 ** 30)
    codes, exps = B.encode(x, H.BF16, block_rows)
    down = exps.shape[0]
    assert np.array_equal(torch.as_strided(q, (3, 200), (2 ** 32, 1)).cpu().numpy(), codes) and np.array_equal(torch.as_strided(e, (down, 2), (2 ** 30, 1)).cpu().numpy(), exps)
    src.zero_()
    H.hif8_block_decode(q, 2 ** 32, e, 2 ** 30, 3, 200, block_rows, src, H.BF16, 2 ** 31)
    assert torch.equal(torch.as_strided(src, (3, 200), (2 ** 31, 1)).cpu(), torch.from_numpy(B.meant(codes, exps, block_rows)).bfloat16())


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rows,cols", [(1, 95), (2, 97), (3, 383), (3, 385), (5, 390), (2, 512), (130, 513), (3, 1101), (1, 4097)])
def test_unaligned_rows(rows, cols, dtype, block_rows):
    check(matrix(rows, cols, dtype, rows + cols), dtype, block_rows, ld=cols | 1, offset=1, ld_q=cols + 3, q_offset=3, exp_pad=1)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rnd", list(MODES))
def test_roundings_of_unaligned_rows(rnd, dtype):
    check(matrix(9, 700, dtype, 19), dtype, 1, ld=701, offset=3, ld_q=703, q_offset=1, target=6, rnd=rnd, seed=0x1234567890)


@pytest.mark.parametrize("flags", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
def test_inf_nan_and_zeros_in_unaligned_rows(dtype, flags):
    x = matrix(6, 600, dtype, 21)
    x[0, 5], x[1, 140], x[2, 599], x[3, 0] = float("inf"), float("-inf"), float("nan"), float("nan")
    x[4] = 0
    x[5, 128:256] = float("nan")
    check(x, dtype, 1, flags=flags, ld=601, offset=1, ld_q=605, q_offset=1)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
def test_many_unaligned_rows_are_those_of_aligned_ones(dtype):
    """More rows than are taken at once."""
    x = torch.randn(9000, 1500, generator=torch.Generator().manual_seed(23)).to(B.TORCH[dtype]).cuda()
    q, e = B.encoded(x, dtype, 1)
    src = torch.zeros(1 + 9000 * 1503, dtype=x.dtype, device="cuda")
    codes, exps = torch.zeros(1 + 9000 * 1501, dtype=torch.uint8, device="cuda"), torch.zeros_like(e)
    far, out = torch.as_strided(src, (9000, 1500), (1503, 1), 1), torch.as_strided(codes, (9000, 1500), (1501, 1), 1)
    far.copy_(x)
    H.hif8_block_encode(far.data_ptr(), dtype, 1503, 9000, 1500, 1, out.data_ptr(), 1501, exps, exps.stride(0))
    assert torch.equal(out, q[:, :1500]) and torch.equal(exps, e)
    back = torch.empty(9000, 1500, dtype=x.dtype, device="cuda")
    H.hif8_block_decode(q, q.stride(0), e, e.stride(0), 9000, 1500, 1, back, dtype, 1500)
    src.zero_()
    H.hif8_block_decode(out.data_ptr(), 1501, exps, exps.stride(0), 9000, 1500, 1, far.data_ptr(), dtype, 1503)
    assert torch.equal(far, back) and bool((torch.as_strided(src, (8999, 3), (1503, 1), 1501) == 0).all())
