"""How large a matrix each call on block-scaled matrices takes: refused for its shape beyond, and at the limit for something that is looked at later (an address that is not aligned), so
that nothing is launched."""
import pytest

import paper_2409_16626_b200 as H
from paper_2409_16626_b200 import binding
from test_block_host import ALIGN, CALLS, SHAPE

M = 1 << 20
BLOCKS, GROUPS, ROWS, DIM, EXPANDED = 2 ** 31 - 1, 2 ** 31 - 1, 32 * (2 ** 31 - 1), 2 ** 31 - 4096, 2 ** 30 - 2 ** 20


def encode(rows, cols, block_rows):
    return "encode", dict(rows=rows, cols=cols, block_rows=block_rows, ld_src=cols, ld_dst=cols, exp_stride=-(-cols // 128), src=16 * M + 1)


def decode(rows, cols, block_rows=1):
    return "decode", dict(rows=rows, cols=cols, block_rows=block_rows, ld_src=cols, ld_dst=cols, exp_stride=-(-cols // 128), dst=16 * M + 2)


def norm(rows):
    return "norm", dict(rows=rows, x=16 * M + 1)


def backward(rows):
    return "backward", dict(rows=rows, dy=16 * M + 1)


def gemm(m, n, k, a_is_km=0, w_is_nk=1, w_block_rows=128):
    pad = lambda v: -(-v // 16) * 16  # noqa: E731
    return "gemm", dict(M=m, N=n, K=k, a_is_km=a_is_km, w_is_nk=w_is_nk, w_block_rows=w_block_rows, lda=pad(m if a_is_km else k), ldw=pad(k if w_is_nk else n), ldc=pad(n),
                        exp_stride_a=2 ** 24, exp_stride_w=2 ** 24, Aq=16 * M + 8)


@pytest.mark.parametrize("call,status", [
    (encode(1, 128 * BLOCKS, 1), ALIGN), (encode(1, 128 * BLOCKS + 1, 1), SHAPE), (encode(BLOCKS, 128, 1), ALIGN), (encode(BLOCKS, 129, 1), SHAPE), (encode(BLOCKS + 1, 1, 1), SHAPE),
    (encode(128 * BLOCKS, 128, 128), ALIGN), (encode(128 * BLOCKS + 1, 128, 128), SHAPE), (encode(128, 128 * BLOCKS, 128), ALIGN), (encode(129, 128 * BLOCKS, 128), SHAPE),
    (decode(1, 16 * GROUPS), ALIGN), (decode(1, 16 * GROUPS + 1), SHAPE), (decode(GROUPS, 16), ALIGN), (decode(GROUPS, 17), SHAPE), (decode(GROUPS + 1, 1), SHAPE), (decode(GROUPS + 1, 1, 128), SHAPE),
    (norm(ROWS), ALIGN), (norm(ROWS + 1), SHAPE), (backward(ROWS), ALIGN), (backward(ROWS + 1), SHAPE),
    (gemm(1, DIM, 1), ALIGN), (gemm(1, DIM + 1, 1), SHAPE), (gemm(1, 1, DIM), ALIGN), (gemm(1, 1, DIM + 1), SHAPE), (gemm(DIM, 1, 1, 1), ALIGN), (gemm(DIM + 1, 1, 1, 1), SHAPE),
    (gemm(1, 1, 2 ** 31 - 1), SHAPE), (gemm(2 ** 31 - 1, 1, 1, 1), SHAPE), (gemm(1, 2 ** 31 - 1, 1), SHAPE),
    (gemm(EXPANDED, 1, 16), ALIGN), (gemm(EXPANDED, 1, 17), SHAPE), (gemm(EXPANDED + 1, 1, 1), SHAPE), (gemm(EXPANDED + 1, 1, 1, 1), ALIGN), (gemm(16, 1, EXPANDED + 1, 1), ALIGN),
    (gemm(16, 1, EXPANDED, 1, 1, 1), ALIGN), (gemm(16, 1, EXPANDED + 1, 1, 1, 1), SHAPE), (gemm(1, EXPANDED, 16, 0, 1, 1), ALIGN), (gemm(1, EXPANDED + 1, 16, 0, 1, 1), SHAPE),
    (gemm(1, 1, EXPANDED * 2, 0, 1, 1), ALIGN), (gemm(1, 1, EXPANDED * 2 + 1, 0, 1, 1), SHAPE), (gemm(1, 9, EXPANDED + 1, 0, 1, 1), SHAPE), (gemm(1, 16, EXPANDED, 0, 0, 1), ALIGN), (gemm(1, 17, EXPANDED, 0, 0, 1), SHAPE), (gemm(1, EXPANDED + 1, 16), ALIGN)])
def test_limits(call, status):
    name, change = call
    fn, good = CALLS[name]
    before = H.hif8_launch_count()
    assert fn(**{**good, **change}, stream=0, check=False) == status
    assert H.hif8_launch_count() == before


def test_large_weights_that_are_decoded_in_the_kernel_have_no_copy():
    """Where an operand is too large to be expanded the workspace has room for the activations alone."""
    size = binding.lib.hif8_gemm_block_workspace_bytes
    assert size(600, 2 ** 20, 2 ** 14, 0, 1, 128) == 256 + 600 * 2 ** 14 * 2
    assert size(600, 2 ** 20 - 2 ** 12, 2 ** 14, 0, 1, 128) == 256 + 600 * 2 ** 14 * 2 + (2 ** 20 - 2 ** 12) * 2 ** 14 * 2


@pytest.mark.parametrize("shape", [(2 ** 31 - 1, 1, 1), (1, 2 ** 31 - 1, 1), (1, 1, 2 ** 31 - 1)])
def test_sizes_of_workspaces_do_not_wrap(shape):
    m, n, k = shape
    for a_is_km in (0, 1):
        for w_is_nk in (0, 1):
            for blocks in (1, 128):
                assert binding.lib.hif8_gemm_block_workspace_bytes(m, n, k, a_is_km, w_is_nk, blocks) >= 256 + 2 * m * k
