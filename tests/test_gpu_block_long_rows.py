"""Block-scaled conversions of rows of more than 2^32 columns: what lies behind column 2^32 is that of the same columns by themselves."""
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H

pytestmark = pytest.mark.gpu
COLS = 2 ** 32 + 300
STEP = 2 ** 27
LD = 2 ** 32 + 512


def pieces():
    """Stretches of whole blocks, those at the beginning, around 2^31 and 2^32, and the end."""
    return [(c, min(COLS, c + n)) for c, n in ((0, STEP), (2 ** 31 - 128, STEP), (2 ** 32 - 1024, 512), (2 ** 32 - 128, 428))]


@pytest.mark.parametrize("rows", [1, 2])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shift", [0, 1])
def test_long_rows(rows, block_rows, shift):
    """shift: rows that start on no 16-byte boundary."""
    n = (rows - 1) * LD + COLS + shift
    raw = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    raw.normal_(generator=torch.Generator(device="cuda").manual_seed(rows))
    x = torch.as_strided(raw, (rows, COLS), (LD, 1), shift)
    codes = torch.zeros(n, dtype=torch.uint8, device="cuda")
    q = torch.as_strided(codes, (rows, COLS), (LD, 1), shift)
    e = torch.full((-(-rows // block_rows), -(-COLS // 128)), 99, dtype=torch.int32, device="cuda")
    H.hif8_block_encode(x.data_ptr(), H.BF16, LD, rows, COLS, block_rows, q.data_ptr(), LD, e, e.stride(0))
    for lo, hi in pieces():
        part = x[:, lo:hi].contiguous()
        want, exps = B.encoded(part, H.BF16, block_rows)
        assert torch.equal(q[:, lo:hi], want[:, :hi - lo]) and torch.equal(e[:, lo // 128:-(-hi // 128)], exps)
    raw.fill_(7)
    H.hif8_block_decode(q.data_ptr(), LD, e, e.stride(0), rows, COLS, block_rows, x.data_ptr(), H.BF16, LD)
    for lo, hi in pieces():
        part, exps = q[:, lo:hi].contiguous(), e[:, lo // 128:-(-hi // 128)].contiguous()
        want = torch.empty(rows, hi - lo, dtype=torch.bfloat16, device="cuda")
        H.hif8_block_decode(part, hi - lo, exps, exps.stride(0), rows, hi - lo, block_rows, want, H.BF16, hi - lo)
        assert torch.equal(x[:, lo:hi], want)
    assert rows == 1 or bool((raw[shift + COLS:shift + LD] == 7).all())
