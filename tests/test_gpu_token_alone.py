"""A token's norm alone and among others: the same bits where its row is added in the same order, otherwise within what the sums' roundings allow; products always from the codes made."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from test_gpu_norm import SUM, call, inputs

pytestmark = pytest.mark.gpu
FEW = 148  # rows up to which long rows have more threads


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("cols", [8, 264, 512, 131, 8200, 9001, 16384])
def test_rows_added_in_the_same_order_have_the_same_bits(cols, dtype):
    x, r, w = inputs(FEW + 10, cols, dtype, cols)
    many = call(x, r, w, dtype)
    for part in (slice(0, 1), slice(77, 78), slice(0, FEW), slice(FEW + 9, FEW + 10)):
        few = call(x[part], r[part], w, dtype)
        assert torch.equal(many[0][part], few[0]) and all(np.array_equal(a[part], b) for a, b in zip(many[1:], few[1:]))


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("cols", [520, 1001, 4096, 8192])
def test_rows_added_in_another_order(cols, dtype):
    x, r, w = inputs(FEW + 10, cols, dtype, cols)
    h, rstd, codes, exps = call(x, r, w, dtype)
    y = B.norm(x, r, w, 1e-5, dtype)[2]
    off = SUM / 2 + 6 * B.U32                             # of a value in front of its rounding, either way
    assert torch.equal(h[:FEW], call(x[:FEW], r[:FEW], w, dtype)[0])
    for t in (0, 77, FEW - 1, FEW + 9):
        one = call(x[t:t + 1], r[t:t + 1], w, dtype)
        assert torch.equal(one[0][0], h[t]) and abs(float(one[1][0]) - float(rstd[t])) <= 2 * (SUM / 2 + 3 * B.U32) * float(rstd[t])
        for e, q in ((one[3][0], one[2][0]), (exps[t], codes[t])):
            scaled = y[t] * 2.0 ** np.repeat(e.astype(float), 128)[:cols]
            got = B.VALUES[q]
            assert np.all((got == B.nearest(scaled * (1 - off))) | (got == B.nearest(scaled * (1 + off))) | (got == B.nearest(scaled)))
        differ = one[2][0] != codes[t]
        assert differ.sum() <= cols // 100 + 1            # (on a border of two values or in a block whose largest is on one of two binades: below one in 10^5)


@pytest.mark.parametrize("cols,outer", [(264, 392), (4096, 512)])
def test_products_of_the_codes_made(cols, outer):
    x, r, w = inputs(FEW + 2, cols, H.BF16, cols)
    g = torch.Generator(device="cuda").manual_seed(cols)
    wq, we = B.encoded(torch.randn(outer, cols, generator=g, device="cuda") * 0.05, H.F32, 128)
    wv = B.meant(wq.cpu().numpy()[:, :cols], we.cpu().numpy(), 128)
    many = call(x, r, w, H.BF16)
    for t in (0, 77, FEW + 1):
        for rows in (slice(t, t + 1), slice(0, FEW + 2)):
            _, _, codes, exps = call(x[rows], r[rows], w, H.BF16) if rows != slice(0, FEW + 2) else many
            q, e = torch.zeros(codes.shape[0], -(-cols // 16) * 16, dtype=torch.uint8, device="cuda"), torch.from_numpy(exps.copy()).cuda()
            q[:, :cols] = torch.from_numpy(codes).cuda()
            y = B.product(q, e, 0, 1, wq, we, 1, 128, codes.shape[0], outer, cols, H.BF16)
            row = 0 if codes.shape[0] == 1 else t
            a = B.meant(codes[row:row + 1], exps[row:row + 1], 1)
            want, scale = (a @ wv.T)[0], (np.abs(a) @ np.abs(wv).T)[0]
            bound = max(1e-5, -(-cols // 16) * 2.0 ** -23)
            assert np.all(np.abs(y[row, :outer].cpu().double().numpy() - want) <= 2.0 ** -8 * 1.01 * np.abs(want) + bound * scale)
