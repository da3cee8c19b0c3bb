"""The norm's gradient where its operands are far from 1 and its results are not: no product on the way leaves FP32.  Tolerances as in the other tests of the gradient, and half a step of
the result's type where it is subnormal."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from test_gpu_norm import SUM, gradient, inputs

pytestmark = pytest.mark.gpu
# scales of h and of dy: dy h beyond FP32; dy h subnormal; dy r subnormal (and so is dx, but not the weight's gradient); both at once, dx near 1
SCALES = [(60, 70), (-60, -83), (60, -73), (-60, -60), (60, 60)]


@pytest.mark.parametrize("dtype", [H.F32, H.BF16])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("rows,cols", [(5, 128), (7, 1001), (20, 4096), (3, 8192), (4, 9000), (2, 20000)])
def test_operands_far_from_one(rows, cols, residual, dtype):
    for k, (h_exp, dy_exp) in enumerate(SCALES):
        h, dy, w = inputs(rows, cols, dtype, rows + cols + k)
        h, dy = h * 2.0 ** h_exp, dy * 2.0 ** dy_exp
        dh = dy * 2.0 ** -h_exp if residual else None   # (about as large as dx)
        r = B.norm(h, None, w, 0.0, dtype)[1].astype(np.float32)
        dx, dweight = gradient(dy, h, dh, w, r, dtype)
        want, scale, dw, dw_scale = B.norm_backward(dy, h, dh, w, r.astype(np.float64))
        half = torch.finfo(B.TORCH[dtype]).eps / 2
        tiny = {H.F32: 2.0 ** -150, H.BF16: 2.0 ** -134}[dtype] + 2.0 ** -148 * np.sqrt(cols)  # (FP32's steps on the way: a factor's, times u, and three sums')
        assert np.all(np.abs(dx.double().numpy() - want) <= half * np.abs(want) + (SUM + 8 * B.U32) * 1.01 * scale + tiny)
        assert np.all(np.abs(dweight.double().numpy() - dw) <= (rows + 24) * B.U32 * dw_scale)
