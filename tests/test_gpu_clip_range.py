"""Clipping to limits that are far below the gradients: results down to FP32's last step.  Against 64 bits: a rounding of the factor, of the product and of the result, and where that is
subnormal a step of FP32 (and half a step of BF16)."""
import numpy as np
import pytest

import block_util as B
import paper_2409_16626_b200 as H
from test_gpu_clip import Gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_norm", [2.0 ** -149, 1e-44, 1e-41, 2.0 ** -126, 1e-30])
@pytest.mark.parametrize("spread,scale_exp", [(1e37, None), (1e37, 100), (1e37, -100), (1e20, 0), (1e-20, 0)])
def test_limits_far_below_the_gradients(max_norm, spread, scale_exp):
    dtypes = [H.F32, H.BF16, H.F32]
    g = Gradients([5, 700, 3000], dtypes, 5, spread)
    g.call(max_norm, scale_exp)
    limit, unscale = float(np.float32(max_norm)), 2.0 ** -(scale_exp or 0)
    host = [x.double().numpy() for x in g.host]
    norm = np.sqrt(sum(float((x * x).sum()) for x in host)) * unscale
    f = unscale * min(1.0, limit / norm)
    for x, got, d in zip(host, g.views(g.dst), dtypes):
        want, got = x * f, got.cpu().double().numpy()
        tol = 8 * B.U32 * np.abs(want) + 2.0 ** -149
        if d == H.BF16:
            tol += 2.0 ** -8 * np.abs(want) + 2.0 ** -134
        assert np.all(np.abs(got - want) <= tol)
