"""How exact the norm of gradients is where squares round alike and their errors add up: squares of 16 bytes are added in FP32, seven roundings of 16-bit elements (whose squares FP32 holds)
and four of FP32 ones, halved by the root; then one rounding of the norm.  At most 5 * 2^-24 of it."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from test_gpu_clip import Gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
def test_equal_elements(dtype):
    g = torch.Generator().manual_seed(1)
    worst = 0.0
    for v in (1 + torch.rand(60, generator=g)).to(B.TORCH[dtype]).unique().tolist():
        n = 4099
        s = Gradients([n], [dtype], 3, values={0: (slice(None), v)})
        s.call(float("inf"))
        want = np.sqrt(float((s.host[0].double() ** 2).sum()))
        worst = max(worst, abs(float(s.norm) - want) / want)
        assert torch.equal(s.views(s.dst)[0].cpu(), s.host[0])
    assert worst <= 5 * B.U32


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("scale_exp", [0, 7, -9])
def test_roundings_of_the_results(dtype, scale_exp):
    """From the norm that was stored, rounded as it is: the factor and its product to FP32, the product once more to the tensor's type."""
    s = Gradients([3000, 17], [dtype, dtype], 5)
    s.call(0.5, scale_exp)
    want = np.sqrt(sum(float((x.double() ** 2).sum()) for x in s.host)) * 2.0 ** -scale_exp
    f = 2.0 ** -scale_exp * min(1.0, 0.5 / want)
    half = torch.finfo(B.TORCH[dtype]).eps / 2
    tiny = {H.F32: 2.0 ** -150, H.BF16: 2.0 ** -134, H.F16: 2.0 ** -25}[dtype]
    for x, got in zip(s.host, s.views(s.dst)):
        x, got = x.double() * f, got.cpu().double()
        assert bool(((got - x).abs() <= ((half if dtype != H.F32 else 0.0) + 6.01 * B.U32) * x.abs() + tiny).all())
