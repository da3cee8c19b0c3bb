"""Products on expanded operands whose edge tiles leave in an odd number of pieces, short sums, several tiles to a pair of CTAs: against 64 bits, and the same bits each time."""
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from gpu_util import gemm_path

pytestmark = pytest.mark.gpu
# columns behind the last whole tile of 256: FP32 1, 3 (32 columns to a piece) and 2 with one or more behind 16 bytes, BF16 1 (64) and 3
SIZES = [(8192, 800, 64, H.F32), (20000, 864, 64, H.F32), (20000, 835, 70, H.F32), (9000, 4099, 128, H.F32), (8192, 832, 64, H.BF16), (20000, 960, 64, H.BF16), (9000, 6464, 64, H.BF16),
         (20000, 837, 100, H.BF16)]


def bound(K):  # (as for the other products: sixteen terms at a time onto an FP32 sum, at most 2^-23 of it each time)
    return max(1e-5, -(-K // 16) * 2.0 ** -23)


def held(C, a, w, K, c_dtype):
    """C against A W^T in 64 bits, some rows at a time."""
    for r in range(0, a.shape[0], 4096):
        x, got = a[r:r + 4096].double(), C[r:r + 4096].double()
        want, scale = x @ w.double().T, x.abs() @ w.double().abs().T
        tol = bound(K) * scale + (2.0 ** -8 * 1.01 * want.abs() if c_dtype == H.BF16 else 0.0)
        assert bool(((got - want).abs() <= tol).all())


@pytest.mark.parametrize("M,N,K,c_dtype", SIZES)
@pytest.mark.parametrize("a_is_km", [0, 1])
def test_block_scaled(M, N, K, c_dtype, a_is_km):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a, w = torch.randn(*((K, M) if a_is_km else (M, K)), generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda")
    (q, e), (wq, we) = B.encoded(a, H.F32, 1), B.encoded(w, H.F32, 1)
    av, wv = torch.empty_like(a), torch.empty_like(w)
    H.hif8_block_decode(q, q.stride(0), e, e.stride(0), *a.shape, 1, av, H.F32, a.shape[1])
    H.hif8_block_decode(wq, wq.stride(0), we, we.stride(0), N, K, 1, wv, H.F32, K)
    ws = torch.empty(H.hif8_gemm_block_workspace_bytes(M, N, K, a_is_km, 1, 1), dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(4):
        C = B.Guarded(M, N, B.TORCH[c_dtype], -(-N // 8) * 8)
        B.product(q, e, a_is_km, 1, wq, we, 1, 1, M, N, K, c_dtype, C.t, ws=ws)
        C.check()
        first = C.t if first is None else first
        assert torch.equal(C.t, first)
    assert H.hif8_last_device_status() == 0
    held(first, av.T if a_is_km else av, wv, K, c_dtype)


@pytest.mark.parametrize("M,N,K,c_dtype", [s for s in SIZES if s[2] % 16 == 0])
def test_unscaled(M, N, K, c_dtype):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda")
    q, wq, av, wv = torch.empty(M, K, dtype=torch.uint8, device="cuda"), torch.empty(N, K, dtype=torch.uint8, device="cuda"), torch.empty_like(a), torch.empty_like(w)
    for x, c, v in ((a, q, av), (w, wq, wv)):
        H.hif8_encode(x, H.F32, c, x.numel())
        H.hif8_decode(c, v, H.F32, x.numel())
    n = H.hif8_workspace_bytes(H.WS_GEMM, M * K + K * N)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    first = None
    with gemm_path(H.GEMM_PATH_EXPAND_BOTH):
        for _ in range(4):
            C = B.Guarded(M, N, B.TORCH[c_dtype], -(-N // 8) * 8)
            H.hif8_gemm(q, K, wq, K, 1, C.ptr, C.ld, c_dtype, M, N, K, None, None, ws, n)
            C.check()
            first = C.t if first is None else first
            assert torch.equal(C.t, first)
    assert H.hif8_last_device_status() == 0
    held(first, av, wv, K, c_dtype)
