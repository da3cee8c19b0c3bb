"""Products of block-scaled operands against 64 bits: |C - C*| <= BOUND(K) sum |a w|, BF16 results half a step more.  The tensor core adds sixteen products at a
time to a sum in FP32 and drops what lies below its last bit, at most 2^-23 of the sum: ceil(K / 16) times that (and 1e-5 where it is less)."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from gpu_util import gemm_path

pytestmark = pytest.mark.gpu


def operand(rows, cols, block_rows, seed, ld=None, offset=0, spread=3):
    """Codes (rows ld bytes apart, guard bytes that stand for NaN around them), exponents, and what they stand for."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 256, size=(rows, cols)).astype(np.uint8)
    far = ((codes & 0x60) == 0x60) & (rng.random((rows, cols)) < 0.9)
    codes[far] &= 0x9F                                   # large and small magnitudes seldom
    codes[(codes & 0x7F) == 0x6F] = 0x08                 # no Inf, no NaN
    codes[codes == 0x80] = 0
    exps = rng.integers(-spread, spread + 1, size=(-(-rows // block_rows), -(-cols // 128))).astype(np.int32)
    ld = ld or -(-cols // 16) * 16
    raw = torch.full((offset + rows * ld + 16,), 0x80, dtype=torch.uint8, device="cuda")
    q = torch.as_strided(raw, (rows, cols), (ld, 1), offset)
    q.copy_(torch.from_numpy(codes))
    return q, torch.from_numpy(exps).cuda(), B.meant(codes, exps, block_rows)


def bound(K):
    return max(1e-5, -(-K // 16) * 2.0 ** -23)


def check(M, N, K, a_is_km=0, ab=1, w_is_nk=1, wb=128, c_dtype=H.F32, accumulate=0, seed=0, ldc=None, **how):
    a, ae, av = operand(K if a_is_km else M, M if a_is_km else K, ab, seed, how.get("lda"), how.get("a_offset", 0))
    w, we, wv = operand(N if w_is_nk else K, K if w_is_nk else N, wb, seed + 1, how.get("ldw"), how.get("w_offset", 0))
    av, wv = (av.T if a_is_km else av), (wv.T if w_is_nk else wv)
    want, scale = av @ wv, np.abs(av) @ np.abs(wv)
    start = torch.randn(M, N, generator=torch.Generator().manual_seed(seed)) * float(scale.mean()) * 0.1
    C = B.Guarded(M, N, B.TORCH[c_dtype], ldc or -(-N // 8) * 8, 0, start.cuda())
    n = H.hif8_gemm_block_workspace_bytes(M, N, K, a_is_km, w_is_nk, wb)
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    H.hif8_gemm_block(a.data_ptr(), a.stride(0), a_is_km, ae, ae.stride(0), ab, w.data_ptr(), w.stride(0), w_is_nk, we, we.stride(0), wb, C.ptr, C.ld, c_dtype, M, N, K, accumulate, ws, n)
    assert H.hif8_last_device_status() == 0
    C.check()
    assert bool((ws[n:] == 0xFF).all())
    got = C.t.cpu().double().numpy()
    if accumulate:
        old = start.to(B.TORCH[c_dtype]).double().numpy()
        want, scale = want + old, scale + np.abs(old)
    err = np.abs(got - want)
    tol = bound(K) * scale + (2.0 ** -8 * np.abs(want) * 1.01 if c_dtype == H.BF16 else 0.0)
    assert np.all(err <= tol), (err / scale).max()


SIZES = [(1, 128, 128), (1, 4096, 512), (5, 300, 1040), (17, 257, 2064), (48, 1000, 1024), (64, 512, 4096), (65, 520, 784), (100, 1000, 1000), (129, 129, 129), (300, 700, 333), (512, 1024, 768), (1, 1, 1), (3, 7, 5)]


@pytest.mark.parametrize("w_is_nk", [0, 1])
@pytest.mark.parametrize("c_dtype", [H.F32, H.BF16])
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("path", [H.GEMM_PATH_AUTO, H.GEMM_PATH_WARP, H.GEMM_PATH_NO_WARP, H.GEMM_PATH_EXPAND_BOTH])
def test_forward_sizes(M, N, K, c_dtype, w_is_nk, path):
    """Every kernel that a product may be given to, where it can take it."""
    with gemm_path(path):
        check(M, N, K, w_is_nk=w_is_nk, c_dtype=c_dtype, seed=M + N + K)


@pytest.mark.parametrize("K", list(range(241, 257)) + list(range(17, 32)))
@pytest.mark.parametrize("w_is_nk", [0, 1])
def test_sums_end_anywhere(K, w_is_nk):
    """What lies behind the last k of a row (codes of NaN here) is not part of the sum, in any kernel."""
    for path in (H.GEMM_PATH_WARP, H.GEMM_PATH_NO_WARP):
        with gemm_path(path):
            check(5, 132, K, w_is_nk=w_is_nk, seed=K)
            check(40, 264, K, w_is_nk=w_is_nk, seed=K)
            check(100, 132, K, w_is_nk=w_is_nk, seed=K)
    with gemm_path(H.GEMM_PATH_EXPAND_BOTH):
        check(520, 132, K, w_is_nk=w_is_nk, seed=K)


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("c_dtype", [H.F32, H.BF16])
@pytest.mark.parametrize("a_is_km", [0, 1])
@pytest.mark.parametrize("ab,wb", [(1, 1), (128, 1), (1, 128), (128, 128)])
@pytest.mark.parametrize("w_is_nk", [0, 1])
def test_blocks_and_layouts(w_is_nk, ab, wb, a_is_km, c_dtype, accumulate):
    check(131, 264, 300, a_is_km, ab, w_is_nk, wb, c_dtype, accumulate, seed=3)
    check(20, 392, 528, a_is_km, ab, w_is_nk, wb, c_dtype, accumulate, seed=4)
    with gemm_path(H.GEMM_PATH_NO_WARP):
        check(20, 392, 528, a_is_km, ab, w_is_nk, wb, c_dtype, accumulate, seed=5)
        check(300, 392, 528, a_is_km, ab, w_is_nk, wb, c_dtype, accumulate, seed=6)


@pytest.mark.parametrize("how", [dict(lda=304, ldw=320), dict(a_offset=16, w_offset=32), dict(ldc=272), dict(lda=1024, w_offset=48, ldc=1000)])
@pytest.mark.parametrize("M", [7, 150, 600])
def test_strides_and_alignments(M, how):
    check(M, 256, 288, seed=5, **how)


@pytest.mark.parametrize("M,N,K", [(1, 14336, 4096), (16, 8192, 8192), (33, 28672, 1024), (64, 1024, 16384), (333, 8003, 4096), (2048, 4096, 1024), (1000, 2048, 6000)])
@pytest.mark.parametrize("w_is_nk", [0, 1])
def test_large_against_32_bits(M, N, K, w_is_nk):
    """Against the product in FP32, whose own error is far below the bound."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(*((N, K) if w_is_nk else (K, N)), generator=g, device="cuda") * 0.05
    (q, e), (wq, we) = B.encoded(a, H.F32, 1), B.encoded(w, H.F32, 128)
    C = B.product(q, e, 0, 1, wq, we, w_is_nk, 128, M, N, K)
    assert H.hif8_last_device_status() == 0
    av, wv = torch.empty_like(a), torch.empty_like(w)
    H.hif8_block_decode(q, q.stride(0), e, e.stride(0), M, K, 1, av, H.F32, K)
    H.hif8_block_decode(wq, wq.stride(0), we, we.stride(0), *w.shape, 128, wv, H.F32, w.shape[1])
    wv = wv.T if w_is_nk else wv
    assert bool(((C[:, :N] - av @ wv).abs() <= bound(K) * (av.abs() @ wv.abs())).all())


def test_exponents_at_their_limits_and_beyond():
    """Exponents of +-96 and ones that are taken as +-96: scales that cancel."""
    rng = np.random.default_rng(7)
    for M in (9, 200):
        a, ae, av = operand(M, 256, 1, 11, spread=0)
        w, we, wv = operand(264, 256, 128, 12, spread=0)
        for ea, ew in ((96, -96), (-96, 96), (500, -1000), (-(1 << 31), (1 << 31) - 1)):
            C = B.product(a, torch.full_like(ae, ea), 0, 1, w, torch.full_like(we, ew), 1, 128, M, 264, 256)
            assert np.all(np.abs(C.cpu().double().numpy() - av @ wv.T) <= 1e-5 * (np.abs(av) @ np.abs(wv.T)))
    del rng


@pytest.mark.parametrize("M", [3, 150])
def test_inf_and_nan_propagate(M):
    a, ae, _ = operand(M, 256, 1, 21)
    w, we, _ = operand(130, 256, 128, 22)
    base = B.product(a, ae, 0, 1, w, we, 1, 128, M, 130, 256)[:, :130].clone()
    a[1, 200], w[5, 7] = 0x6F, 0x80                      # Inf in a row, NaN in a column
    w[:, 200] = 0x08                                     # (Inf times a positive value)
    C = B.product(a, ae, 0, 1, w, we, 1, 128, M, 130, 256)[:, :130]
    bad = ~torch.isfinite(C)
    want = torch.zeros_like(bad)
    want[1], want[:, 5] = True, True
    assert torch.equal(bad, want) and bool(torch.isnan(C[:, 5]).all()) and bool((C[1, :5] == float("inf")).all())
    assert bool(torch.isfinite(base).all())


def test_results_are_reproducible_and_streams_do_not_mix():
    a, ae, _ = operand(40, 2048, 1, 31)
    w, we, _ = operand(1024, 2048, 128, 32)
    first = B.product(a, ae, 0, 1, w, we, 1, 128, 40, 1024, 2048).clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(B.product(a, ae, 0, 1, w, we, 1, 128, 40, 1024, 2048))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_captured(M):
    a, ae, _ = operand(M, 1024, 1, 41)
    w, we, _ = operand(512, 1024, 128, 42)
    n = H.hif8_gemm_block_workspace_bytes(M, 512, 1024, 0, 1, 128)
    ws, C = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(M, 512, device="cuda")
    want = B.product(a, ae, 0, 1, w, we, 1, 128, M, 512, 1024, C=torch.zeros_like(C), ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.product(a, ae, 0, 1, w, we, 1, 128, M, 512, 1024, C=C, ws=ws)
    ws.fill_(0xFF)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(C, want)
    a.copy_(a.flip(0))                                   # new codes, the same graph
    want = B.product(a, ae, 0, 1, w, we, 1, 128, M, 512, 1024, C=torch.zeros_like(C))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(C, want)


@pytest.mark.parametrize("M,N,K", [(192, 512, 2810), (64, 72, 5000), (300, 7, 1000), (1, 1, 4096), (257, 520, 1537), (33, 1000, 700), (1500, 700, 3000)])
@pytest.mark.parametrize("a_is_km,w_is_nk", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("c_dtype", [H.F32, H.BF16])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_long_sums_of_few_tiles(M, N, K, a_is_km, w_is_nk, c_dtype, accumulate):
    """Sums that are divided: parts that end with zeros, added up in order."""
    check(M, N, K, a_is_km, 1, w_is_nk, 1, c_dtype, accumulate, seed=M)


def test_rows_far_apart():
    """Offsets beyond 32 bits: rows of codes 2^31 bytes apart, rows of C 2^32 bytes."""
    for M, N, K in ((3, 40, 256), (2, 300, 512)):
        a, ae, av = operand(M, K, 1, 51)
        w, we, wv = operand(N, K, 128, 52)
        far = torch.zeros((M - 1) * 2 ** 31 + K, dtype=torch.uint8, device="cuda")
        fa = torch.as_strided(far, (M, K), (2 ** 31, 1))
        fa.copy_(a)
        out = torch.zeros((M - 1) * 2 ** 30 + N, device="cuda")
        n = H.hif8_gemm_block_workspace_bytes(M, N, K, 0, 1, 128)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        for path in (H.GEMM_PATH_WARP, H.GEMM_PATH_NO_WARP):
            out.fill_(7)
            with gemm_path(path):
                H.hif8_gemm_block(fa, 2 ** 31, 0, ae, ae.stride(0), 1, w, w.stride(0), 1, we, we.stride(0), 128, out, 2 ** 30, H.F32, M, N, K, 0, ws, n)
            C = torch.as_strided(out, (M, N), (2 ** 30, 1))
            assert np.all(np.abs(C.cpu().double().numpy() - av @ wv.T) <= bound(K) * (np.abs(av) @ np.abs(wv.T)))
            assert float(out[N]) == 7 and float(out[2 ** 30 - 1]) == 7
        del far, out


@pytest.mark.parametrize("M,N,K", [(2304, 2304, 130), (4600, 2302, 70), (2500, 4099, 200)])
@pytest.mark.parametrize("c_dtype", [H.F32, H.BF16])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_several_tiles_to_a_pair(M, N, K, c_dtype, accumulate):
    check(M, N, K, 1, 1, 0, 1, c_dtype, accumulate, seed=K)
    check(M, N, K, 0, 1, 1, 1, c_dtype, accumulate, seed=K)


@pytest.mark.parametrize("M", [1, 2, 3, 4])
@pytest.mark.parametrize("N,K", [(1, 4096), (7, 130), (131, 512), (300, 1000), (1000, 2064), (2500, 513), (517, 4097), (260, 5000), (140, 8192), (130, 9000), (72, 16384), (20000, 272)])
@pytest.mark.parametrize("c_dtype,accumulate", [(H.F32, 1), (H.BF16, 0), (H.BF16, 1)])
def test_single_tokens(M, N, K, c_dtype, accumulate):
    with gemm_path(H.GEMM_PATH_NO_WARP):
        check(M, N, K, 0, 1 if M % 2 else 128, 1, 128, c_dtype, accumulate, seed=N + K)
        check(M, N, K, 0, 1, 1, 128, c_dtype, accumulate, seed=N, lda=-(-K // 16) * 16 + 32, ldw=-(-K // 16) * 16 + 16, a_offset=16, w_offset=48, ldc=-(-N // 8) * 8 + 8)


@pytest.mark.parametrize("M", [1, 2])
def test_single_tokens_with_exponents_at_their_limits(M):
    a, ae, av = operand(M, 700, 1, 11, spread=0)
    w, we, wv = operand(264, 700, 128, 12, spread=0)
    with gemm_path(H.GEMM_PATH_NO_WARP):
        for ea, ew in ((96, -96), (-96, 96), (500, -1000), (-(1 << 31), (1 << 31) - 1)):
            C = B.product(a, torch.full_like(ae, ea), 0, 1, w, torch.full_like(we, ew), 1, 128, M, 264, 700)[:, :264]
            assert np.all(np.abs(C.cpu().double().numpy() - av @ wv.T) <= 1e-5 * (np.abs(av) @ np.abs(wv.T)))
        # activations that leave FP32 with both scales, products that do not: 2^111 and 2^20 by weights of 2^-22 .. 2^-16
        rng = np.random.default_rng(3)
        big, small = rng.choice([0x6E, 0xEE, 0x08, 0x30], size=(M, 700)).astype(np.uint8), (rng.integers(1, 8, size=(264, 700)) + 128 * rng.integers(0, 2, size=(264, 700))).astype(np.uint8)
        a[:], w[:] = torch.from_numpy(big).cuda(), torch.from_numpy(small).cuda()
        C = B.product(a, torch.full_like(ae, -96), 0, 1, w, torch.full_like(we, -20), 1, 128, M, 264, 700)[:, :264].cpu().double().numpy()
        av, wv = B.VALUES[big] * 2.0 ** 96, B.VALUES[small] * 2.0 ** 20
        assert np.all(np.isfinite(C)) and np.all(np.abs(C - av @ wv.T) <= 1e-5 * (np.abs(av) @ np.abs(wv.T)))


@pytest.mark.parametrize("M", [1, 2])
def test_inf_and_nan_of_single_tokens(M):
    a, ae, _ = operand(M, 523, 1, 21)
    w, we, _ = operand(130, 523, 128, 22)
    a[0, 200], w[5, 7] = 0x6F, 0x80                      # Inf in a row, NaN in a column
    w[:, 200] = 0x08                                     # (Inf times a positive value)
    with gemm_path(H.GEMM_PATH_NO_WARP):
        C = B.product(a, ae, 0, 1, w, we, 1, 128, M, 130, 523)[:, :130]
    assert bool(torch.isnan(C[:, 5]).all()) and bool((C[0, :5] == float("inf")).all()) and bool((C[0, 6:] == float("inf")).all())
    assert M == 1 or bool(torch.isfinite(C[1, :5]).all() and torch.isfinite(C[1, 6:]).all())
