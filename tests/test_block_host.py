"""The refusals of the entry points on block-scaled matrices, of the norm and of clipping: found on the host, before anything is launched."""
import pytest

import paper_2409_16626_b200 as H
from paper_2409_16626_b200 import _hif8_call as call
from paper_2409_16626_b200 import binding

OK, NULL, DTYPE, ROUND, FLAGS, RANGE, SHAPE, ALIGN, WORKSPACE, OVERLAP = 0, 1, 2, 3, 4, 5, 6, 7, 8, 11
M = 1 << 20
ENCODE = dict(src=16 * M, src_dtype=H.BF16, ld_src=300, rows=200, cols=300, block_rows=1, dst=32 * M, ld_dst=304, d_exp=48 * M, exp_stride=3, target_exp=3, rnd=H.RND_TA, flags=0, seed=0)
DECODE = dict(src=32 * M, ld_src=304, d_exp=48 * M, exp_stride=3, rows=200, cols=300, block_rows=128, dst=16 * M, dst_dtype=H.F32, ld_dst=300)
NORM = dict(x=16 * M, ld_x=300, residual=17 * M, ld_residual=300, dtype=H.BF16, weight=18 * M, eps=1e-5, rows=200, cols=300, h=19 * M, ld_h=300, d_rstd=20 * M, dst=32 * M, ld_dst=304,
            d_exp=48 * M, exp_stride=3, target_exp=3, rnd=H.RND_TA, flags=0)
BACKWARD = dict(dy=16 * M, ld_dy=300, h=17 * M, ld_h=300, dh=18 * M, ld_dh=300, dtype=H.F16, weight=19 * M, d_rstd=20 * M, rows=200, cols=300, dx=21 * M, ld_dx=300, d_weight_grad=22 * M,
                accumulate=0, workspace=64 * M, workspace_bytes=1 << 24)
GEMM = dict(Aq=16 * M, lda=256, a_is_km=0, d_exp_a=17 * M, exp_stride_a=2, a_block_rows=1, Wq=18 * M, ldw=256, w_is_nk=1, d_exp_w=19 * M, exp_stride_w=2, w_block_rows=128, Cmat=20 * M,
            ldc=64, c_dtype=H.BF16, M=50, N=60, K=250, accumulate=0, workspace=64 * M, workspace_bytes=1 << 24)
CLIP = dict(d_src=16 * M, d_dst=17 * M, d_dtype=18 * M, d_start=19 * M, n_tensors=3, n_elements=1000, d_scale_exp=20 * M, max_norm=1.0, d_norm=21 * M, d_found_inf=22 * M,
            workspace=64 * M, workspace_bytes=1 << 16)
CALLS = {"encode": (H.hif8_block_encode, ENCODE), "decode": (H.hif8_block_decode, DECODE), "norm": (H.hif8_rmsnorm_encode, NORM), "backward": (H.hif8_rmsnorm_backward, BACKWARD),
         "gemm": (H.hif8_gemm_block, GEMM), "clip": (H.hif8_grad_clip, CLIP)}
REFUSED = {
    "encode": [(dict(src_dtype=3), DTYPE), (dict(rnd=5), ROUND), (dict(flags=4), FLAGS), (dict(target_exp=16), RANGE), (dict(target_exp=-23), RANGE), (dict(rows=-1), SHAPE),
               (dict(cols=-1), SHAPE), (dict(block_rows=64), SHAPE), (dict(block_rows=0), SHAPE), (dict(ld_src=299), SHAPE), (dict(ld_dst=299), SHAPE), (dict(exp_stride=2), SHAPE),
               (dict(rows=1 << 31), SHAPE), (dict(src=None), NULL), (dict(dst=None), NULL), (dict(d_exp=None), NULL), (dict(src=16 * M + 1), ALIGN), (dict(d_exp=48 * M + 2), ALIGN),
               (dict(dst=16 * M), OVERLAP), (dict(dst=16 * M + 2 * (199 * 300 + 299)), OVERLAP), (dict(d_exp=32 * M + 304), OVERLAP), (dict(d_exp=16 * M + 4), OVERLAP), (dict(rows=0), OK), (dict(cols=0), OK)],
    "decode": [(dict(dst_dtype=-1), DTYPE), (dict(rows=-1), SHAPE), (dict(block_rows=2), SHAPE), (dict(ld_src=299), SHAPE), (dict(ld_dst=299), SHAPE), (dict(exp_stride=2), SHAPE),
               (dict(rows=1 << 31), SHAPE), (dict(src=None), NULL), (dict(dst=None), NULL), (dict(d_exp=None), NULL), (dict(dst=16 * M + 2), ALIGN), (dict(d_exp=48 * M + 1), ALIGN),
               (dict(dst=32 * M), OVERLAP), (dict(dst=48 * M), OVERLAP), (dict(rows=0), OK)],
    "norm": [(dict(dtype=4), DTYPE), (dict(rnd=H.RND_SR), ROUND), (dict(rnd=-1), ROUND), (dict(flags=8), FLAGS), (dict(target_exp=16), RANGE), (dict(eps=-1e-9), RANGE),
             (dict(eps=float("nan")), RANGE), (dict(eps=float("inf")), RANGE), (dict(rows=-1), SHAPE), (dict(cols=32769, ld_x=40000, ld_residual=40000, ld_h=40000, ld_dst=40000, exp_stride=400), SHAPE),
             (dict(ld_x=299), SHAPE), (dict(ld_residual=299), SHAPE), (dict(ld_h=299), SHAPE), (dict(ld_dst=299), SHAPE), (dict(exp_stride=2), SHAPE), (dict(x=None), NULL), (dict(weight=None), NULL),
             (dict(dst=None), NULL), (dict(d_exp=None), NULL), (dict(x=16 * M + 1), ALIGN), (dict(weight=18 * M + 1), ALIGN), (dict(h=19 * M + 1), ALIGN), (dict(d_rstd=20 * M + 2), ALIGN),
             (dict(h=16 * M + 2), OVERLAP), (dict(h=16 * M, ld_h=304), OVERLAP), (dict(h=17 * M + 600), OVERLAP), (dict(h=18 * M), OVERLAP), (dict(dst=16 * M), OVERLAP), (dict(dst=19 * M), OVERLAP),
             (dict(d_rstd=19 * M), OVERLAP), (dict(d_rstd=18 * M), OVERLAP), (dict(d_exp=20 * M), OVERLAP), (dict(rows=0), OK), (dict(cols=0), OK)],
    "backward": [(dict(dtype=3), DTYPE), (dict(rows=-1), SHAPE), (dict(cols=32769), SHAPE), (dict(ld_dy=299), SHAPE), (dict(ld_h=299), SHAPE), (dict(ld_dh=299), SHAPE), (dict(ld_dx=299), SHAPE),
                 (dict(dy=None), NULL), (dict(h=None), NULL), (dict(weight=None), NULL), (dict(d_rstd=None), NULL), (dict(dx=None), NULL), (dict(dy=16 * M + 1), ALIGN), (dict(d_rstd=20 * M + 2), ALIGN),
                 (dict(d_weight_grad=22 * M + 2), ALIGN), (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=1200), WORKSPACE), (dict(workspace=64 * M + 16), WORKSPACE),
                 (dict(dx=16 * M + 2), OVERLAP), (dict(dx=16 * M, ld_dx=304), OVERLAP), (dict(dx=17 * M), OVERLAP), (dict(dx=18 * M + 600), OVERLAP), (dict(dx=19 * M), OVERLAP),
                 (dict(dx=20 * M), OVERLAP), (dict(d_weight_grad=21 * M + 4), OVERLAP), (dict(d_weight_grad=64 * M), OVERLAP), (dict(workspace=16 * M), OVERLAP), (dict(cols=0), OK)],
    "gemm": [(dict(c_dtype=H.F16), DTYPE), (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(a_block_rows=2), SHAPE), (dict(w_block_rows=64), SHAPE), (dict(lda=249), SHAPE), (dict(ldw=249), SHAPE),
             (dict(ldc=56), SHAPE), (dict(exp_stride_a=1), SHAPE), (dict(exp_stride_w=1), SHAPE), (dict(a_is_km=1, lda=49), SHAPE), (dict(w_is_nk=0, ldw=59), SHAPE), (dict(Aq=None), NULL), (dict(Wq=None), NULL),
             (dict(Cmat=None), NULL), (dict(d_exp_a=None), NULL), (dict(d_exp_w=None), NULL), (dict(Cmat=20 * M + 8), ALIGN), (dict(Aq=16 * M + 8), ALIGN), (dict(Wq=18 * M + 1), ALIGN), (dict(lda=264), ALIGN), (dict(ldw=257), ALIGN), (dict(ldc=61), ALIGN), (dict(d_exp_a=17 * M + 2), ALIGN),
             (dict(d_exp_w=19 * M + 1), ALIGN), (dict(workspace=None), WORKSPACE), (dict(workspace=64 * M + 16), WORKSPACE), (dict(workspace_bytes=255), WORKSPACE), (dict(Cmat=16 * M), OVERLAP),
             (dict(Cmat=18 * M), OVERLAP), (dict(Cmat=19 * M), OVERLAP), (dict(Cmat=64 * M + 256), OVERLAP), (dict(workspace=16 * M), OVERLAP), (dict(M=0), OK), (dict(N=0), OK)],
    "clip": [(dict(max_norm=0.0), RANGE), (dict(max_norm=-1.0), RANGE), (dict(max_norm=float("nan")), RANGE), (dict(n_tensors=-1), SHAPE), (dict(n_elements=-1), SHAPE), (dict(n_elements=1 << 51), SHAPE),
             (dict(d_src=None), NULL), (dict(d_dtype=None), NULL), (dict(d_start=None), NULL), (dict(d_src=16 * M + 4), ALIGN), (dict(d_dst=17 * M + 4), ALIGN), (dict(d_dtype=18 * M + 2), ALIGN),
             (dict(d_start=19 * M + 4), ALIGN), (dict(d_norm=21 * M + 2), ALIGN), (dict(d_found_inf=22 * M + 1), ALIGN), (dict(d_scale_exp=20 * M + 2), ALIGN), (dict(workspace=None), WORKSPACE),
             (dict(workspace_bytes=8), WORKSPACE), (dict(workspace=64 * M + 8), WORKSPACE), (dict(d_norm=16 * M + 8), OVERLAP), (dict(d_norm=22 * M), OVERLAP), (dict(workspace=18 * M), OVERLAP),
             (dict(d_found_inf=20 * M), OVERLAP)],
}


@pytest.mark.parametrize("name,change,status", [(c, *e) for c in CALLS for e in REFUSED[c]])
def test_refusals(name, change, status):
    fn, good = CALLS[name]
    before = H.hif8_launch_count()
    assert fn(**{**good, **change}, stream=0, check=False) == status
    assert H.hif8_launch_count() == before


def test_a_refusal_raises():
    with pytest.raises(H.Hif8Error):
        H.hif8_block_encode(**{**ENCODE, "block_rows": 3}, stream=0)


@pytest.mark.parametrize("name", ["hif8_block_encode", "hif8_block_decode", "hif8_rmsnorm_encode", "hif8_rmsnorm_backward", "hif8_gemm_block", "hif8_grad_clip",
                                  "hif8_rmsnorm_backward_workspace_bytes", "hif8_gemm_block_workspace_bytes"])
def test_prototypes_agree(name):
    n = len(getattr(binding.lib, name).argtypes)
    assert getattr(call, name)(*[object()] * n) is None and getattr(call, name)(*[0] * (n - 1)) is None


def test_workspace_bytes():
    norm = H.hif8_rmsnorm_backward_workspace_bytes
    assert norm(0, 100) == norm(10, 0) == norm(10, 40000) == 0 and 0 < norm(1, 100) <= norm(1000, 100) and norm(100000, 8192) < 1 << 24
    gemm = H.hif8_gemm_block_workspace_bytes
    assert gemm(0, 5, 5, 0, 1, 128) >= 256 and gemm(5, 7, 1000, 0, 1, 128) % 256 == 0
    assert gemm(8192, 8192, 8192, 0, 1, 128) >= 256 + 4 * 8192 * 8192                         # room for both operands
    assert H.hif8_grad_clip_workspace_bytes() % 8 == 0
