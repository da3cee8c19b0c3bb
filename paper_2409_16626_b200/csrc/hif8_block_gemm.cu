// Products of block-scaled operands: the entry points.  A power-of-two scale leaves a value's four significant bits as they are and its exponent within BF16's range,
// so the scales ride in the operands' BF16 copies, whichever way the blocks lie to the sum, and nothing is rescaled between k-blocks (see launch_block_gemm for the kernels).
#include "hif8_block_types.cuh"

using namespace hif8;

extern "C" size_t hif8_gemm_block_workspace_bytes(int M, int N, int K, int a_is_km, int w_is_nk, int w_block_rows)
{
    if (M <= 0 || N <= 0 || K <= 0) return BlockWorkspace::kStatus;
    return BlockWorkspace(M, N, K, a_is_km != 0, w_is_nk != 0, w_block_rows).bytes();
}

extern "C" int hif8_gemm_block(const uint8_t* Aq, int64_t lda, int a_is_km, const int* d_exp_a, int64_t exp_stride_a, int a_block_rows, const uint8_t* Wq, int64_t ldw,
                               int w_is_nk, const int* d_exp_w, int64_t exp_stride_w, int w_block_rows, void* C, int64_t ldc, int c_dtype, int M, int N, int K, int accumulate,
                               void* workspace, size_t workspace_bytes, hif8_stream_t stream)
{
    if (c_dtype != HIF8_BF16 && c_dtype != HIF8_F32) return HIF8_ERR_DTYPE;
    if (M < 0 || N < 0 || K < 0 || M > BlockWorkspace::kMostDim || N > BlockWorkspace::kMostDim || K > BlockWorkspace::kMostDim || (a_block_rows != 1 && a_block_rows != HIF8_BLOCK) || (w_block_rows != 1 && w_block_rows != HIF8_BLOCK)) return HIF8_ERR_SHAPE;
    const BlockCodes a{const_cast<uint8_t*>(Aq), lda, const_cast<int*>(d_exp_a), exp_stride_a, a_is_km ? K : M, a_is_km ? M : K, a_block_rows == 1 ? 0 : 7};
    const BlockCodes w{const_cast<uint8_t*>(Wq), ldw, const_cast<int*>(d_exp_w), exp_stride_w, w_is_nk ? N : K, w_is_nk ? K : N, w_block_rows == 1 ? 0 : 7};
    if (lda < a.cols || ldw < w.cols || ldc < N || exp_stride_a < a.blocks_across() || exp_stride_w < w.blocks_across()) return HIF8_ERR_SHAPE;
    if (M == 0 || N == 0) return HIF8_OK;
    const BlockWorkspace plan(M, N, K, a_is_km != 0, w_is_nk != 0, w_block_rows);
    if (K == 0 || !plan.fits) return HIF8_ERR_SHAPE;
    if (!Aq || !Wq || !C || !d_exp_a || !d_exp_w) return HIF8_ERR_NULL;
    const size_t c_item = c_dtype == HIF8_F32 ? 4 : 2;
    if (!aligned_to(Aq, 16) || !aligned_to(Wq, 16) || ((lda | ldw) & 15) || !aligned_to(C, 16) || ((ldc * c_item) & 15) || !aligned_to(d_exp_a, 4) || !aligned_to(d_exp_w, 4)) return HIF8_ERR_ALIGN;
    if (!workspace || workspace_bytes < plan.bytes() || !aligned_to(workspace, 256)) return HIF8_ERR_WORKSPACE;
    if (written_over({{C, matrix_bytes(M, N, ldc, c_item)}, {workspace, plan.bytes()}}, {{Aq, a.code_bytes()}, {Wq, w.code_bytes()}, {d_exp_a, a.exp_bytes()}, {d_exp_w, w.exp_bytes()}}))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    GemmParams p{};
    p.C = C; p.ldc = ldc; p.c_is_f32 = c_dtype == HIF8_F32; p.M = M; p.N = N; p.K = K; p.accumulate = accumulate ? 1 : 0;
    p.status = reinterpret_cast<int*>(workspace);
    note_status_word(st, p.status);
    return launch_block_gemm(a, a_is_km != 0, w, w_is_nk != 0, p, plan, workspace, st);
}
