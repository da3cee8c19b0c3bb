// Products of block-scaled operands: which kernels take one, and the launches in front of them.
#include "hif8_block_types.cuh"

namespace hif8 {
namespace {

constexpr size_t kStatusBytes = 256;  // the status word's part of the workspace

// Products of block-scaled operands.  A power-of-two scale leaves a value's four significant bits as they are and its exponent within BF16's range, so the
// scales ride in the operands' BF16 copies, whichever way the blocks lie to the sum: nothing is rescaled between k-blocks.
struct BlockPlan {
    long long a_pitch, w_pitch;  // elements between rows of the BF16 copies
    size_t a_bytes, w_bytes;
    BlockPlan(int M, int N, int K, int w_is_nk)
    {
        auto pad8 = [](long long n) { return (n + 7) & ~7ll; };
        auto pad256 = [](size_t n) { return (n + 255) & ~(size_t)255; };
        a_pitch = pad8(K);
        w_pitch = pad8(w_is_nk ? K : N);
        a_bytes = pad256((size_t)M * (size_t)a_pitch * 2);
        w_bytes = pad256((size_t)(w_is_nk ? N : K) * (size_t)w_pitch * 2);
    }
    size_t bytes() const { return kStatusBytes + a_bytes + w_bytes; }
};

}  // namespace
}  // namespace hif8

using namespace hif8;

extern "C" size_t hif8_gemm_block_workspace_bytes(int M, int N, int K, int a_is_km, int w_is_nk, int w_block_rows)
{
    (void)a_is_km; (void)w_block_rows;
    if (M <= 0 || N <= 0 || K <= 0) return kStatusBytes;
    return BlockPlan(M, N, K, w_is_nk).bytes();
}

extern "C" int hif8_gemm_block(const uint8_t* Aq, int64_t lda, int a_is_km, const int* d_exp_a, int64_t exp_stride_a, int a_block_rows, const uint8_t* Wq, int64_t ldw,
                               int w_is_nk, const int* d_exp_w, int64_t exp_stride_w, int w_block_rows, void* C, int64_t ldc, int c_dtype, int M, int N, int K, int accumulate,
                               void* workspace, size_t workspace_bytes, hif8_stream_t stream)
{
    if (c_dtype != HIF8_BF16 && c_dtype != HIF8_F32) return HIF8_ERR_DTYPE;
    if (M < 0 || N < 0 || K < 0 || (a_block_rows != 1 && a_block_rows != HIF8_BLOCK) || (w_block_rows != 1 && w_block_rows != HIF8_BLOCK)) return HIF8_ERR_SHAPE;
    const BlockCodes a{const_cast<uint8_t*>(Aq), lda, const_cast<int*>(d_exp_a), exp_stride_a, a_is_km ? K : M, a_is_km ? M : K, a_block_rows == 1 ? 0 : 7};
    const BlockCodes w{const_cast<uint8_t*>(Wq), ldw, const_cast<int*>(d_exp_w), exp_stride_w, w_is_nk ? N : K, w_is_nk ? K : N, w_block_rows == 1 ? 0 : 7};
    if (lda < a.cols || ldw < w.cols || ldc < N || exp_stride_a < a.blocks_across() || exp_stride_w < w.blocks_across()) return HIF8_ERR_SHAPE;
    if (M == 0 || N == 0) return HIF8_OK;
    if (K == 0) return HIF8_ERR_SHAPE;
    if (!Aq || !Wq || !C || !d_exp_a || !d_exp_w) return HIF8_ERR_NULL;
    const size_t c_item = c_dtype == HIF8_F32 ? 4 : 2;
    if (!aligned_to(C, 16) || ((ldc * c_item) & 15) || !aligned_to(d_exp_a, 4) || !aligned_to(d_exp_w, 4)) return HIF8_ERR_ALIGN;
    const BlockPlan plan(M, N, K, w_is_nk);
    if (!workspace || workspace_bytes < plan.bytes() || !aligned_to(workspace, 256)) return HIF8_ERR_WORKSPACE;
    if (written_over({{C, matrix_bytes(M, N, ldc, c_item)}, {workspace, plan.bytes()}}, {{Aq, a.code_bytes()}, {Wq, w.code_bytes()}, {d_exp_a, a.exp_bytes()}, {d_exp_w, w.exp_bytes()}}))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    GemmParams p{};
    p.C = C; p.ldc = ldc; p.c_is_f32 = c_dtype == HIF8_F32; p.M = M; p.N = N; p.K = K; p.accumulate = accumulate ? 1 : 0;
    p.status = reinterpret_cast<int*>(workspace);
    note_status_word(st, p.status);
    unsigned char* a_bf = reinterpret_cast<unsigned char*>(workspace) + kStatusBytes;
    unsigned char* w_bf = a_bf + plan.a_bytes;
    if (int rc = expand_block_codes(a, a_bf, plan.a_pitch, a_is_km ? plan.a_pitch : M, a_is_km ? M : plan.a_pitch, a_is_km != 0, reinterpret_cast<uint32_t*>(workspace), st)) return rc;
    if (int rc = expand_block_codes(w, w_bf, plan.w_pitch, w.rows, plan.w_pitch, false, nullptr, st)) return rc;
    return launch_bf16_pair_gemm(a_bf, w_bf, w_is_nk, p, st, 0, 0, plan.a_pitch, plan.w_pitch);
}
