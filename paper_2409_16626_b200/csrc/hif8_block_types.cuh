// Block-scaled matrices (scales for each 1 x 128 or 128 x 128 elements) as the host describes them, and checks of their arguments.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "hif8.h"
#include "hif8_cache.cuh"
#include "hif8_internal.cuh"

namespace hif8 {
extern std::atomic<uint64_t> g_launches;

// Codes [rows, cols], rows ld bytes apart, with the exponents of their blocks: block (i, j) holds rows i << shift .. and columns 128 j .. .
struct BlockCodes {
    uint8_t* codes;
    long long ld;
    int* exps;
    long long exp_stride;
    long long rows, cols;
    int shift;  // 0 or 7

    long long blocks_down() const { return (rows + (1ll << shift) - 1) >> shift; }
    long long blocks_across() const { return (cols + 127) >> 7; }
    size_t code_bytes() const { return rows > 0 ? (size_t)(rows - 1) * (size_t)ld + (size_t)cols : 0; }
    size_t exp_bytes() const { return rows > 0 ? ((size_t)(blocks_down() - 1) * (size_t)exp_stride + (size_t)blocks_across()) * sizeof(int) : 0; }
};

// What the workspace of a block-scaled product holds behind the status word: the activations as BF16, and either the weights as BF16 too and the parts of a divided sum, or
// the narrow kernel's tickets and partial sums.  (Sizes follow from the arguments alone, so that they can be asked for without a device.)
struct BlockWorkspace {
    static constexpr size_t kStatus = 256;
    static constexpr int kNarrowRows = 64;   // up to so many rows the weight-streaming kernel takes the product
    static constexpr int kExpandRows = 512;  // from so many on there is room to expand the weights too, and where the tiles are few and the sum is long
    static constexpr int kPairs = 74, kMaxSplit = 16;
    static constexpr int kMostDim = 0x7FFFF000;                        // M, N and K: what is rounded up to tiles of them stays below 2^31
    static constexpr long long kMostGroups = (1ll << 30) - (1ll << 20);  // groups of sixteen columns of an operand that is expanded (with the rows or groups that parts of a sum are filled up to: 2^30)
    long long a_pitch, a_pitch_km, w_pitch;  // elements between rows of the BF16 copies (of A as [M,K], as [K,M])
    size_t a_bytes, w_bytes, narrow_bytes, part_bytes;   // 0 where there is none
    bool fits;                               // operands that are expanded in any case have no more groups than that
    bool in_kernel;                          // the weights' blocks let the kernels that decode weights take the product
    int split;                               // parts of the sum, 1: not divided
    double cycles;                           // of a round of tiles of the pair kernel, with what joins the parts
    long long w_rows;                        // of the weights' copy
    long long part_k, part_rows, part_cols;  // of a part: its k (the operands' copies end with zeros), rows and columns of its FP32 result; 0 if there is one
    BlockWorkspace(int M, int N, int K, bool a_is_km, bool w_is_nk, int w_block_rows)
    {
        auto pad8 = [](long long n) { return (n + 7) & ~7ll; };
        auto pad256 = [](size_t n) { return (n + 255) & ~(size_t)255; };
        in_kernel = w_block_rows == HIF8_BLOCK;
        split = 1;
        cycles = 0.0;
        part_k = part_rows = part_cols = 0;
        part_bytes = 0;
        auto groups_fit = [](long long rows, long long cols) { return rows * ((cols + 15) / 16) <= kMostGroups; };
        const bool a_fits = a_is_km ? groups_fit(K, M) : groups_fit(M, K), w_fits = w_is_nk ? groups_fit(pad8(N), K) : groups_fit(K, N);  // (parts of a sum have rows of W for whole groups of eight columns)
        fits = in_kernel ? a_fits || a_is_km : a_fits && w_fits;  // (beside weights that are decoded in the kernel, an A as [K,M] is transposed by tiles)
        const long long tiles = (((long long)M + 255) / 256) * (((long long)N + 255) / 256), kb = ((long long)K + 63) / 64;
        const bool expand = !in_kernel || (a_fits && w_fits && (M >= kExpandRows || (M > kNarrowRows && 2 * tiles <= kPairs && kb >= 16)));  // room for the weights' copy
        if (expand) {
            // Cycles of the pair kernel's 64 k, of the parts written and read again and of the launch that adds them (gradients of 192 x 512 over 2810 rows 22.6 us, so 13.1; 256 x 256 over 8192 47.6 and 15.9).
            const double part = 8.0 * (double)M * (double)N / 2500.0;
            cycles = 545.0 * (double)kb;
            for (int s = 2; s <= kMaxSplit && tiles * s <= kPairs && kb / s >= 2; s++) {
                const double t = 545.0 * (double)((kb + s - 1) / s) + part * s + 5000.0;
                if (t < cycles) { cycles = t; split = s; }
            }
            if (split > 1) {
                part_k = (kb + split - 1) / split * 64;
                split = (int)((kb * 64 + part_k - 1) / part_k);
                part_rows = ((long long)M + 31) & ~31ll;
                part_cols = pad8(N);
                part_bytes = pad256((size_t)split * (size_t)part_rows * (size_t)part_cols * 4);
            }
        }
        const long long k_rows = split > 1 ? part_k * split : K;  // of what is stored with k as rows; and its row length otherwise
        a_pitch = pad8(k_rows);
        a_pitch_km = pad8(M);
        w_pitch = pad8(w_is_nk ? k_rows : N);
        a_bytes = pad256((size_t)M * (size_t)a_pitch * 2);
        if (a_is_km && (size_t)k_rows * (size_t)a_pitch_km * 2 > a_bytes) a_bytes = pad256((size_t)k_rows * (size_t)a_pitch_km * 2);
        const bool narrow = in_kernel && M <= kNarrowRows;
        w_rows = !w_is_nk ? k_rows : split > 1 ? part_cols : N;
        w_bytes = !expand ? 0 : pad256((size_t)w_rows * (size_t)w_pitch * 2);
        // partial sums of 128 columns by the rows: a slice for each block of up to 160 and two more for each slab, which two blocks may share
        const size_t slabs = ((size_t)N + 127) / 128;
        narrow_bytes = narrow ? pad256(slabs * 16) + (160 + 3 * slabs) * (size_t)((M + 15) & ~15) * 512 : 0;
    }
    size_t bytes() const { return kStatus + a_bytes + w_bytes + narrow_bytes + part_bytes; }
};

// C of `p` (+)= the sum of n FP32 matrices of `rows` x `cols` in a row, in their order
struct GemmParams;
int add_product_parts(const float* parts, int n, long long rows, long long cols, const GemmParams& p, cudaStream_t st);

// C of `p` from block-scaled operands, the rest of `p` filled in here; the arguments have been checked.
int launch_block_gemm(const BlockCodes& a, bool a_is_km, const BlockCodes& w, bool w_is_nk, const GemmParams& p, const BlockWorkspace& sizes, void* workspace, cudaStream_t st);

// The same for few rows of A [M,K] and weights [N,K] with scales for each 128 x 128, codes of both operands decoded in the kernel; and its cycles (1e30: it has no form for these).
double block_rows_cycles(int M, int N, int K, int sms);
int launch_block_rows(const BlockCodes& a, const BlockCodes& w, const GemmParams& p, cudaStream_t st);

// A product's operand to be decoded into BF16 with its blocks' scales (exact: four significant bits, exponents within -118 .. 111):
// dst [rows_out, cols_out], or with `transposed` element (r, c) at dst[c][r]; rows and columns beyond the matrix become zeros.  cols_out (transposed:
// rows_out) and ld_dst are multiples of 8, dst is 16-byte aligned.
struct BlockOperand {
    BlockCodes m;
    void* dst;
    long long ld_dst, rows_out, cols_out;
    bool transposed;
};
// One launch for an operand, or for two as they are stored; it also clears clear_words words.
int expand_block_codes(const BlockOperand& a, const BlockOperand* w, uint32_t* clear, unsigned clear_words, cudaStream_t st);

namespace {

inline bool bad_dtype(int t) { return t != HIF8_F32 && t != HIF8_BF16 && t != HIF8_F16; }
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// bytes from the first to the last element of [rows, cols], rows ld elements apart
inline size_t matrix_bytes(long long rows, long long cols, long long ld, size_t item) { return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * item : 0; }
// whether rows of that many elements, ld apart, start on 16-byte boundaries
inline bool vector_rows(const void* p, long long rows, long long ld, size_t item) { return aligned_to(p, 16) && (rows <= 1 || ((size_t)ld * item & 15u) == 0); }

}  // namespace
}  // namespace hif8
