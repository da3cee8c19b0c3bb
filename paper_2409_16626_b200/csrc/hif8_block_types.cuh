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

// Codes of a product's operand, decoded into BF16 with their blocks' scales (exact: four significant bits, exponents within -118 .. 111):
// dst [rows_out, cols_out], or with `transposed` element (r, c) at dst[c][r]; rows and columns beyond the matrix become zeros.  cols_out (transposed:
// rows_out) and ld_dst are multiples of 8, dst is 16-byte aligned.  The launch also clears *clear_word (may be null).
int expand_block_codes(const BlockCodes& m, void* dst, long long ld_dst, long long rows_out, long long cols_out, bool transposed, uint32_t* clear_word, cudaStream_t st);

namespace {

inline bool bad_dtype(int t) { return t != HIF8_F32 && t != HIF8_BF16 && t != HIF8_F16; }
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// bytes from the first to the last element of [rows, cols], rows ld elements apart
inline size_t matrix_bytes(long long rows, long long cols, long long ld, size_t item) { return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * item : 0; }
// whether rows of that many elements, ld apart, start on 16-byte boundaries
inline bool vector_rows(const void* p, long long rows, long long ld, size_t item) { return aligned_to(p, 16) && (rows <= 1 || ((size_t)ld * item & 15u) == 0); }

}  // namespace
}  // namespace hif8
