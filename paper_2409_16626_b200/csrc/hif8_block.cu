// Block-scaled matrices: conversion to HiF8 with one power-of-two scale for each 1 x 128 or 128 x 128 elements, back, and into BF16 as
// operands of a product.
//
//   e = clamp(target_exp - floor(log2 amax)),  code = To_HiF8(x 2^e),  x ~ value(code) 2^-e
//
// All of it is bound by memory: every element is read once.  Eight threads hold a block of 1 x 128, sixteen elements each, so its maximum takes three exchanges; a block of
// 128 x 128 is one thread block's, held in registers between its maximum and its codes.
#include "hif8_block.cuh"

namespace hif8 {
namespace {

struct EncodeParams {
    const void* src;
    long long ld_src;
    BlockCodes m;
    FastDiv across;       // blocks of a row
    unsigned units;       // 1 x 128: blocks of the matrix; 128 x 128: the same
    int target_exp;
    unsigned flags;
    unsigned long long seed;
    bool vectors, vectors32, codes8, codes16;  // rows of the source start on boundaries of 16 and 32 bytes, those of the codes of 8 and 16
    bool late;             // the next launch may start at the end (see launch_encode)
};

// eight elements -> codes; `flat`: the flat index of the first one (stochastic rounding draws by it)
template <int SRC, int MODE>
__device__ __forceinline__ uint2 encode_eight(const Eight<SRC>& e, float scale, const SmemTables& sm, unsigned long long flat, unsigned long long seed)
{
    if (MODE == HIF8_RND_TA && SRC == HIF8_BF16) {
        const uint32_t s2 = bf16x2_of_pow2(scale);
        const uint32_t scales2[4] = {s2, s2, s2, s2};
        const float scales[8] = {scale, scale, scale, scale, scale, scale, scale, scale};
        return encode_vector_ta<SRC>(e.v[0], scales2, scales, sm.ta);
    }
    uint32_t w[2] = {0u, 0u};
    uint4 draws = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        float x; uint32_t raw, word = 0;
        unpack_eight<SRC>(e, i, x, raw);
        if (MODE == HIF8_RND_SR) {
            const unsigned long long at = flat + i;
            if (i == 0 || (at & 3u) == 0) draws = philox4x32_10((uint32_t)(at >> 2), (uint32_t)(at >> 34), (uint32_t)seed, (uint32_t)(seed >> 32));
            word = philox_word(draws, (unsigned)at & 3u);
        }
        w[i >> 2] |= (encode_one<MODE, SRC>(x, raw, scale, sm.ta, sm.thr, word) & 0xFFu) << (8 * (i & 3));
    }
    return make_uint2(w[0], w[1]);
}

template <int SRC>
__device__ __forceinline__ uint32_t amax_of_eight(const Eight<SRC>& e)
{
    uint32_t m = amax_vector<SRC>(0u, e.v[0]);
    if (SRC == HIF8_F32) m = amax_vector<SRC>(m, e.v[sizeof(e.v) / 16 - 1]);
    return __float_as_uint(amax_value<SRC>(m));
}

// Sixteen neighbouring elements of a row, from column c on; `vectors32`: the row starts on a 32-byte boundary
template <int DT> struct Sixteen { Eight<DT> lo, hi; };
template <int DT>
__device__ __forceinline__ Sixteen<DT> load_sixteen(const void* row, long long c, long long cols, bool vectors, bool vectors32)
{
    Sixteen<DT> s;
    if (vectors32 && c + 16 <= cols) {
        const char* p = reinterpret_cast<const char*>(row) + c * (DT == HIF8_F32 ? 4 : 2);
        auto get = [](const char* from, uint4& a, uint4& b) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(from));
        };
        constexpr int last = sizeof(s.lo.v) / 16 - 1;
        if (DT == HIF8_F32) {
            get(p, s.lo.v[0], s.lo.v[last]);
            get(p + 32, s.hi.v[0], s.hi.v[last]);
        } else get(p, s.lo.v[0], s.hi.v[0]);
        return s;
    }
    s.lo = load_eight<DT>(row, c, cols, vectors);
    s.hi = load_eight<DT>(row, c + 8, cols, vectors);
    return s;
}

// Blocks of 1 x 128: eight threads to a block, four blocks to a warp and step.  Issue slots are what it costs beside the bytes: with sixteen threads of eight elements each, four
// steps in flight, it took 17.6 instructions an element (16384 x 8192, us: BF16 94.6, FP16 89.8, FP32 109.7; so 70.9, 68.9 and 100.0; with two steps in flight and fewer blocks
// 73.0, 71.3 and 101.0).
constexpr int row_blocks(int src, int mode) { return mode == HIF8_RND_SR ? 2 : src == HIF8_F32 ? 5 : 6; }
template <int SRC, int MODE>
__global__ void __launch_bounds__(kThreads, row_blocks(SRC, MODE)) block_row_encode_kernel(const EncodeParams p)
{
    __shared__ SmemTables sm;
    setup_tables<true, MODE != HIF8_RND_TA, false, MODE, SRC>(sm, p.flags);
    pdl_wait_prior_grid();
    if (!p.late) pdl_launch_dependents();
    constexpr size_t item = SRC == HIF8_F32 ? 4 : 2;
    const unsigned lane = threadIdx.x & 31u, part = lane >> 3, at = (lane & 7u) * 16u;
    const unsigned warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
    for (unsigned long long first = (unsigned long long)warp * 4; first < p.units; first += (unsigned long long)warps * 4) {
        const unsigned u = (unsigned)first + part, row = p.across.div(u), blk = u - row * p.across.d;
        const long long c = (long long)blk * 128 + at;
        const Sixteen<SRC> e = load_sixteen<SRC>(reinterpret_cast<const char*>(p.src) + (size_t)row * (size_t)p.ld_src * item, u < p.units ? c : p.m.cols, p.m.cols, p.vectors, p.vectors32);
        uint32_t top = max(amax_of_eight<SRC>(e.lo), amax_of_eight<SRC>(e.hi));
#pragma unroll
        for (int d = 4; d; d >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const int se = block_exp_from_amax(top, p.target_exp);
        if (u >= p.units) continue;
        if (at == 0) p.m.exps[(size_t)row * (size_t)p.m.exp_stride + blk] = se;
        if (c >= p.m.cols) continue;
        const float scale = pow2f(se);
        const unsigned long long flat = (unsigned long long)row * (unsigned long long)p.m.cols + (unsigned long long)c;
        const uint2 lo = encode_eight<SRC, MODE>(e.lo, scale, sm, flat, p.seed), hi = encode_eight<SRC, MODE>(e.hi, scale, sm, flat + 8, p.seed);
        uint8_t* out = p.m.codes + (size_t)row * (size_t)p.m.ld;
        if (p.codes16 && c + 16 <= p.m.cols) *reinterpret_cast<uint4*>(out + c) = make_uint4(lo.x, lo.y, hi.x, hi.y);
        else {
            store_codes8(out, c, p.m.cols, p.codes8, lo);
            store_codes8(out, c + 8, p.m.cols, p.codes8, hi);
        }
    }
    if (p.late) pdl_launch_dependents();
}

// The same where rows lie on no such boundaries: a warp takes two neighbouring blocks of a row at a time, spread over its lanes (see load_spread).
template <int SRC, int MODE>
__global__ void __launch_bounds__(kThreads, row_blocks(SRC, MODE)) block_row_encode_spread_kernel(const EncodeParams p)
{
    __shared__ SmemTables sm;
    setup_tables<true, MODE != HIF8_RND_TA, false, MODE, SRC>(sm, p.flags);
    pdl_wait_prior_grid();
    if (!p.late) pdl_launch_dependents();
    constexpr size_t item = SRC == HIF8_F32 ? 4 : 2;
    const int lane = threadIdx.x & 31, cols = (int)p.m.cols;
    const unsigned warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
    for (unsigned long long u = warp; u < p.units; u += warps) {  // p.across: pairs of blocks of a row
        const unsigned row = p.across.div((unsigned)u), pair = (unsigned)u - row * p.across.d;
        const int c = (int)pair * 256 + lane;
        const Eight<SRC> e = load_spread<SRC>(reinterpret_cast<const char*>(p.src) + (size_t)row * (size_t)p.ld_src * item, c, cols);
        int se[2];
        uint32_t code[2] = {0u, 0u};
#pragma unroll
        for (int k = 0; k < 2; k++) {
            float top = 0.f;
#pragma unroll
            for (int i = 4 * k; i < 4 * k + 4; i++) top = amax_step(top, value_of_eight<SRC>(e, i));
            se[k] = block_exp_from_amax(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)), p.target_exp);
            const float scale = pow2f(se[k]);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float x; uint32_t raw, word = 0;
                unpack_eight<SRC>(e, 4 * k + i, x, raw);
                if (MODE == HIF8_RND_SR) {
                    const unsigned long long at = (unsigned long long)row * (unsigned long long)p.m.cols + (unsigned long long)(c + 32 * (4 * k + i));
                    word = philox_word(philox4x32_10((uint32_t)(at >> 2), (uint32_t)(at >> 34), (uint32_t)p.seed, (uint32_t)(p.seed >> 32)), (unsigned)at & 3u);
                }
                code[k] |= (encode_one<MODE, SRC>(x, raw, scale, sm.ta, sm.thr, word) & 0xFFu) << (8 * i);
            }
        }
        store_codes_spread(p.m.codes + (size_t)row * (size_t)p.m.ld, c, cols, make_uint2(code[0], code[1]));
        if (lane < 2 && (int)pair * 256 + 128 * lane < cols) p.m.exps[(size_t)row * (size_t)p.m.exp_stride + 2 * pair + lane] = lane ? se[1] : se[0];
    }
    if (p.late) pdl_launch_dependents();
}

// Blocks of 128 x 128: a thread block takes one at a time, half a warp eight of its rows.
constexpr int tile_blocks(int src) { return src == HIF8_F32 ? 2 : 4; }
template <int SRC, int MODE>
__global__ void __launch_bounds__(kThreads, tile_blocks(SRC)) block_tile_encode_kernel(const EncodeParams p)
{
    __shared__ SmemTables sm;
    __shared__ uint32_t s_top[2][kThreads / 32];
    setup_tables<true, MODE != HIF8_RND_TA, false, MODE, SRC>(sm, p.flags);
    pdl_wait_prior_grid();
    if (!p.late) pdl_launch_dependents();
    constexpr size_t item = SRC == HIF8_F32 ? 4 : 2;
    constexpr int kRows = 128 / (kThreads / 16);
    const unsigned at = (threadIdx.x & 15u) * 8u, r0 = threadIdx.x >> 4;
    int turn = 0;
    for (unsigned u = blockIdx.x; u < p.units; u += gridDim.x, turn ^= 1) {
        const unsigned down = p.across.div(u), blk = u - down * p.across.d;
        const long long c = (long long)blk * 128 + at, row = (long long)down * 128 + r0;
        Eight<SRC> e[kRows];
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < kRows; j++) {
            const long long r = row + j * (kThreads / 16);
            e[j] = load_eight<SRC>(reinterpret_cast<const char*>(p.src) + (size_t)r * (size_t)p.ld_src * item, r < p.m.rows ? c : p.m.cols, p.m.cols, p.vectors);
        }
#pragma unroll
        for (int j = 0; j < kRows; j++) top = max(top, amax_of_eight<SRC>(e[j]));
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if ((threadIdx.x & 31u) == 0) s_top[turn][threadIdx.x >> 5] = top;
        __syncthreads();  // (two sets of words in turn: whoever still reads the other one has not passed this barrier)
        top = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; w++) top = max(top, s_top[turn][w]);
        const int se = block_exp_from_amax(top, p.target_exp);
        if (threadIdx.x == 0) p.m.exps[(size_t)down * (size_t)p.m.exp_stride + blk] = se;
        const float scale = pow2f(se);
        if (c < p.m.cols) {
#pragma unroll
            for (int j = 0; j < kRows; j++) {
                const long long r = row + j * (kThreads / 16);
                if (r >= p.m.rows) continue;
                const uint2 w = encode_eight<SRC, MODE>(e[j], scale, sm, (unsigned long long)r * (unsigned long long)p.m.cols + (unsigned long long)c, p.seed);
                store_codes8(p.m.codes + (size_t)r * (size_t)p.m.ld, c, p.m.cols, p.codes8, w);
            }
        }
    }
    if (p.late) pdl_launch_dependents();
}

// ------------------------------------------------------------------------------------------------
// codes -> values
// ------------------------------------------------------------------------------------------------
struct DecodeParams {
    BlockCodes m;
    void* dst;
    long long ld_dst, rows_out, cols_out;
    FastDiv chunks;      // groups of sixteen columns of a row that is written
    unsigned units;      // such groups
    bool codes8, codes16, vectors, vectors32;  // rows of the codes start on boundaries of 8 and of 16 bytes, those written of 16 and of 32
    uint32_t* clear;
    unsigned clear_words;
    bool late;           // the next launch may start at the end (see launch_decode)
};
// One matrix, or two (a product's operands) in one launch: the groups of the second follow those of the first.
template <bool TWO> struct DecodeJob {
    DecodeParams m[TWO ? 2 : 1];
    unsigned units;
};

__device__ __forceinline__ int exp_at(const BlockCodes& m, long long r, long long c)
{
    return clamp_block_exp(__ldg(m.exps + (size_t)(r >> m.shift) * (size_t)m.exp_stride + (size_t)(c >> 7)));
}

// four codes through a table of one word per code (LANE: a copy per lane), as two words of two BF16
template <bool LANE>
__device__ __forceinline__ uint2 bf16_of_four(const uint32_t* table, uint32_t w, uint32_t lane4)
{
    if (LANE) return lane_lookup4(table, w, lane4);
    return make_uint2(table[w & 0xFFu] | (table[(w >> 8) & 0xFFu] << 16), table[(w >> 16) & 0xFFu] | (table[w >> 24] << 16));
}

template <int DST>
__device__ __forceinline__ Eight<DST> scaled_eight(uint2 lo, uint2 hi, int e)
{
    if (DST == HIF8_BF16) {  // (exact, no subnormals: |e| is at most 96)
        const uint32_t s = bf16x2_of_pow2(pow2f(-e));
        Eight<DST> r;
        r.v[0] = make_uint4(mul_bf16x2(lo.x, s), mul_bf16x2(lo.y, s), mul_bf16x2(hi.x, s), mul_bf16x2(hi.y, s));
        return r;
    }
    const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
    const float s = pow2f(-e);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16) * s;
    return pack_eight<DST>(x);
}

// sixteen values of a row: two words of 32 bytes (FP32) or one, whole sectors a lane where the row lies so
template <int DST>
__device__ __forceinline__ void store_sixteen(void* row, long long c, long long cols, bool vectors, bool vectors32, const Eight<DST>& lo, const Eight<DST>& hi)
{
    if (vectors32 && c + 16 <= cols) {
        char* p = reinterpret_cast<char*>(row) + c * (DST == HIF8_F32 ? 4 : 2);
        auto put = [](char* to, const uint4& a, const uint4& b) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(to), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
        };
        constexpr int last = sizeof(lo.v) / 16 - 1;
        if (DST == HIF8_F32) {
            put(p, lo.v[0], lo.v[last]);
            put(p + 32, hi.v[0], hi.v[last]);
        } else put(p, lo.v[0], hi.v[0]);
        return;
    }
    store_eight<DST>(row, c, cols, vectors, lo);
    store_eight<DST>(row, c + 8, cols, vectors, hi);
}

// LANE: a copy of the table for each lane.  One table for all costs a warp several wavefronts a lookup; filling 32 copies costs a block more than a
// small matrix takes.  The next groups' codes are on their way while those at hand are looked up.
template <int DST, bool LANE, bool TWO>
__global__ void __launch_bounds__(kThreads, LANE ? 6 : 4) block_decode_kernel(const __grid_constant__ DecodeJob<TWO> job)
{
    __shared__ __align__(16) uint32_t table[LANE ? kLaneTableWords : 256];
    if (LANE) fill_lane_table(table, decode_bits_f32(threadIdx.x) >> 16);
    else table[threadIdx.x] = decode_bits_f32(threadIdx.x) >> 16;
    __syncthreads();
    pdl_wait_prior_grid();
    if (!job.m[0].late) pdl_launch_dependents();
    if (blockIdx.x == 0)
        for (unsigned i = threadIdx.x; i < job.m[0].clear_words; i += kThreads) job.m[0].clear[i] = 0u;
    const uint32_t lane4 = (threadIdx.x & 31u) * 4u;
    constexpr size_t item = DST == HIF8_F32 ? 4 : 2;
    struct Group {
        uint4 v;
        int e;
        unsigned row, chunk;  // (of sixteen columns: a row may have more than 2^32)
    };
    auto which = [&](unsigned long long u) { return TWO && u >= job.m[0].units ? 1 : 0; };
    auto load = [&](unsigned long long u64) {
        Group g;
        g.v = make_uint4(0u, 0u, 0u, 0u);
        g.e = 0; g.row = 0; g.chunk = 0;
        if (u64 >= job.units) return g;
        const int k = which(u64);
        const DecodeParams& p = job.m[k];
        const unsigned u = (unsigned)(u64 - (k ? job.m[0].units : 0u));
        g.row = p.chunks.div(u); g.chunk = u - g.row * p.chunks.d;
        const long long col = (long long)g.chunk * 16;
        if (g.row < p.m.rows && col < p.m.cols) {
            const uint8_t* at = p.m.codes + (size_t)g.row * (size_t)p.m.ld;
            g.e = exp_at(p.m, g.row, col);
            if (p.codes16 && col + 16 <= p.m.cols) g.v = __ldcs(reinterpret_cast<const uint4*>(at + col));
            else {
                const uint2 lo = load_codes8(at, col, p.m.cols, p.codes8), hi = load_codes8(at, col + 8, p.m.cols, p.codes8);
                g.v = make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
        }
        return g;
    };
    const unsigned long long step = (unsigned long long)gridDim.x * kThreads;
    unsigned long long base = (unsigned long long)blockIdx.x * kThreads + threadIdx.x;
    Group next = load(base);
    for (; base < job.units; base += step) {
        const Group now = next;
        if (LANE) next = load(base + step);
        const DecodeParams& p = job.m[which(base)];
        const Eight<DST> lo = scaled_eight<DST>(bf16_of_four<LANE>(table, now.v.x, lane4), bf16_of_four<LANE>(table, now.v.y, lane4), now.e);
        const Eight<DST> hi = scaled_eight<DST>(bf16_of_four<LANE>(table, now.v.z, lane4), bf16_of_four<LANE>(table, now.v.w, lane4), now.e);
        store_sixteen<DST>(reinterpret_cast<char*>(p.dst) + (size_t)now.row * (size_t)p.ld_dst * item, (long long)now.chunk * 16, p.cols_out, p.vectors, p.vectors32, lo, hi);
        if (!LANE) break;  // (as many threads as groups)
    }
    if (job.m[0].late) pdl_launch_dependents();
}

// The same to rows that lie on no 16-byte boundary, or from such: a warp takes 512 columns of a row, spread over its lanes: sixteen codes each, their exponents four.
template <int DST>
__global__ void __launch_bounds__(kThreads, 6) block_decode_spread_kernel(const DecodeParams p)
{
    __shared__ __align__(16) uint32_t table[kLaneTableWords];
    fill_lane_table(table, decode_bits_f32(threadIdx.x));
    __syncthreads();
    pdl_wait_prior_grid();
    const uint32_t lane4 = (threadIdx.x & 31u) * 4u;
    const int lane = threadIdx.x & 31, cols = (int)p.m.cols;
    const unsigned warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
    for (unsigned long long u = warp; u < p.units; u += warps) {  // p.chunks: stretches of 512 columns of a row
        const unsigned row = p.chunks.div((unsigned)u);
        const int c = (int)((unsigned)u - row * p.chunks.d) * 512 + lane;
        const uint8_t* from = p.m.codes + (size_t)row * (size_t)p.m.ld;
        uint32_t code[16];
        float scale[4];
#pragma unroll
        for (int i = 0; i < 16; i++) code[i] = c + 32 * i < cols ? __ldcs(from + c + 32 * i) : 0u;
#pragma unroll
        for (int k = 0; k < 4; k++) scale[k] = pow2f(c + 128 * k < cols ? -exp_at(p.m, row, c + 128 * k) : 0);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            if (c + 32 * i >= cols) continue;
            const float x = __uint_as_float(lane_lookup<0>(table, code[i], lane4)) * scale[i >> 2];
            const size_t at = (size_t)row * (size_t)p.ld_dst + (size_t)(c + 32 * i);
            if (DST == HIF8_F32) reinterpret_cast<float*>(p.dst)[at] = x;
            else if (DST == HIF8_BF16) reinterpret_cast<unsigned short*>(p.dst)[at] = (unsigned short)to_bits<HIF8_BF16>(x);
            else reinterpret_cast<unsigned short*>(p.dst)[at] = (unsigned short)to_bits<HIF8_F16>(x);
        }
    }
    pdl_launch_dependents();
}

// Codes [rows, cols] -> BF16 [cols, ld_dst], transposed: tiles of 64 rows by 64 columns.  A thread takes two rows' eight columns and puts a column's two
// values into one word, lines of 33 words apart: eight row pairs and four groups of columns to a warp meet in no bank, and read whole 32-byte sectors.
constexpr int kFlipRows = 64, kFlipCols = 64, kFlipLine = kFlipRows / 2 + 1;
template <bool LANE>
__global__ void __launch_bounds__(kThreads) block_decode_transpose_kernel(const DecodeParams p)
{
    __shared__ __align__(16) uint32_t table[LANE ? kLaneTableWords : 256];
    __shared__ uint32_t tile[kFlipCols * kFlipLine];
    if (LANE) fill_lane_table(table, decode_bits_f32(threadIdx.x) >> 16);
    else table[threadIdx.x] = decode_bits_f32(threadIdx.x) >> 16;
    __syncthreads();
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    if (blockIdx.x == 0)
        for (unsigned i = threadIdx.x; i < p.clear_words; i += kThreads) p.clear[i] = 0u;
    const unsigned lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t lane4 = lane * 4u;
    for (unsigned t = blockIdx.x; t < p.units; t += gridDim.x) {  // p.chunks: tiles across
        const unsigned down = p.chunks.div(t), across = t - down * p.chunks.d;
        const long long r0 = (long long)down * kFlipRows, c0 = (long long)across * kFlipCols;
        uint2 v[2];
        int e[2];
        const unsigned group = (warp & 1u) * 4u + (lane & 3u), pair = (warp >> 1) * 8u + (lane >> 2);  // eight groups of columns by 32 row pairs
        const long long c = c0 + group * 8u;
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const long long r = r0 + 2 * pair + i;
            const bool inside = r < p.m.rows && c < p.m.cols;
            v[i] = inside ? load_codes8(p.m.codes + (size_t)r * (size_t)p.m.ld, c, p.m.cols, p.codes8) : make_uint2(0u, 0u);
            e[i] = inside ? exp_at(p.m, r, c) : 0;
        }
        const Eight<HIF8_BF16> a = scaled_eight<HIF8_BF16>(bf16_of_four<LANE>(table, v[0].x, lane4), bf16_of_four<LANE>(table, v[0].y, lane4), e[0]);
        const Eight<HIF8_BF16> b = scaled_eight<HIF8_BF16>(bf16_of_four<LANE>(table, v[1].x, lane4), bf16_of_four<LANE>(table, v[1].y, lane4), e[1]);
        const uint32_t x[4] = {a.v[0].x, a.v[0].y, a.v[0].z, a.v[0].w}, y[4] = {b.v[0].x, b.v[0].y, b.v[0].z, b.v[0].w};
#pragma unroll
        for (int i = 0; i < 8; i++) tile[(group * 8 + i) * kFlipLine + pair] = __byte_perm(x[i >> 1], y[i >> 1], (i & 1) ? 0x7632 : 0x5410);
        __syncthreads();
        for (unsigned k = warp; k < kFlipCols; k += kThreads / 32) {
            const long long at = c0 + k, r = r0 + 2 * lane;
            if (at < p.m.cols && r < p.rows_out) *reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned short*>(p.dst) + (size_t)at * (size_t)p.ld_dst + r) = tile[k * kFlipLine + lane];
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------
// parts of a product's sum
// ------------------------------------------------------------------------------------------------
// C (+)= the parts, added in their order: a thread has four columns of a row, every part's on its way before the first is added
template <bool F32>
__global__ void __launch_bounds__(kThreads) add_parts_kernel(const float4* __restrict__ parts, int n, long long part4, unsigned units, FastDiv quads, void* C, long long ldc, int N,
                                                             int accumulate)
{
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const unsigned u = blockIdx.x * kThreads + threadIdx.x;
    if (u >= units) return;
    const unsigned row = quads.div(u), c = (u - row * quads.d) * 4u;  // (quads: groups of four columns of a part's row)
    float4 v[BlockWorkspace::kMaxSplit];
#pragma unroll
    for (int i = 0; i < BlockWorkspace::kMaxSplit; i++)
        if (i < n) v[i] = __ldcs(parts + (size_t)i * (size_t)part4 + u);
    float x[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
    for (int i = 1; i < BlockWorkspace::kMaxSplit; i++)
        if (i < n) { x[0] += v[i].x; x[1] += v[i].y; x[2] += v[i].z; x[3] += v[i].w; }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if ((int)c + i >= N) continue;
        const long long at = (long long)row * ldc + c + i;
        if (F32) {
            float* out = reinterpret_cast<float*>(C) + at;
            *out = accumulate ? *out + x[i] : x[i];
        } else {
            unsigned short* out = reinterpret_cast<unsigned short*>(C) + at;
            const float y = accumulate ? __uint_as_float((uint32_t)*out << 16) + x[i] : x[i];
            *out = __bfloat16_as_ushort(__float2bfloat16_rn(y));
        }
    }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
int finish(int launches)
{
    g_launches.fetch_add((uint64_t)launches, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}

// Large matrices: as many blocks as are resident, since a second round of blocks as long as the first one would find the device half empty.  (Blocks of the next launch
// that only wait take the places that are free, and sit unevenly when they start: behind launches of several rounds they come at the end.)
template <int SRC, int MODE>
void launch_encode(EncodeParams p, int sms, cudaStream_t st)
{
    if (p.m.shift == 7) {
        const unsigned most = (unsigned)(sms * tile_blocks(SRC));
        p.late = p.units > most;
        launch_pdl(block_tile_encode_kernel<SRC, MODE>, dim3(p.late ? most : p.units), st, p);
        return;
    }
    const unsigned most = (unsigned)(sms * row_blocks(SRC, MODE));
    if (!(p.vectors && p.codes8) && p.m.cols >= 384 && p.m.cols < 0x7FFFFF00ll) {  // (a warp's two blocks have to be there: rows of 100 BF16 values 90 us, spread 179)
        const long long pairs = (p.m.cols + 255) / 256, units = pairs * p.m.rows;  // (no more than blocks of the matrix)
        p.across = FastDiv((uint32_t)pairs); p.units = (unsigned)units;
        const unsigned blocks = (p.units + 7u) / 8u;
        p.late = blocks > most;
        launch_pdl(block_row_encode_spread_kernel<SRC, MODE>, dim3(p.late ? most : blocks), st, p);
        return;
    }
    const unsigned blocks = (p.units + 31u) / 32u;
    p.late = blocks > most;
    launch_pdl(block_row_encode_kernel<SRC, MODE>, dim3(p.late ? most : blocks), st, p);
}
template <int SRC>
void launch_encode_mode(int rnd, const EncodeParams& p, int sms, cudaStream_t st)
{
    switch (rnd) {
        case HIF8_RND_TA: return launch_encode<SRC, HIF8_RND_TA>(p, sms, st);
        case HIF8_RND_HR: return launch_encode<SRC, HIF8_RND_HR>(p, sms, st);
        case HIF8_RND_SSR: return launch_encode<SRC, HIF8_RND_SSR>(p, sms, st);
        case HIF8_RND_TE: return launch_encode<SRC, HIF8_RND_TE>(p, sms, st);
        default: return launch_encode<SRC, HIF8_RND_SR>(p, sms, st);
    }
}

template <int DST, bool TWO>
void launch_decode(DecodeJob<TWO> job, int sms, cudaStream_t st)
{
    job.units = job.m[0].units + (TWO ? job.m[TWO ? 1 : 0].units : 0u);
    const unsigned most = (unsigned)sms * 6u, few = (job.units + kThreads - 1) / kThreads;
    if (few <= (unsigned)sms * 4u) {
        job.m[0].late = false;
        launch_pdl(block_decode_kernel<DST, false, TWO>, dim3(few), st, job);
    } else launch_pdl(block_decode_kernel<DST, true, TWO>, dim3(few < most ? few : most), st, job);
}

// a product's operand, to be decoded as it is stored (or transposed); false: too large
bool operand_job(const BlockOperand& o, DecodeParams* p)
{
    *p = DecodeParams{};
    p->m = o.m; p->dst = o.dst; p->ld_dst = o.ld_dst; p->rows_out = o.rows_out; p->cols_out = o.cols_out;
    p->codes8 = aligned_to(o.m.codes, 8) && (o.m.rows <= 1 || (o.m.ld & 7) == 0); p->codes16 = aligned_to(o.m.codes, 16) && (o.m.rows <= 1 || (o.m.ld & 15) == 0);
    p->vectors = true; p->vectors32 = aligned_to(o.dst, 32) && (o.ld_dst & 15) == 0;
    const long long across = o.transposed ? (o.cols_out + kFlipCols - 1) / kFlipCols : (o.cols_out + 15) / 16;
    const long long down = o.transposed ? (o.rows_out + kFlipRows - 1) / kFlipRows : o.rows_out;
    if (across > 0x3FFFFFFFll / (down > 0 ? down : 1)) return false;
    p->chunks = FastDiv((uint32_t)across); p->units = (unsigned)(across * down);
    return true;
}

}  // namespace

int expand_block_codes(const BlockOperand& a, const BlockOperand* w, uint32_t* clear, unsigned clear_words, cudaStream_t st)
{
    int sms; if (int rc = checked_device(&sms)) return rc;
    DecodeJob<true> two{};
    if (!operand_job(a, &two.m[0]) || (w && !operand_job(*w, &two.m[1]))) return HIF8_ERR_SHAPE;
    two.m[0].clear = clear; two.m[0].clear_words = clear_words;
    if (w) launch_decode<HIF8_BF16, true>(two, sms, st);
    else if (a.transposed) {
        const DecodeParams& p = two.m[0];
        const unsigned most = (unsigned)sms * 4u;
        if (p.units <= (unsigned)sms * 2u) launch_pdl(block_decode_transpose_kernel<false>, dim3(p.units), st, p);
        else launch_pdl(block_decode_transpose_kernel<true>, dim3(p.units < most ? p.units : most), st, p);
    } else {
        DecodeJob<false> one{};
        one.m[0] = two.m[0];
        launch_decode<HIF8_BF16, false>(one, sms, st);
    }
    return finish(1);
}

int add_product_parts(const float* parts, int n, long long rows, long long cols, const GemmParams& p, cudaStream_t st)
{
    const long long units = (long long)p.M * (cols / 4);  // (rows of a part in front of the padding ones)
    if (n > BlockWorkspace::kMaxSplit || units > 0x7FFFFFFFll) return HIF8_ERR_SHAPE;
    const FastDiv quads((uint32_t)(cols / 4));
    const dim3 grid((unsigned)((units + kThreads - 1) / kThreads));
    const float4* from = reinterpret_cast<const float4*>(parts);
    if (p.c_is_f32) launch_pdl(add_parts_kernel<true>, grid, st, from, n, rows * cols / 4, (unsigned)units, quads, p.C, p.ldc, p.N, p.accumulate);
    else launch_pdl(add_parts_kernel<false>, grid, st, from, n, rows * cols / 4, (unsigned)units, quads, p.C, p.ldc, p.N, p.accumulate);
    return finish(1);
}

}  // namespace hif8

using namespace hif8;

extern "C" int hif8_block_encode(const void* src, int src_dtype, int64_t ld_src, int64_t rows, int64_t cols, int block_rows, uint8_t* dst, int64_t ld_dst, int* d_exp,
                                 int64_t exp_stride, int target_exp, int rnd, unsigned flags, uint64_t seed, hif8_stream_t stream)
{
    if (bad_dtype(src_dtype)) return HIF8_ERR_DTYPE;
    if (rnd < HIF8_RND_TA || rnd > HIF8_RND_SR) return HIF8_ERR_ROUND;
    if (flags & ~(unsigned)(HIF8_FLAG_SATURATE | HIF8_FLAG_NAN_TO_ZERO)) return HIF8_ERR_FLAGS;
    if (target_exp < -22 || target_exp > 15) return HIF8_ERR_SCALE_RANGE;
    if (rows < 0 || cols < 0 || (block_rows != 1 && block_rows != HIF8_BLOCK)) return HIF8_ERR_SHAPE;
    EncodeParams p{};
    p.m = BlockCodes{dst, ld_dst, d_exp, exp_stride, rows, cols, block_rows == 1 ? 0 : 7};
    if (ld_src < cols || ld_dst < cols || exp_stride < p.m.blocks_across()) return HIF8_ERR_SHAPE;
    if (rows == 0 || cols == 0) return HIF8_OK;
    if (!src || !dst || !d_exp) return HIF8_ERR_NULL;
    if (p.m.blocks_across() > 0x7FFFFFFFll / p.m.blocks_down()) return HIF8_ERR_SHAPE;
    const size_t item = dtype_bytes(src_dtype);
    if (!aligned_to(src, item) || !aligned_to(d_exp, sizeof(int))) return HIF8_ERR_ALIGN;
    if (written_over({{dst, p.m.code_bytes()}, {d_exp, p.m.exp_bytes()}}, {{src, matrix_bytes(rows, cols, ld_src, item)}})) return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.src = src; p.ld_src = ld_src; p.target_exp = target_exp; p.flags = flags; p.seed = seed;
    p.across = FastDiv((uint32_t)p.m.blocks_across()); p.units = (unsigned)(p.m.blocks_across() * p.m.blocks_down());
    p.vectors = vector_rows(src, rows, ld_src, item);
    p.vectors32 = aligned_to(src, 32) && (rows <= 1 || ((size_t)ld_src * item & 31u) == 0);
    p.codes8 = aligned_to(dst, 8) && (rows <= 1 || (ld_dst & 7) == 0); p.codes16 = aligned_to(dst, 16) && (rows <= 1 || (ld_dst & 15) == 0);
    cudaStream_t st = (cudaStream_t)stream;
    if (src_dtype == HIF8_F32) launch_encode_mode<HIF8_F32>(rnd, p, sms, st);
    else if (src_dtype == HIF8_BF16) launch_encode_mode<HIF8_BF16>(rnd, p, sms, st);
    else launch_encode_mode<HIF8_F16>(rnd, p, sms, st);
    return finish(1);
}

extern "C" int hif8_block_decode(const uint8_t* src, int64_t ld_src, const int* d_exp, int64_t exp_stride, int64_t rows, int64_t cols, int block_rows, void* dst, int dst_dtype,
                                 int64_t ld_dst, hif8_stream_t stream)
{
    if (bad_dtype(dst_dtype)) return HIF8_ERR_DTYPE;
    if (rows < 0 || cols < 0 || (block_rows != 1 && block_rows != HIF8_BLOCK)) return HIF8_ERR_SHAPE;
    DecodeJob<false> job{};
    DecodeParams& p = job.m[0];
    p.late = true;
    p.m = BlockCodes{const_cast<uint8_t*>(src), ld_src, const_cast<int*>(d_exp), exp_stride, rows, cols, block_rows == 1 ? 0 : 7};
    if (ld_src < cols || ld_dst < cols || exp_stride < p.m.blocks_across()) return HIF8_ERR_SHAPE;
    if (rows == 0 || cols == 0) return HIF8_OK;
    if (!src || !dst || !d_exp) return HIF8_ERR_NULL;
    const long long across = (cols + 15) / 16;
    if (across > 0x7FFFFFFFll / rows) return HIF8_ERR_SHAPE;
    const size_t item = dtype_bytes(dst_dtype);
    if (!aligned_to(dst, item) || !aligned_to(d_exp, sizeof(int))) return HIF8_ERR_ALIGN;
    if (written_over({{dst, matrix_bytes(rows, cols, ld_dst, item)}}, {{src, p.m.code_bytes()}, {d_exp, p.m.exp_bytes()}})) return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.dst = dst; p.ld_dst = ld_dst; p.rows_out = rows; p.cols_out = cols;
    p.chunks = FastDiv((uint32_t)across); p.units = (unsigned)(across * rows);
    p.codes8 = aligned_to(src, 8) && (rows <= 1 || (ld_src & 7) == 0); p.codes16 = aligned_to(src, 16) && (rows <= 1 || (ld_src & 15) == 0);
    p.vectors = vector_rows(dst, rows, ld_dst, item); p.vectors32 = aligned_to(dst, 32) && (rows <= 1 || ((size_t)ld_dst * item & 31u) == 0);
    cudaStream_t st = (cudaStream_t)stream;
    if (!(p.vectors && p.codes8) && cols >= 96 && cols < 0x7FFFFE00ll) {  // (2^26 codes, rows of 20: 247 us, spread 1470; of 100 337 and 322, of 1001 360 and 93)
        const long long stretches = (cols + 511) / 512;
        p.chunks = FastDiv((uint32_t)stretches); p.units = (unsigned)(stretches * rows);
        const unsigned most = (unsigned)sms * 6u, blocks = (p.units + 7u) / 8u;
        const dim3 grid(blocks < most ? blocks : most);
        if (dst_dtype == HIF8_F32) launch_pdl(block_decode_spread_kernel<HIF8_F32>, grid, st, p);
        else if (dst_dtype == HIF8_BF16) launch_pdl(block_decode_spread_kernel<HIF8_BF16>, grid, st, p);
        else launch_pdl(block_decode_spread_kernel<HIF8_F16>, grid, st, p);
        return finish(1);
    }
    if (dst_dtype == HIF8_F32) launch_decode<HIF8_F32, false>(job, sms, st);
    else if (dst_dtype == HIF8_BF16) launch_decode<HIF8_BF16, false>(job, sms, st);
    else launch_decode<HIF8_F16, false>(job, sms, st);
    return finish(1);
}
