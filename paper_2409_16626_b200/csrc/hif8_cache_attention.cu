// Attention over the HiF8 key/value cache.
//
//   s_ij = scale * sum_d q_i[d] k_j[d],   out_i = sum_j softmax_j(s_i) v_j,   lse_i = ln sum_j exp(s_ij)
//
// over the cached tokens j that query i may look at.  A code's value has at most 4 significant bits and an exponent in [-22, 15], so it is exact
// in FP16 (the smallest ones as FP16 subnormals), and codes are multiplied as they are: the block exponents of K go into the factor of a score and
// those of V into the softmax.  With x_ij = s_ij / ln 2 - e_v(j), e_v(j) the exponent of the block that v_j lies in, and m_i = max_j x_ij,
//   P_ij = 2^(x_ij - m_i + 8),   out_i = sum_j P_ij code_v(j) / sum_j P_ij 2^(e_v(j)),
// so P <= 2^8 whatever the blocks' spreads are, and nothing is rounded but P (to FP16, 11 bits; products and sums are FP32).  The 2^8 keeps P in the
// normal range of FP16 down to 2^-22 of the largest.  Exponents lie within +-48, so the denominator stays far inside FP32.
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "hif8.h"
#include "hif8_cache.cuh"
#include "hif8_device.cuh"
#include "hif8_host_cache.h"
#include "hif8_internal.cuh"

namespace hif8 {
extern std::atomic<uint64_t> g_launches;
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kPShift = 8.f;
constexpr float kNegInf = -__builtin_huge_valf();

struct AttentionParams {
    CacheView c;
    const void* q;
    long long q_token, q_head;  // strides in elements
    const int* q_start;
    const int* lengths;
    int n_seqs, n_q, heads, group;  // group: query heads to a key head
    int vectors;                    // q and out take 16-byte accesses
    float scale_log2;               // softmax scale / ln 2
    int causal, window;
    void* out;
    long long out_token, out_head;
    float* lse;
    int* status;
    long long* prefix;              // chunks in front of each sequence
    float* partial;
};

// FP16 bits of one code (Eq. 1, Eq. 2, specials)
constexpr uint32_t f16_bits_of_code(uint32_t c)
{
    const uint32_t sign = (c & 0x80u) << 8, m = c & 0x7Fu;
    if (m == 0) return sign ? 0x7E00u : 0u;
    if (m == 0x6F) return sign | 0x7C00u;
    if (m < 8) return sign | (1u << (m + 1));  // 2^(m - 23) in units of 2^-24
    int E = 0; uint32_t M = m & 7u, w = 3;
    if (m >= 0x60) { E = (int)(8u | ((m >> 1) & 7u)); M = m & 1u; w = 1; }
    else if (m >= 0x40) { E = (int)(4u | ((m >> 2) & 3u)); M = m & 3u; w = 2; }
    else if (m >= 0x20) E = (int)(2u | ((m >> 3) & 1u));
    else if (m >= 0x10) E = 1;
    if (m >= 0x20 ? (m & 0x10u) != 0 : m >= 0x10 && (m & 8u)) E = -E;
    if (E < -14) return sign | (512u + ((M << 9) >> w));  // E == -15: subnormal
    return sign | (uint32_t)(E + 15) << 10 | (M << (10 - w));
}
struct F16OfCode { uint16_t v[256]; };
constexpr F16OfCode make_f16_of_code()
{
    F16OfCode t{};
    for (uint32_t c = 0; c < 256; c++) t.v[c] = (uint16_t)f16_bits_of_code(c);
    return t;
}
__device__ const F16OfCode g_f16_of_code = make_f16_of_code();

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t lds_u32(uint32_t addr)
{
    uint32_t v;
    asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void mma_16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint4 ld_stream_v4(const uint8_t* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_stream_v2(const uint8_t* p)
{
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
// bytes that hold Inf or NaN codes (0x6F, 0xEF, 0x80) become zero
__device__ __forceinline__ uint32_t finite_codes(uint32_t w)
{
    const uint32_t special = __vcmpeq4(w & 0x7F7F7F7Fu, 0x6F6F6F6Fu) | __vcmpeq4(w, 0x80808080u);
    return w & ~special;
}
// 2^a for integers of any size, within the finite floats and not below 2^-126
__device__ __forceinline__ float pow2_clamped(int a) { return pow2f(max(-126, min(126, a))); }

// exponent that brings a row of queries with that largest finite magnitude into FP16: amax to [2^14, 2^15).  What then lies below FP16's subnormals
// is below 2^-38 of it.
__device__ __forceinline__ int query_exp(float amax) { return scale_exp_from_amax(__float_as_uint(amax), 14); }

// What query rows may look at.  A row is a query and one of the heads that share a key head: row r of a sequence's n_q * group belongs to query r / group.
struct SeqView {
    int first, n_q, len;  // first query of the batch, queries, tokens in the cache
    __device__ int pos(int i) const { return len - n_q + i; }  // position of query i
};
__device__ __forceinline__ SeqView seq_view(const AttentionParams& p, int s)
{
    SeqView v;
    v.first = start_at(p.q_start, s, p.n_q);
    v.n_q = max(0, start_at(p.q_start, s + 1, p.n_q) - v.first);
    v.len = p.c.length(p.lengths[s]);
    return v;
}
__device__ __forceinline__ int hi_of(const AttentionParams& p, const SeqView& v, int i) { return p.causal ? max(0, v.pos(i) + 1) : v.len; }
__device__ __forceinline__ int lo_of(const AttentionParams& p, const SeqView& v, int i) { return p.window ? max(0, v.pos(i) - p.window + 1) : 0; }

// ---------------------------------------------------------------------------------------------------------
// Few query rows (decoding, drafted tokens): bound by reading the cache once.
//
// A warp multiplies 16 tokens at a time on mma.sync with the tokens as the 16 rows of the A operand and up to 8 NT query rows as columns, so K and V
// bytes go from global memory to registers, through the lookup, into the operand: S^T = K Q^T, O^T += V^T P^T.  Which of the 16 tokens or 64 elements
// meet in a product is the operands' own business as long as both agree, so every thread's bytes come in 16-byte loads.  A table of the 256 FP16
// values with a copy for every lane takes a byte permute and a conflict-free lookup a code.  The tensor-memory path would write every decoded
// value to shared memory and read it again: eight bytes of shared-memory traffic a code instead of four, and that traffic is what comes next after DRAM here.
//
// Chunks of 64 tokens of a (sequence, key head, row tile) are dealt out evenly: group g of four warps takes the chunks [T g / G, T (g + 1) / G) of all
// T, in order.  A unit whose chunks lie in several groups leaves partial sums in the workspace, which a second kernel adds in a fixed order.
// ---------------------------------------------------------------------------------------------------------
constexpr int kGroupWarps = 4, kChunk = 16 * kGroupWarps;
constexpr uint32_t kLutBytes = 65536;  // rows of 256 bytes on a 64 KiB boundary: the address is one byte permute away from the code

template <int D, int NT>
struct RowsShape {
    static constexpr int kGroups = D == 256 ? 2 : (D == 128 && NT == 2 ? 3 : 4);  // what the registers leave room for
    static constexpr int kThreads = kGroups * kGroupWarps * 32;
    static constexpr int kRows = 8 * NT;
    static constexpr int kPitch = D + 4;                                 // floats of a row of the warps' sums
    static constexpr uint32_t kSumBytes = kGroupWarps * kRows * kPitch * 4;  // of a group
    static constexpr int kRecord = kRows * (D + 2);                      // floats of a partial result: sums, maxima, denominators
    static constexpr uint32_t kFront = (HIF8_CACHE_MAX_SEQS + 2) * 8 + kGroups * (kGroupWarps * kRows * 8) + 32 * 8 + 16;
    // what lies in front of the table's boundary (a block's shared memory begins 1 KiB into its window), the table, the sums
    static constexpr uint32_t kSmem = 2 * kLutBytes - 1024 + kGroups * kSumBytes;
    static_assert(kFront <= kLutBytes - 2048 && kSmem <= 227 * 1024, "shared memory");
};

__device__ __forceinline__ void group_sync(int group) { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(kGroupWarps * 32) : "memory"); }

// first chunk of group g
__host__ __device__ __forceinline__ long long share_of(long long chunks, int g, int groups) { return chunks * g / groups; }

// The work of one sequence in chunks
struct SeqChunks {
    int lo, per_unit, tiles;  // first token (on a chunk), chunks of a unit, row tiles
    __device__ SeqChunks(const AttentionParams& p, const SeqView& v, int rows)
    {
        lo = v.n_q ? lo_of(p, v, 0) / kChunk * kChunk : 0;
        per_unit = max(1, (v.len - lo + kChunk - 1) / kChunk);
        tiles = (int)(((long long)v.n_q * p.group + rows - 1) / rows);
    }
};

template <int DT> __device__ __forceinline__ float q_value(uint32_t half_word) { return DT == HIF8_BF16 ? __uint_as_float(half_word << 16) : __half2float(__ushort_as_half((unsigned short)half_word)); }

template <int DT> __device__ __forceinline__ uint32_t pack_out(float a, float b)
{
    uint32_t r;
    if (DT == HIF8_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
// four consecutive results of a row
template <int DT> __device__ __forceinline__ void store_out4(const AttentionParams& p, long long at, const float (&x)[4])
{
    unsigned short* out = reinterpret_cast<unsigned short*>(p.out) + at;
    const uint2 w = make_uint2(pack_out<DT>(x[0], x[1]), pack_out<DT>(x[2], x[3]));
    if (p.vectors) *reinterpret_cast<uint2*>(out) = w;
    else { out[0] = (unsigned short)w.x; out[1] = (unsigned short)(w.x >> 16); out[2] = (unsigned short)w.y; out[3] = (unsigned short)(w.y >> 16); }
}
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? kNegInf : (m - kPShift + log2f(l)) * kLn2; }
__device__ __forceinline__ float part_factor(float m, float top) { return m == kNegInf ? 0.f : exp2_approx(m - top); }

template <int D, int NT, int DT>
__global__ void __launch_bounds__(RowsShape<D, NT>::kThreads, 1) cache_attention_rows_kernel(const AttentionParams p)
{
    using S = RowsShape<D, NT>;
    constexpr int J = D / 64;                       // blocks of 64 elements of a key
    constexpr int VB = D / 8;                       // bytes of a value row that a thread holds
    constexpr int MT = D / 16;                      // m16 tiles of the output
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), lut_base = (raw + kLutBytes - 1) & ~(kLutBytes - 1);
    long long* s_prefix = reinterpret_cast<long long*>(smem_raw + ((0u - raw) & 15u));
    float2* s_ml = reinterpret_cast<float2*>(s_prefix + HIF8_CACHE_MAX_SEQS + 2);  // [group][warp][row]
    long long* s_warp = reinterpret_cast<long long*>(s_ml + S::kGroups * kGroupWarps * S::kRows);
    float* s_sum = reinterpret_cast<float*>(smem_raw + (lut_base - raw) + kLutBytes);
    if (lut_base + kLutBytes + S::kGroups * S::kSumBytes > raw + S::kSmem || raw + S::kFront > lut_base) {  // (the same answer in every thread of the grid)
        pdl_wait_prior_grid();
        if (blockIdx.x == 0 && threadIdx.x == 0) { *p.status = 7; p.prefix[p.n_seqs] = 0; }
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int grp = warp / kGroupWarps, gw = warp % kGroupWarps;
    uint32_t* lut_words = reinterpret_cast<uint32_t*>(smem_raw + (lut_base - raw));
    for (int i = threadIdx.x; i < 256 * 8; i += S::kThreads) {
        const uint32_t v = g_f16_of_code.v[i >> 3];
        *reinterpret_cast<uint4*>(lut_words + (i >> 3) * 64 + (i & 7) * 4) = make_uint4(v, v, v, v);
    }
    pdl_wait_prior_grid();
    pdl_launch_dependents();

    // chunks in front of each sequence: every thread takes consecutive sequences
    {
        const int each = (p.n_seqs + S::kThreads - 1) / S::kThreads, s0 = min(p.n_seqs, (int)threadIdx.x * each), s1 = min(p.n_seqs, s0 + each);
        long long mine = 0;
        for (int s = s0; s < s1; s++) {
            const SeqView v = seq_view(p, s);
            const SeqChunks k(p, v, S::kRows);
            s_prefix[s] = mine;
            mine += (long long)k.tiles * p.c.heads * k.per_unit;
        }
        long long x = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const long long y = __shfl_up_sync(0xFFFFFFFFu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) s_warp[warp] = x;
        __syncthreads();
        long long before = x - mine;
        for (int w = 0; w < warp; w++) before += s_warp[w];
        for (int s = s0; s < s1; s++) s_prefix[s] += before;
        if (threadIdx.x == S::kThreads - 1) s_prefix[p.n_seqs] = before + mine;
        __syncthreads();
        if (blockIdx.x == 0) {
            for (int s = threadIdx.x; s <= p.n_seqs; s += S::kThreads) p.prefix[s] = s_prefix[s];
            if (threadIdx.x == 0) *p.status = 0;
        }
    }
    const long long chunks = s_prefix[p.n_seqs];
    const int groups = (int)min((long long)gridDim.x * S::kGroups, chunks);
    const int me = (int)blockIdx.x + grp * (int)gridDim.x;  // (few chunks: a group on every SM before a second one)
    if (me >= groups) return;
    long long x0 = share_of(chunks, me, groups);
    const long long x_end = share_of(chunks, me + 1, groups);
    const uint32_t lut = lut_base + 4u * lane;
    float* my_sum = s_sum + (size_t)grp * (S::kSumBytes / 4);
    float2* my_ml = s_ml + grp * kGroupWarps * S::kRows;

    while (x0 < x_end) {
        int s = 0;
        for (int n = p.n_seqs; n > 1;) {  // last sequence that starts at or before x0 (those without chunks share their start with the next)
            const int half = n >> 1;
            if (s_prefix[s + half] <= x0) { s += half; n -= half; }
            else n = half;
        }
        const SeqView v = seq_view(p, s);
        const SeqChunks k(p, v, S::kRows);
        const long long in_seq = x0 - s_prefix[s], unit = in_seq / k.per_unit;
        const int c0 = (int)(in_seq - unit * k.per_unit), c1 = (int)min((long long)k.per_unit, c0 + (x_end - x0));
        const int head = (int)(unit / k.tiles), r0 = (int)(unit - (long long)head * k.tiles) * S::kRows;
        const int n_rows = (int)min((long long)S::kRows, (long long)v.n_q * p.group - r0);
        const int ia = r0 / p.group, ib = (r0 + n_rows - 1) / p.group;  // first and last query of the tile
        const int hi_min = min(v.len, hi_of(p, v, ia)), hi_max = min(v.len, hi_of(p, v, ib)), lo_min = lo_of(p, v, ia), lo_max = lo_of(p, v, ib);

        // queries: column g of n8 tile i is row r0 + 8 i + g; a thread takes the elements 64 j + 16 t .. + 15
        uint32_t qb[NT][J][4][2];
        float row_mul[NT][2];
        int row_lo[NT][2], row_hi[NT][2];
#pragma unroll
        for (int i = 0; i < NT; i++) {
            const int r = r0 + 8 * i + g;
            uint32_t w[J][8];
            if (8 * i + g < n_rows) {
                const int qi = r / p.group;
                const long long at = (long long)(v.first + qi) * p.q_token + (long long)(head * p.group + r - qi * p.group) * p.q_head + 16 * t;
                const unsigned short* src = reinterpret_cast<const unsigned short*>(p.q) + at;
#pragma unroll
                for (int j = 0; j < J; j++) {
                    if (p.vectors) {
                        const uint4 a = __ldg(reinterpret_cast<const uint4*>(src + 64 * j)), b = __ldg(reinterpret_cast<const uint4*>(src + 64 * j) + 1);
                        w[j][0] = a.x; w[j][1] = a.y; w[j][2] = a.z; w[j][3] = a.w; w[j][4] = b.x; w[j][5] = b.y; w[j][6] = b.z; w[j][7] = b.w;
                    } else {
#pragma unroll
                        for (int x = 0; x < 8; x++) w[j][x] = (uint32_t)src[64 * j + 2 * x] | ((uint32_t)src[64 * j + 2 * x + 1] << 16);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < J; j++)
#pragma unroll
                    for (int x = 0; x < 8; x++) w[j][x] = 0u;
            }
            int e = 0;
            if (DT == HIF8_BF16) {  // FP16 queries are multiplied as they are
                uint32_t acc = 0;
#pragma unroll
                for (int j = 0; j < J; j++)
#pragma unroll
                    for (int x = 0; x < 8; x++) acc = amax_word<DT>(acc, w[j][x]);
                float a = amax_value<DT>(acc);
                a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
                a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
                e = query_exp(a);
                const float f = pow2f(e);
#pragma unroll
                for (int j = 0; j < J; j++)
#pragma unroll
                    for (int x = 0; x < 8; x++) w[j][x] = pack_f16(q_value<DT>(w[j][x] & 0xFFFFu) * f, q_value<DT>(w[j][x] >> 16) * f);
            }
#pragma unroll
            for (int j = 0; j < J; j++)
#pragma unroll
                for (int st = 0; st < 4; st++) { qb[i][j][st][0] = w[j][2 * st]; qb[i][j][st][1] = w[j][2 * st + 1]; }
#pragma unroll
            for (int b = 0; b < 2; b++) {  // the scores' columns of this thread: rows 2 t and 2 t + 1 of the tile
                const int re = __shfl_sync(0xFFFFFFFFu, e, 4 * (2 * t + b)), row = 8 * i + 2 * t + b;
                const int qi = (r0 + row) / p.group;
                row_mul[i][b] = fminf(p.scale_log2 * pow2_clamped(-re), 3.0e38f);
                row_hi[i][b] = row < n_rows ? min(v.len, hi_of(p, v, qi)) : v.len;  // (columns without a row compute something that nobody reads)
                row_lo[i][b] = row < n_rows ? lo_of(p, v, qi) : 0;
            }
        }

        float m[NT][2], l[NT][2], o[NT][MT][4];
#pragma unroll
        for (int i = 0; i < NT; i++) {
            m[i][0] = m[i][1] = kNegInf;
            l[i][0] = l[i][1] = 0.f;
#pragma unroll
            for (int x = 0; x < MT; x++)
#pragma unroll
                for (int y = 0; y < 4; y++) o[i][x][y] = 0.f;
        }

        // pages and exponents of this warp's tiles: lane n holds those of the n-th chunk of a batch of 32
        int b_page = -1, b_ke = 0, b_ve = 0, b_first = c0;
        auto load_batch = [&](int c) {
            b_first = c;
            const int at = k.lo + (c + lane) * kChunk + 16 * gw;  // (below 2^31: a length, at most 2^30, and less than 2^12 more)
            b_page = c + lane < c1 && at < v.len ? p.c.page_of(s, at >> p.c.shift) : -1;
            const long long e = (long long)max(b_page, 0) * p.c.heads + head;
            b_ke = b_page >= 0 ? clamp_cache_exp(p.c.k_exp[e]) : 0;
            b_ve = b_page >= 0 ? clamp_cache_exp(p.c.v_exp[e]) : 0;
        };
        uint4 kw[2][J];       // rows g and g + 8
        uint32_t vw[4][VB / 4];  // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        auto tile_of = [&](int c) -> int { return k.lo + c * kChunk + 16 * gw; };
        auto load_k = [&](int page, int t0) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int tok = t0 + g + 8 * h;
                const bool in = page >= 0 && tok >= lo_min && tok < hi_max;
                const uint8_t* src = p.c.k + p.c.block_at(max(page, 0), head) + (long long)(tok & ((1 << p.c.shift) - 1)) * D + 16 * t;
#pragma unroll
                for (int j = 0; j < J; j++) kw[h][j] = in ? ld_stream_v4(src + 64 * j) : make_uint4(0, 0, 0, 0);
            }
        };
        auto load_v = [&](int page, int t0) {
#pragma unroll
            for (int h = 0; h < 4; h++) {
                const int tok = t0 + 2 * t + (h & 1) + 8 * (h >> 1);
                const bool in = page >= 0 && tok >= lo_min && tok < hi_max;
                const uint8_t* src = p.c.v + p.c.block_at(max(page, 0), head) + (long long)(tok & ((1 << p.c.shift) - 1)) * D;
                if (D == 64) {
                    const uint2 a = in ? ld_stream_v2(src + 8 * g) : make_uint2(0, 0);
                    vw[h][0] = a.x; vw[h][1] = a.y;
                } else {
#pragma unroll
                    for (int y = 0; y < VB / 16; y++) {
                        const uint4 a = in ? ld_stream_v4(src + 128 * y + 16 * g) : make_uint4(0, 0, 0, 0);
                        vw[h][4 * y] = a.x; vw[h][4 * y + 1] = a.y; vw[h][(4 * y + 2) % (VB / 4)] = a.z; vw[h][(4 * y + 3) % (VB / 4)] = a.w;
                    }
                }
            }
        };

        load_batch(c0);
        int page = __shfl_sync(0xFFFFFFFFu, b_page, 0), ke = __shfl_sync(0xFFFFFFFFu, b_ke, 0), ve = __shfl_sync(0xFFFFFFFFu, b_ve, 0);
        load_k(page, tile_of(c0));
        load_v(page, tile_of(c0));
        for (int c = c0; c < c1; c++) {
            const int t0 = tile_of(c);
            // scores, transposed: token g (+ 8) x rows 2 t, 2 t + 1
            float sc[NT][4];
#pragma unroll
            for (int i = 0; i < NT; i++) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
            for (int j = 0; j < J; j++) {
                const uint32_t wa[4] = {kw[0][j].x, kw[0][j].y, kw[0][j].z, kw[0][j].w}, wb[4] = {kw[1][j].x, kw[1][j].y, kw[1][j].z, kw[1][j].w};
#pragma unroll
                for (int st = 0; st < 4; st++) {
                    const uint32_t a0 = __byte_perm(lds_u32(__byte_perm(wa[st], lut, 0x7604)), lds_u32(__byte_perm(wa[st], lut, 0x7614)), 0x5410);
                    const uint32_t a2 = __byte_perm(lds_u32(__byte_perm(wa[st], lut, 0x7624)), lds_u32(__byte_perm(wa[st], lut, 0x7634)), 0x5410);
                    const uint32_t a1 = __byte_perm(lds_u32(__byte_perm(wb[st], lut, 0x7604)), lds_u32(__byte_perm(wb[st], lut, 0x7614)), 0x5410);
                    const uint32_t a3 = __byte_perm(lds_u32(__byte_perm(wb[st], lut, 0x7624)), lds_u32(__byte_perm(wb[st], lut, 0x7634)), 0x5410);
#pragma unroll
                    for (int i = 0; i < NT; i++) mma_16816_f16(sc[i], a0, a1, a2, a3, qb[i][j][st][0], qb[i][j][st][1]);
                }
            }
            // the next tile's keys are on their way while this one's values are multiplied
            int n_page = -1, n_ke = 0, n_ve = 0;
            if (c + 1 < c1) {
                if (c + 1 - b_first == 32) load_batch(c + 1);
                n_page = __shfl_sync(0xFFFFFFFFu, b_page, c + 1 - b_first);
                n_ke = __shfl_sync(0xFFFFFFFFu, b_ke, c + 1 - b_first);
                n_ve = __shfl_sync(0xFFFFFFFFu, b_ve, c + 1 - b_first);
                load_k(n_page, tile_of(c + 1));
            }
            const bool whole = page >= 0 && t0 >= lo_max && t0 + 16 <= hi_min;  // every row sees every token
            const float k_mul = pow2f(-ke), v_mul = pow2f(ve), v_add = (float)-ve;
            if (page >= 0 && t0 < hi_max && t0 + 16 > lo_min) {  // (the same in the whole warp)
                float top[NT][2];
                bool grows = false;
#pragma unroll
                for (int i = 0; i < NT; i++) {
#pragma unroll
                    for (int b = 0; b < 2; b++) {
                        const float f = fminf(row_mul[i][b] * k_mul, 3.0e38f);
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            float x = fmaf(sc[i][2 * h + b], f, v_add);
                            if (!whole) {
                                const int tok = t0 + g + 8 * h;
                                if (tok < row_lo[i][b] || tok >= row_hi[i][b]) x = kNegInf;
                            }
                            sc[i][2 * h + b] = x;
                        }
                        float a = fmaxf(sc[i][b], sc[i][2 + b]);
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 4));
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 8));
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 16));
                        top[i][b] = a;
                        grows |= a > m[i][b];
                    }
                }
                if (__any_sync(0xFFFFFFFFu, grows)) {
#pragma unroll
                    for (int i = 0; i < NT; i++)
#pragma unroll
                        for (int b = 0; b < 2; b++) {
                            const float n = fmaxf(m[i][b], top[i][b]), f = part_factor(m[i][b], n);
                            m[i][b] = n;
                            l[i][b] *= f;
#pragma unroll
                            for (int x = 0; x < MT; x++) { o[i][x][b] *= f; o[i][x][2 + b] *= f; }
                        }
                }
                uint32_t pb[NT][2];
#pragma unroll
                for (int i = 0; i < NT; i++) {
                    float e[4];
#pragma unroll
                    for (int b = 0; b < 2; b++) {
                        const float base = m[i][b] == kNegInf ? 0.f : m[i][b];
                        e[b] = exp2_approx(sc[i][b] - base + kPShift);  // (the difference is exact where it counts; base - 8 is not for large scores)
                        e[2 + b] = exp2_approx(sc[i][2 + b] - base + kPShift);
                        l[i][b] = fmaf(e[b] + e[2 + b], v_mul, l[i][b]);
                    }
                    pb[i][0] = transpose_8x8(pack_f16(e[0], e[1]));
                    pb[i][1] = transpose_8x8(pack_f16(e[2], e[3]));
                }
                if (!whole && (hi_min < hi_max || lo_min < lo_max)) {
                    // Some rows see a token that others do not, and 0 times an Inf or NaN would reach those: such codes are left out here, and
                    // cache_attention_specials_kernel adds them to the rows that do see them.
                    const bool mixed = t0 + 16 > hi_min || t0 < lo_max;
                    if (mixed) {
#pragma unroll
                        for (int h = 0; h < 4; h++)
#pragma unroll
                            for (int y = 0; y < VB / 4; y++) vw[h][y] = finite_codes(vw[h][y]);
                    }
                }
#pragma unroll
                for (int x = 0; x < MT; x++) {  // element pair x of the thread's bytes: row g the first, row g + 8 the second
                    const int wd = x / 2;
                    uint32_t a[4];
#pragma unroll
                    for (int b = 0; b < 2; b++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const int by = 2 * (x & 1) + b;
                            const uint32_t sel = 0x7604u + 0x10u * (uint32_t)by;
                            a[2 * h + b] = __byte_perm(lds_u32(__byte_perm(vw[2 * h][wd], lut, sel)), lds_u32(__byte_perm(vw[2 * h + 1][wd], lut, sel)), 0x5410);
                        }
#pragma unroll
                    for (int i = 0; i < NT; i++) mma_16816_f16(o[i][x], a[0], a[1], a[2], a[3], pb[i][0], pb[i][1]);
                }
            }
            if (c + 1 < c1) load_v(n_page, tile_of(c + 1));
            page = n_page; ke = n_ke; ve = n_ve;
        }

        // ---- the four warps' sums of the segment
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int b = 0; b < 2; b++) {
                l[i][b] += __shfl_xor_sync(0xFFFFFFFFu, l[i][b], 4);
                l[i][b] += __shfl_xor_sync(0xFFFFFFFFu, l[i][b], 8);
                l[i][b] += __shfl_xor_sync(0xFFFFFFFFu, l[i][b], 16);
                if (g == 0) my_ml[gw * S::kRows + 8 * i + 2 * t + b] = make_float2(m[i][b], l[i][b]);
            }
        group_sync(grp);
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int b = 0; b < 2; b++) {
                const int row = 8 * i + 2 * t + b;
                float top = kNegInf;
#pragma unroll
                for (int w = 0; w < kGroupWarps; w++) top = fmaxf(top, my_ml[w * S::kRows + row].x);
                const float f = part_factor(m[i][b], top);
                float* to = my_sum + (gw * S::kRows + row) * S::kPitch;
#pragma unroll
                for (int x = 0; x < MT; x += 2) {
                    const int d = D == 64 ? 8 * g + 2 * x : 128 * (x / 8) + 16 * g + 2 * (x % 8);
                    *reinterpret_cast<float4*>(to + d) = make_float4(o[i][x][b] * f, o[i][x][2 + b] * f, o[i][x + 1][b] * f, o[i][x + 1][2 + b] * f);
                }
            }
        group_sync(grp);
        const bool is_whole = c0 == 0 && c1 == k.per_unit;
        float* record = p.partial + (size_t)(2 * me + (c0 == 0 ? 1 : 0)) * S::kRecord;
        for (int i = gw * 32 + lane; i < n_rows * (D / 4); i += kGroupWarps * 32) {
            const int row = i / (D / 4), d = (i - row * (D / 4)) * 4;
            float top = kNegInf, den = 0.f;
#pragma unroll
            for (int w = 0; w < kGroupWarps; w++) top = fmaxf(top, my_ml[w * S::kRows + row].x);
#pragma unroll
            for (int w = 0; w < kGroupWarps; w++) den += my_ml[w * S::kRows + row].y * part_factor(my_ml[w * S::kRows + row].x, top);
            float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kGroupWarps; w++) {
                const float4 a = *reinterpret_cast<const float4*>(my_sum + (w * S::kRows + row) * S::kPitch + d);
                x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
            }
            if (is_whole) {
                const int r = r0 + row, qi = r / p.group, h = head * p.group + r - qi * p.group;
                const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
                for (int y = 0; y < 4; y++) x[y] *= inv;
                store_out4<DT>(p, (long long)(v.first + qi) * p.out_token + (long long)h * p.out_head + d, x);
                if (p.lse && d == 0) p.lse[(long long)(v.first + qi) * p.heads + h] = lse_of(top, den);
            } else {
                *reinterpret_cast<float4*>(record + row * D + d) = make_float4(x[0], x[1], x[2], x[3]);
                if (d == 0) { record[S::kRows * D + 2 * row] = top; record[S::kRows * D + 2 * row + 1] = den; }
            }
        }
        group_sync(grp);  // the sums' place is free again
        x0 += c1 - c0;
    }
}

// Block b - 1 joins the unit that the boundary between groups b - 1 and b cuts, if that is the first one to do so; the parts are added in the groups' order.
constexpr int kCombineThreads = 256;
template <int D, int NT, int DT>
__global__ void __launch_bounds__(kCombineThreads) cache_attention_combine_kernel(const AttentionParams p, int all_groups)
{
    using S = RowsShape<D, NT>;
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const long long chunks = p.prefix[p.n_seqs];
    const int groups = (int)min((long long)all_groups, chunks), b = (int)blockIdx.x + 1;
    if (b >= groups) return;
    const long long x = share_of(chunks, b, groups);
    int s = 0;
    for (int n = p.n_seqs; n > 1;) {
        const int half = n >> 1;
        if (p.prefix[s + half] <= x) { s += half; n -= half; }
        else n = half;
    }
    const SeqView v = seq_view(p, s);
    const SeqChunks k(p, v, S::kRows);
    const long long in_seq = x - p.prefix[s], unit = in_seq / k.per_unit, begin = p.prefix[s] + unit * k.per_unit, end = begin + k.per_unit;
    if (x == begin || share_of(chunks, b - 1, groups) > begin) return;
    int parts = 2;  // groups b - 1 .. b - 2 + parts
    while (b - 1 + parts < groups && share_of(chunks, b - 1 + parts, groups) < end) parts++;
    const int head = (int)(unit / k.tiles), r0 = (int)(unit - (long long)head * k.tiles) * S::kRows;
    const int n_rows = (int)min((long long)S::kRows, (long long)v.n_q * p.group - r0);
    auto record = [&](int i) { return p.partial + (size_t)(2 * (b - 1 + i) + (i == 0 ? 1 : 0)) * S::kRecord; };
    for (int i = threadIdx.x; i < n_rows * (D / 4); i += kCombineThreads) {
        const int row = i / (D / 4), d = (i - row * (D / 4)) * 4;
        float top = kNegInf, den = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < parts; j++) {
            const float* r = record(j);
            const float2 ml = *reinterpret_cast<const float2*>(r + S::kRows * D + 2 * row);
            const float4 a = *reinterpret_cast<const float4*>(r + row * D + d);
            const float n = fmaxf(top, ml.x), f = part_factor(top, n), h = part_factor(ml.x, n);
            den = den * f + ml.y * h;
            o[0] = o[0] * f + a.x * h; o[1] = o[1] * f + a.y * h; o[2] = o[2] * f + a.z * h; o[3] = o[3] * f + a.w * h;
            top = n;
        }
        const int r = r0 + row, qi = r / p.group, h = head * p.group + r - qi * p.group;
        const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
        for (int y = 0; y < 4; y++) o[y] *= inv;
        store_out4<DT>(p, (long long)(v.first + qi) * p.out_token + (long long)h * p.out_head + d, o);
        if (p.lse && d == 0) p.lse[(long long)(v.first + qi) * p.heads + h] = lse_of(top, den);
    }
}

// Inf and NaN among the values of tokens that only some of a sequence's queries see: the rows that do see them get them here.  (Those that all queries
// see took the ordinary way.)  A block looks through 16 elements of a key head's value rows; there is hardly ever anything to do.
template <int DT>
__global__ void __launch_bounds__(kThreads) cache_attention_specials_kernel(const AttentionParams p)
{
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int slice = blockIdx.x, head = blockIdx.y, s = blockIdx.z;
    const SeqView v = seq_view(p, s);
    if (v.n_q < 2) return;
    // tokens that the last query sees or the first, and not both
    const int hi0 = min(v.len, hi_of(p, v, 0)), hi1 = min(v.len, hi_of(p, v, v.n_q - 1)), lo0 = lo_of(p, v, 0), lo1 = lo_of(p, v, v.n_q - 1);
    const int a0 = lo0, a1 = min(lo1, hi1), b0 = max(hi0, a1), b1 = hi1;  // [a0, a1) and [b0, b1)
    const int n = max(0, a1 - a0) + max(0, b1 - b0);
    auto token = [&](int i) { return i < max(0, a1 - a0) ? a0 + i : b0 + (i - max(0, a1 - a0)); };
    auto codes = [&](int tok) -> uint4 {
        const int page = p.c.page_of(s, tok >> p.c.shift);
        if (page < 0) return make_uint4(0, 0, 0, 0);
        return __ldg(reinterpret_cast<const uint4*>(p.c.v + p.c.block_at(page, head) + (long long)(tok & ((1 << p.c.shift) - 1)) * p.c.dim + 16 * slice));
    };
    int found = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint4 w = codes(token(i));
        found |= finite_codes(w.x) != w.x || finite_codes(w.y) != w.y || finite_codes(w.z) != w.z || finite_codes(w.w) != w.w;
    }
    if (!__syncthreads_or(found)) return;
    const long long work = (long long)v.n_q * p.group * 16;
    for (long long i = threadIdx.x; i < work; i += kThreads) {
        const int d = (int)(i & 15), r = (int)(i >> 4), qi = r / p.group, h = head * p.group + r - qi * p.group;
        const int hi = min(v.len, hi_of(p, v, qi)), lo = lo_of(p, v, qi);
        float add = 0.f;
        for (int j = 0; j < n; j++) {
            const int tok = token(j);
            if (tok < lo || tok >= hi) continue;
            const uint4 w = codes(tok);
            const uint32_t word = d < 4 ? w.x : d < 8 ? w.y : d < 12 ? w.z : w.w, c = (word >> (8 * (d & 3))) & 0xFFu;
            if (c == 0x80u || (c & 0x7Fu) == 0x6Fu) add += __uint_as_float(decode_bits_f32(c));
        }
        if (add != 0.f) {  // (an Inf or a NaN)
            unsigned short* out = reinterpret_cast<unsigned short*>(p.out) + (long long)(v.first + qi) * p.out_token + (long long)h * p.out_head + 16 * slice + d;
            *out = (unsigned short)to_bits<DT>(q_value<DT>(*out) + add);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------
constexpr int kMaxGroups = 148 * 4;
constexpr size_t kHeadBytes = 256 + ((size_t)HIF8_CACHE_MAX_SEQS + 1) * 8 + 248;  // status word, chunks in front of each sequence
static_assert(kHeadBytes % 256 == 0, "what follows is aligned");

size_t round_up_256(size_t n) { return (n + 255) & ~(size_t)255; }

// n8 tiles of query rows that a warp takes: two where the rows fill more than one and the registers allow it
int row_tiles_of(int max_q, int group, int dim) { return (long long)max_q * group > 8 && dim <= 128 ? 2 : 1; }

size_t partial_bytes(int dim, int nt)
{
    const int per_cta = dim == 256 ? 2 : (dim == 128 && nt == 2 ? 3 : 4);
    return round_up_256((size_t)2 * (kMaxGroups / 4 * per_cta) * 8 * nt * (dim + 2) * 4);
}

struct DeviceSetup {
    cudaError_t rc;
};
PerDevice<DeviceSetup> g_setup;

template <int D, int NT, int DT>
cudaError_t allow_shared()
{
    return cudaFuncSetAttribute((const void*)cache_attention_rows_kernel<D, NT, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RowsShape<D, NT>::kSmem);
}
template <int DT>
cudaError_t allow_shared_of()
{
    cudaError_t e[5] = {allow_shared<64, 1, DT>(), allow_shared<64, 2, DT>(), allow_shared<128, 1, DT>(), allow_shared<128, 2, DT>(), allow_shared<256, 1, DT>()};
    for (cudaError_t x : e)
        if (x != cudaSuccess) return x;
    return cudaSuccess;
}

template <int D, int NT, int DT>
cudaError_t launch_rows(const AttentionParams& p, int sms, cudaStream_t st)
{
    using S = RowsShape<D, NT>;
    cudaLaunchConfig_t cfg{};
    const int ctas = sms < kMaxGroups / 4 ? sms : kMaxGroups / 4;
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t rc = cudaLaunchKernelEx(&cfg, cache_attention_rows_kernel<D, NT, DT>, p);
    if (rc != cudaSuccess) return rc;
    const int groups = ctas * S::kGroups;
    rc = launch_pdl_threads(kCombineThreads, cache_attention_combine_kernel<D, NT, DT>, dim3((unsigned)(groups - 1)), st, p, groups);
    g_launches.fetch_add(2, std::memory_order_relaxed);
    return rc;
}
template <int DT>
cudaError_t launch_rows_of(const AttentionParams& p, int nt, int sms, cudaStream_t st)
{
    if (p.c.dim == 64) return nt == 2 ? launch_rows<64, 2, DT>(p, sms, st) : launch_rows<64, 1, DT>(p, sms, st);
    if (p.c.dim == 128) return nt == 2 ? launch_rows<128, 2, DT>(p, sms, st) : launch_rows<128, 1, DT>(p, sms, st);
    return launch_rows<256, 1, DT>(p, sms, st);
}

}  // namespace
}  // namespace hif8

using namespace hif8;

extern "C" size_t hif8_cache_attention_workspace_bytes(int n_seqs, int n_q, int max_q, int max_length, int heads, int kv_heads, int head_dim)
{
    if (n_seqs < 0 || n_q < 0 || max_q < 0 || max_length < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || (head_dim != 64 && head_dim != 128 && head_dim != 256)) return 0;
    return kHeadBytes + partial_bytes(head_dim, row_tiles_of(max_q, heads / kv_heads, head_dim));
}

extern "C" int hif8_cache_attention(const void* q, int dtype, int64_t q_token_stride, int64_t q_head_stride, const int* d_q_start, const int* d_lengths, int n_seqs, int n_q,
                                    int max_q, int max_length, const uint8_t* k_pages, const uint8_t* v_pages, const int* k_exp, const int* v_exp, int n_pages,
                                    int kv_heads, int page_tokens, int head_dim, const int* page_table, int64_t table_stride, int heads, float softmax_scale, int causal,
                                    int window, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace, size_t workspace_bytes,
                                    hif8_stream_t stream)
{
    if (dtype != HIF8_BF16 && dtype != HIF8_F16) return HIF8_ERR_DTYPE;
    if (n_seqs < 0 || n_seqs > HIF8_CACHE_MAX_SEQS || n_q < 0 || max_q < 0 || max_length < 0 || window < 0) return HIF8_ERR_SHAPE;
    if (q_token_stride < 0 || q_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0) return HIF8_ERR_SHAPE;
    AttentionParams p;
    if (int rc = check_cache(k_pages, v_pages, k_exp, v_exp, n_pages, kv_heads, page_tokens, head_dim, page_table, table_stride, &p.c)) return rc;
    if (heads < 1 || heads % kv_heads || heads / kv_heads > HIF8_CACHE_MAX_GROUP) return HIF8_ERR_SHAPE;
    if (!(softmax_scale > 0.f) || !(softmax_scale <= 3.4e38f)) return HIF8_ERR_SCALE_RANGE;
    if ((int64_t)n_q * (heads / kv_heads) > 0x3FFFFFFF) return HIF8_ERR_SHAPE;
    if (n_seqs == 0 || n_q == 0) return HIF8_OK;
    if (!q || !out || !d_q_start || !d_lengths) return HIF8_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 1u) return HIF8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(d_q_start) | reinterpret_cast<uintptr_t>(d_lengths) | reinterpret_cast<uintptr_t>(lse)) & 3u) return HIF8_ERR_ALIGN;
    // rows of the result must not share elements: tokens outermost, or heads
    const int64_t inner = out_token_stride < out_head_stride ? out_token_stride : out_head_stride, outer = out_token_stride < out_head_stride ? out_head_stride : out_token_stride;
    const int64_t n_inner = out_token_stride < out_head_stride ? n_q : heads, n_outer = out_token_stride < out_head_stride ? heads : n_q;
    if ((n_inner > 1 && inner < head_dim) || (n_outer > 1 && outer < (n_inner - 1) * inner + head_dim)) return HIF8_ERR_SHAPE;
    const size_t q_bytes = ((size_t)(n_q - 1) * (size_t)q_token_stride + (size_t)(heads - 1) * (size_t)q_head_stride + (size_t)head_dim) * 2;
    const size_t out_bytes = ((size_t)(n_q - 1) * (size_t)out_token_stride + (size_t)(heads - 1) * (size_t)out_head_stride + (size_t)head_dim) * 2;
    const size_t pool = (size_t)n_pages * (size_t)p.c.page_bytes();
    if (ranges_overlap(q, q_bytes, out, out_bytes) || ranges_overlap(k_pages, pool, out, out_bytes) || ranges_overlap(v_pages, pool, out, out_bytes)) return HIF8_ERR_OVERLAP;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HIF8_ERR_WORKSPACE;
    const int group = heads / kv_heads, nt = row_tiles_of(max_q, group, head_dim);
    if (workspace_bytes < kHeadBytes + partial_bytes(head_dim, nt)) return HIF8_ERR_WORKSPACE;
    int sms; if (int rc = checked_device(&sms)) return rc;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HIF8_ERR_CUDA;
    const DeviceSetup* setup = g_setup.get(dev, [](int, DeviceSetup* o) {
        o->rc = allow_shared_of<HIF8_BF16>();
        if (o->rc == cudaSuccess) o->rc = allow_shared_of<HIF8_F16>();
    });
    if (!setup || setup->rc != cudaSuccess) return HIF8_ERR_CUDA;
    p.q = q; p.q_token = q_token_stride; p.q_head = q_head_stride; p.q_start = d_q_start; p.lengths = d_lengths; p.n_seqs = n_seqs; p.n_q = n_q; p.heads = heads; p.group = group;
    p.vectors = !((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) && !((q_token_stride | q_head_stride | out_token_stride | out_head_stride) & 7);
    p.scale_log2 = fminf(softmax_scale * kLog2e, 3.0e38f); p.causal = causal != 0; p.window = window;
    p.out = out; p.out_token = out_token_stride; p.out_head = out_head_stride; p.lse = lse;
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
    p.status = reinterpret_cast<int*>(ws);
    p.prefix = reinterpret_cast<long long*>(ws + 256);
    p.partial = reinterpret_cast<float*>(ws + kHeadBytes);
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t rc = dtype == HIF8_BF16 ? launch_rows_of<HIF8_BF16>(p, nt, sms, st) : launch_rows_of<HIF8_F16>(p, nt, sms, st);
    if (rc == cudaSuccess && max_q > 1 && (p.causal || p.window)) {
        const dim3 grid((unsigned)(head_dim / 16), (unsigned)kv_heads, (unsigned)n_seqs);
        rc = dtype == HIF8_BF16 ? launch_pdl(cache_attention_specials_kernel<HIF8_BF16>, grid, st, p) : launch_pdl(cache_attention_specials_kernel<HIF8_F16>, grid, st, p);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    note_status_word(st, p.status);
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}
