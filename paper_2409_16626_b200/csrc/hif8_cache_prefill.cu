// Attention over the HiF8 key/value cache for many query rows (chunks of prompts): bound by the products, so it runs on the tensor cores (tcgen05).
//
// Three steps.  (1) plan: where each sequence's tokens lie in the workspace, how many tiles of 128 tokens each pair of row tiles has to look at, and where blocks begin.
// (2) expand: the codes of K and V that are looked at and the queries become FP16 tiles in the workspace (exact, see hif8_cache_attention.cu; the queries
// packed by key head, with the power of two they are scaled by aside), once for all rows that use them: 5 bytes of traffic a code, 3 % of the time of
// a chunk of 2048 queries against 16 K tokens.  Decoding inside the product kernel was not built: with 256 query rows to a tile of keys its lookups and stores
// would take 1500 cycles of shared memory beside the 1500 that the products' operands take, and a tile's products take 2048.
// (3) attention: a block holds two tiles of 128 query rows.  For each, S = Q K^T goes to tensor memory, four warps (a thread a row) turn it into P = 2^(x - m + 4) in
// FP16, written over S, and O += P V accumulates in tensor memory; while one tile's warps work, the tensor cores do the other tile's products.  O is only
// rescaled when a row's maximum has grown by more than 2^8 (P stays below 2^12), by the warps themselves: the next scores' barrier says that the sums are not in use.
// All units are dealt out over the blocks by a cost of their tiles and of themselves; a unit that several blocks share leaves FP32 parts, which a last kernel joins in a fixed order.
//
// Measured: a chunk of 2048 queries against 16461 tokens, 32/8 heads of 128: 515 to 520 us a call (1000 TFLOP/s; cuBLAS sustains 1346 to 1384 here at the same 1000 W), 465 of them in the
// attention kernel, whose tensor pipe is busy 59 % of the time and the exponentials' unit as long.  A pair of tiles takes 3250 cycles where the products alone take 2048: what a row
// tile's warps do to its scores (load 90, maximum 380, weights 1650 cycles) and its products (770, and 500 until each side has noticed the other) make a chain
// as long as that, and two row tiles are what tensor memory holds.  Exponentials as polynomials on the FMA pipe, for an eighth to half of the elements, made it slower (531 ->
// 534 to 558 us), and so did a warp of its own to issue each row tile's products (540 -> 588).
#include "hif8_cache_attention.cuh"

namespace hif8 {
namespace {

constexpr int kTileRows = 128, kTileTokens = 128;
constexpr float kShift = 4.f, kLazy = 8.f;
// Row tiles of a block: two, except for heads of 256, whose sums take half of tensor memory: there the two places of scores belong to consecutive tiles of tokens.
template <int D> struct TileShape {
    static constexpr int kTiles = D == 256 ? 1 : 2, kUnitRows = kTiles * kTileRows;
    static constexpr int kStages = D == 256 ? 2 : 4;  // (heads of 256: one for keys, one for values)
};
constexpr int kTmaWarp = 8, kMmaWarp = 9, kPlanWarp = 10, kThreadsA = 12 * 32;
// Registers: 168 a thread at launch, 64512 in all; the eight warps that hold rows of scores take 208, the third group of four warps (one of them idle) 88.
constexpr int kRegsRows = 208, kRegsOther = 88;
static_assert(256 * kRegsRows + 128 * kRegsOther <= kThreadsA * 168, "no more than the block has");
constexpr int kMetaRing = 8, kSegRing = 4;
__device__ __forceinline__ bool warp_all(bool x) { return __all_sync(0xFFFFFFFFu, x); }
__device__ __forceinline__ bool warp_any(bool x) { return __any_sync(0xFFFFFFFFu, x); }

struct PrefillParams {
    AttentionParams a;
    __half* kx;            // [heads][cap_blocks * 128][dim]
    __half* vx;
    __half* qx;            // [heads][n_q * group][dim]
    float* q_mul;          // [heads][n_q * group]: the row's part of a score's factor (query_factor)
    float4* meta;          // [heads][cap_blocks * 8]: of 16 tokens: 2^-e_k, -e_v (-Inf: no page), 2^e_v
    int* block_at;         // [n_seqs + 1] first 128-token block of each sequence
    long long* tiles_at;   // [pairs + 1] tiles in front of each pair of row tiles (of one head)
    int* units_at;         // [pairs] those of the pairs in front that have tiles
    int* pair_seq;         // [pairs]
    long long* bound;      // [blocks + 1] first tile of each block: heads x tiles_at
    int4* cut;             // [blocks] two of each, of the unit that the block's first tile lies in: tiles in front of that one, tiles, key head, first row; first query, rows, pair
    int* specials;         // set when some token that a query sees holds Inf or NaN in V
    int cap_blocks, pairs, blocks;
    long long rows;        // n_q * group
    int unit_rows;         // query rows of a unit
};

// pairs of row tiles of the sequence, and their numbers: from first_pair on (see Piece: no sums over the batch)
__device__ __forceinline__ long long first_pair(const PrefillParams& p, int s) { return ((long long)start_at(p.a.q_start, s, p.a.n_q) * p.a.group) / p.unit_rows + s; }

struct PairView {
    int seq, r0, n_rows, base, j0, tiles;  // rows r0 .. of the sequence; first token of its blocks in the workspace; first tile, tiles
    int lo_min, lo_max, hi_min, hi_max;    // what the rows look at
    SeqView v;
};
__device__ __forceinline__ PairView pair_view(const PrefillParams& p, int seq, long long number)
{
    PairView u;
    u.seq = seq;
    u.v = seq_view(p.a, seq);
    const long long i = number - first_pair(p, seq), rows = (long long)u.v.n_q * p.a.group;
    u.base = lo_of(p.a, u.v, 0) / kTileTokens * kTileTokens;
    u.r0 = (int)(i * p.unit_rows);
    u.n_rows = i < 0 || i * p.unit_rows >= rows ? 0 : (int)min((long long)p.unit_rows, rows - i * p.unit_rows);
    if (!u.n_rows) { u.r0 = u.j0 = u.tiles = u.lo_min = u.lo_max = u.hi_min = u.hi_max = 0; return u; }
    const int qa = u.r0 / p.a.group, qb = (u.r0 + u.n_rows - 1) / p.a.group;
    u.lo_min = lo_of(p.a, u.v, qa); u.lo_max = lo_of(p.a, u.v, qb);
    u.hi_min = min(u.v.len, hi_of(p.a, u.v, qa)); u.hi_max = min(u.v.len, hi_of(p.a, u.v, qb));
    u.j0 = min(u.lo_min, max(u.v.len - 1, 0)) / kTileTokens - u.base / kTileTokens;
    u.tiles = max(1, (u.hi_max - u.base + kTileTokens - 1) / kTileTokens - u.j0);
    return u;
}

// ---------------------------------------------------------------------------------------------------------
// Plan
// ---------------------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;
// What is dealt out evenly: two for a tile, three for a unit (its queries, its results, and tiles that are masked; heads of 64: 3600 cycles a tile, 4900 a unit.  By tiles alone blocks
// of 12 prompts of up to 2047 tokens with a window of 700 had 5 to 12 units and took 128 to 162 thousand cycles.  us with two / three / four / five for a unit: heads of 128, 8 prompts of 1000
// 180 / 175 / 174 / 174, 8 of 2000 449 / 443 / 444 / 446, 30 of up to 500 147 / 145 / 145 / 148; of 64, 8 of 2000 328 / 326 / 330 / 333; of 256, 4 of 2000 240 / 232 / 231 / 233).
constexpr int kTileCost = 2, kUnitCost = 3;
__device__ __forceinline__ long long plan_prefix(long long v, long long* total, long long* s_warp)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    long long w = s_warp[lane];  // (32 warps)
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, w, d);
        if (lane >= d) w += y;
    }
    *total = __shfl_sync(0xFFFFFFFFu, w, 31);
    const long long before = __shfl_sync(0xFFFFFFFFu, w, warp ? warp - 1 : 0);
    return (warp ? before : 0) + x - v;
}

__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(const PrefillParams p)
{
    __shared__ long long s_warp[32];
    __shared__ long long s_cost[kPlanThreads];  // in front of each pair, and of each: tiles, first row, first query of its sequence, rows
    __shared__ int4 s_info[kPlanThreads];
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    if (threadIdx.x == 0) { *p.a.status = 0; *p.specials = 0; }
    long long carry = 0, total;
    for (int s0 = 0; s0 < p.a.n_seqs; s0 += kPlanThreads) {
        const int s = s0 + threadIdx.x;
        long long n = 0;
        if (s < p.a.n_seqs) {
            const SeqView v = seq_view(p.a, s);
            const int base = lo_of(p.a, v, 0) / kTileTokens * kTileTokens;
            n = v.n_q ? max(1, (v.len - base + kTileTokens - 1) / kTileTokens) : 0;
        }
        const long long before = carry + plan_prefix(n, &total, s_warp);
        if (s < p.a.n_seqs) p.block_at[s] = (int)min(before, (long long)p.cap_blocks);
        carry += total;
    }
    if (threadIdx.x == 0) p.block_at[p.a.n_seqs] = (int)min(carry, (long long)p.cap_blocks);
    long long carry_units = 0;
    carry = 0;
    for (int x0 = 0; x0 < p.pairs; x0 += kPlanThreads) {
        const int x = x0 + threadIdx.x;
        long long n = 0;
        int4 info = make_int4(0, 0, 0, 0);
        if (x < p.pairs) {
            int s = 0;
            for (int k = p.a.n_seqs; k > 1;) {
                const int half = k >> 1;
                if (first_pair(p, s + half) <= x) { s += half; k -= half; }
                else k = half;
            }
            p.pair_seq[x] = s;
            const PairView u = pair_view(p, s, x);
            n = u.tiles;
            info = make_int4(u.tiles, u.r0, u.v.first, u.n_rows);
        }
        const long long before = carry + plan_prefix(n, &total, s_warp);
        if (x < p.pairs) p.tiles_at[x] = before;
        carry += total;
        const long long units = carry_units + plan_prefix(n > 0, &total, s_warp);
        if (x < p.pairs) p.units_at[x] = (int)units;
        if (x < kPlanThreads) { s_cost[x] = kTileCost * before + kUnitCost * units; s_info[x] = info; }
        carry_units += total;
    }
    if (threadIdx.x == 0) p.tiles_at[p.pairs] = carry;
    __syncthreads();
    // Where each block begins.  (Few pairs, as small calls have them, are looked for in shared memory.)
    const bool here = p.pairs <= kPlanThreads;
    const long long cost = kTileCost * carry + kUnitCost * carry_units;  // of a head
    for (int b = threadIdx.x; b <= p.blocks; b += kPlanThreads) {
        if (b == p.blocks || !carry) { p.bound[b] = carry * p.a.c.heads; continue; }
        const long long at = share_of(cost * p.a.c.heads, b, p.blocks);
        const int head = (int)(at / cost);
        const long long off = at - head * cost;
        int a = 0;  // the last pair that begins at or before that (empty ones share their start with the next)
        for (int k = p.pairs; k > 1;) {
            const int half = k >> 1;
            if ((here ? s_cost[a + half] : kTileCost * p.tiles_at[a + half] + kUnitCost * p.units_at[a + half]) <= off) { a += half; k -= half; }
            else k = half;
        }
        int4 of = s_info[here ? a : 0];
        if (!here) {
            const PairView u = pair_view(p, p.pair_seq[a], a);
            of = make_int4(u.tiles, u.r0, u.v.first, u.n_rows);
        }
        const int tiles = of.x;
        const long long tiles_at = p.tiles_at[a], in = off - (here ? s_cost[a] : kTileCost * tiles_at + kUnitCost * p.units_at[a]) - kUnitCost;
        int c = in <= 0 ? 0 : (int)min((long long)tiles, (in + kTileCost / 2) / kTileCost);
        if (cost * p.a.c.heads >= 4ll * kTileCost * p.blocks) {  // a tile alone is not worth a segment
            if (c == 1) c = 0;
            else if (c && c == tiles - 1) c = tiles;
        }
        p.bound[b] = head * carry + tiles_at + c;
        const bool next = c == tiles;  // it begins with the next unit, whichever that is
        p.cut[2 * b] = make_int4(next ? 0 : c, tiles, head, of.y);
        p.cut[2 * b + 1] = make_int4(of.z, of.w, next ? -1 : a, 0);
    }
}

// ---------------------------------------------------------------------------------------------------------
// Expand
// ---------------------------------------------------------------------------------------------------------
// A block takes units in turn: 128 tokens of one head of K or V, and behind all of those 32 KiB of query rows.
template <int D, int DT>
__global__ void __launch_bounds__(kThreads) cache_expand_kernel(const PrefillParams p)
{
    __shared__ __align__(16) uint32_t table[kLaneTableWords];
    fill_lane_table(table, g_f16_of_code.v[threadIdx.x]);  // kThreads == 256 codes
    __syncthreads();
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const CacheView& c = p.a.c;
    constexpr int kLanes = D / 8, kRowsWarp = 32 / kLanes, kUnroll4 = 4, kRowsUnit = 8 * kRowsWarp * kUnroll4;  // lanes to a query row, rows of a warp at a time, rows of a unit
    const int n_blocks = p.block_at[p.a.n_seqs];
    const long long code_units = 2ll * n_blocks * c.heads, rows = (long long)p.a.n_q * p.a.heads, units = code_units + (rows + kRowsUnit - 1) / kRowsUnit;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        if (u < code_units) {  // a warp takes 16 tokens, which lie in one page
            const int blk = (int)(div_small(u, 2 * c.heads)), part = (int)(u - (long long)blk * 2 * c.heads), head = part >> 1;
            const bool is_v = part & 1;
            int s = 0;
            for (int k = p.a.n_seqs; k > 1;) {  // (sequences without blocks share their start with the next)
                const int half = k >> 1;
                if (p.block_at[s + half] <= blk) { s += half; k -= half; }
                else k = half;
            }
            const SeqView v = seq_view(p.a, s);
            const int base = lo_of(p.a, v, 0) / kTileTokens * kTileTokens, t0 = base + (blk - p.block_at[s]) * kTileTokens + 16 * warp;
            const int hi0 = min(v.len, hi_of(p.a, v, 0)), hi1 = min(v.len, hi_of(p.a, v, v.n_q - 1)), lo0 = lo_of(p.a, v, 0), lo1 = lo_of(p.a, v, v.n_q - 1);
            const bool seen = t0 < hi1 && t0 + 16 > lo0;
            const int page = seen ? c.page_of(s, t0 >> c.shift) : -1;
            const long long row = ((long long)head * p.cap_blocks + blk) * kTileTokens + 16 * warp;
            const uint8_t* src = (is_v ? c.v : c.k) + c.block_at(max(page, 0), head) + (long long)(t0 & ((1 << c.shift) - 1)) * D;
            uint4* dst = reinterpret_cast<uint4*>((is_v ? p.vx : p.kx) + row * D);
            constexpr int kSteps = 16 * D / 8 / 32;  // eight codes a lane and step
            uint2 w[kSteps];
#pragma unroll
            for (int i = 0; i < kSteps; i++) w[i] = page >= 0 ? __ldg(reinterpret_cast<const uint2*>(src) + lane + 32 * i) : make_uint2(0, 0);
            const int exponent = page >= 0 ? clamp_cache_exp((is_v ? c.v_exp : c.k_exp)[(long long)page * c.heads + head]) : 0;
            bool some = false;  // of the values is not zero
#pragma unroll
            for (int i = 0; i < kSteps; i++) {
                // tokens that no query sees are not there; Inf and NaN of V are left to cache_attention_specials_kernel (0 times them would reach queries that do not see them, and
                // make NaN of an Inf)
                const int tok = t0 + (lane + 32 * i) * 8 / D;
                if (tok < lo0 || tok >= hi1) w[i] = make_uint2(0, 0);
                else if (is_v) {
                    const uint2 f = make_uint2(finite_codes(w[i].x), finite_codes(w[i].y));
                    if (f.x != w[i].x || f.y != w[i].y) *p.specials = 1;
                    w[i] = f;
                }
                some |= (w[i].x | w[i].y) != 0u;
                const uint2 a = lane_lookup4(table, w[i].x, 4u * lane), b = lane_lookup4(table, w[i].y, 4u * lane);
                dst[lane + 32 * i] = make_uint4(a.x, a.y, b.x, b.y);
            }
            // Values that are zeros have no say in what the weights refer to: they count as values of the largest exponent.  (Their blocks have exponent 0, which would push
            // the weights of small values in other blocks out of FP16.)
            const int ve = warp_any(some) ? exponent : HIF8_CACHE_EXP_MAX;
            if (lane == 0) {
                float* meta = reinterpret_cast<float*>(p.meta + (row >> 4));
                if (is_v) *reinterpret_cast<float2*>(meta) = make_float2(page >= 0 ? (float)-ve : kNegInf, pow2f(ve));
                else meta[2] = pow2f(kMulShift - exponent);
            }
            continue;
        }
        // query rows: eight elements a lane
        uint4 w[kUnroll4];
        long long r[kUnroll4], to[kUnroll4];
#pragma unroll
        for (int x = 0; x < kUnroll4; x++) {
            r[x] = (u - code_units) * kRowsUnit + (x * 8 + warp) * kRowsWarp + lane / kLanes;
            w[x] = make_uint4(0, 0, 0, 0);
            to[x] = 0;
            if (r[x] < rows) {
                const int tok = (int)div_small(r[x], p.a.heads), h = (int)(r[x] - (long long)tok * p.a.heads), head = h / p.a.group;
                to[x] = head * p.rows + (long long)tok * p.a.group + (h - head * p.a.group);
                const unsigned short* src = reinterpret_cast<const unsigned short*>(p.a.q) + (long long)tok * p.a.q_token + (long long)h * p.a.q_head + 8 * (lane % kLanes);
                if (p.a.vectors) w[x] = __ldcs(reinterpret_cast<const uint4*>(src));
                else {
                    uint32_t a[4];
#pragma unroll
                    for (int y = 0; y < 4; y++) a[y] = (uint32_t)src[2 * y] | ((uint32_t)src[2 * y + 1] << 16);
                    w[x] = make_uint4(a[0], a[1], a[2], a[3]);
                }
            }
        }
#pragma unroll
        for (int x = 0; x < kUnroll4; x++) {
            int e = 0;
            if (DT == HIF8_BF16) {
                float a = amax_value<DT>(amax_vector<DT>(0u, w[x]));
#pragma unroll
                for (int d = 1; d < kLanes; d *= 2) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, d));
                e = query_exp(a);
                const float f = pow2f(e);
                w[x] = make_uint4(pack_f16(q_value<DT>(w[x].x & 0xFFFFu) * f, q_value<DT>(w[x].x >> 16) * f), pack_f16(q_value<DT>(w[x].y & 0xFFFFu) * f, q_value<DT>(w[x].y >> 16) * f),
                                  pack_f16(q_value<DT>(w[x].z & 0xFFFFu) * f, q_value<DT>(w[x].z >> 16) * f), pack_f16(q_value<DT>(w[x].w & 0xFFFFu) * f, q_value<DT>(w[x].w >> 16) * f));
            }
            if (r[x] < rows) {
                *reinterpret_cast<uint4*>(p.qx + to[x] * D + 8 * (lane % kLanes)) = w[x];
                if (lane % kLanes == 0) p.q_mul[to[x]] = query_factor(p.a.scale_log2, e);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) { asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tc_mma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// A (128 rows) in tensor memory: row i in lane i, two FP16 a column
__device__ __forceinline__ void tc_mma_f16_a_tmem(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// shared-memory matrix descriptor: start address, leading / stride byte offsets (16-byte units), version 1, 128-byte swizzle
__device__ __forceinline__ uint64_t make_smem_desc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16 | (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void tmem_ld_x32(uint32_t taddr, uint32_t* r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t* r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
          "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// What the planning warp tells the others of a segment: tiles c0 .. c1 of a unit (a pair of row tiles of a sequence and key head).  tiles == 0: there is no other.
struct SegmentInfo {
    int tiles, head, first, n_q, len, r0, n_rows, t0, lo_max, hi_min, whole, from_start;  // t0: first token of the first tile; whole: c0 == 0 and c1 the unit's tiles
    int q_row, block0, pad[2];                                                          // first row of the packed queries, first block of tokens
};
static_assert(sizeof(SegmentInfo) == 64, "read in 16-byte pieces");

template <int D>
struct PrefillSmem {
    static constexpr int kStages = TileShape<D>::kStages, kTiles = TileShape<D>::kTiles;
    static constexpr int kQBufs = D == 64 ? 2 : 1;  // (short units, as windows and short prompts have them, wait for their queries otherwise: see the kernel's figures)
    // Heads of 64: the two row tiles' warps take turns with their exponentials, or both would want them at once and then both wait for products (1000 queries against 8000 tokens,
    // 32/8 heads: 136 -> 122 us; heads of 128, whose products keep them apart: 152 -> 154).
    static constexpr bool kTurns = D == 64;
    static constexpr uint32_t kQ = kTileRows * D * 2, kStage = kTileTokens * D * 2;
    static constexpr uint32_t q = 0, stages = kQBufs * kTiles * kQ, out = stages + kStages * kStage, meta = out + 4 * kTiles * 4096, seg = meta + kMetaRing * 128, bars = seg + kSegRing * 64;
    // barriers: queries there / free, stages full / empty, factors of a tile there, segment told / read, scores there [2], weights there (half of them, all) [2], sums complete, a tile's products with
    // values done (one row tile), sums read, all products ended (after a wait that gave up)
    static constexpr uint32_t q_full = bars, q_empty = q_full + 8 * kQBufs, full = q_empty + 8 * kQBufs, empty = full + 8 * kStages, meta_full = empty + 8 * kStages,
                              seg_full = meta_full + 8 * kMetaRing, seg_empty = seg_full + 8 * kSegRing, s_full = seg_empty + 8 * kSegRing, p_half = s_full + 16, p_full = p_half + 16,
                              o_full = p_full + 16, pv_done = o_full + 8, o_empty = pv_done + 8, drain = o_empty + 8, turn = drain + 8, tmem_slot = turn + 64, abort_flag = tmem_slot + 4, total = abort_flag + 4;
    static constexpr uint32_t kBytes = total + 1024;
    static_assert(kBytes <= 227 * 1024, "shared memory");
};

template <int D> struct Record {
    static constexpr int kRows = TileShape<D>::kUnitRows;
    static constexpr size_t floats = (size_t)kRows * (D + 2);
};

// a segment: tiles c0 .. c1 of a unit
struct Segment {
    PairView u;
    int head, c0, c1;
    __device__ Segment(const PrefillParams& p, long long x0, long long x_end, int pair, int head_)  // (the first one of a block)
    {
        const long long per_head = p.tiles_at[p.pairs];
        head = head_;
        set(p, pair, x0 - head * per_head, x_end - x0);
    }
    __device__ Segment(const PrefillParams& p, long long x0, long long x_end)
    {
        const long long per_head = p.tiles_at[p.pairs];
        head = (int)(x0 / per_head);
        const long long x = x0 - head * per_head;
        int a = 0;  // last pair that starts at or before x (empty ones share their start with the next); one probe a lane and round
        for (int n = p.pairs; n > 1;) {
            const int step = (n + 31) >> 5, i = ((int)threadIdx.x & 31) * step;
            const int last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, i == 0 || (i < n && p.tiles_at[a + i] <= x)));
            a += last * step;
            n = min(step, n - last * step);
        }
        set(p, a, x, x_end - x0);
    }
    __device__ void set(const PrefillParams& p, int a, long long x, long long left)
    {
        u = pair_view(p, p.pair_seq[a], a);
        c0 = (int)(x - p.tiles_at[a]);
        c1 = (int)min((long long)u.tiles, c0 + left);
    }
};

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint64_t pack2(float a, float b)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void unpack2(uint64_t d, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(d)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float4 lds_f4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts_v4(uint32_t addr, uint4 v) { asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }
// `bytes` (a multiple of 16) from global to shared memory
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <int D, int DT>
__global__ void __launch_bounds__(kThreadsA, 1) cache_attention_tiles_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                             const __grid_constant__ CUtensorMap map_v, const PrefillParams p)
{
    using L = PrefillSmem<D>;
    constexpr int kTiles = L::kTiles, kStages = L::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* sm = smem_raw + (base - smem_u32(smem_raw));
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + L::abort_flag);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + L::tmem_slot);
    auto bar = [&](uint32_t at, int i = 0) { return base + at + 8u * i; };
    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kQBufs; i++) { mbar_init(bar(L::q_full, i), 1); mbar_init(bar(L::q_empty, i), 1); }
        for (int i = 0; i < kStages; i++) { mbar_init(bar(L::full, i), 1); mbar_init(bar(L::empty, i), 1); }
        for (int i = 0; i < kMetaRing; i++) mbar_init(bar(L::meta_full, i), 1);
        for (int i = 0; i < kSegRing; i++) { mbar_init(bar(L::seg_full, i), 1); mbar_init(bar(L::seg_empty, i), 2 + 4 * kTiles); }  // (read by the copying warp, the products' and the rows')
        for (int i = 0; i < 2; i++) { mbar_init(bar(L::s_full, i), 1); mbar_init(bar(L::p_half, i), 4); mbar_init(bar(L::p_full, i), 4); }
        mbar_init(bar(L::o_full), 1); mbar_init(bar(L::pv_done), 1); mbar_init(bar(L::o_empty), 4 * kTiles); mbar_init(bar(L::drain), 1);
        for (int i = 0; i < 8; i++) mbar_init(bar(L::turn, i), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::tmem_slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait_prior_grid();
    pdl_launch_dependents();

    // tensor memory: scores (and weights over them) of the two tiles at columns 0 and 128, sums at 256 and 384 (one row tile: scores of tiles of tokens in turn, sums from 256 on)
    const int me = blockIdx.x;
    bool ok = true;
    uint32_t seg = 0;  // segments so far
    auto next_segment = [&](SegmentInfo& g, int where) -> bool {  // as the planning warp tells it
        ok = warp_all(mbar_wait(bar(L::seg_full, seg % kSegRing), (seg / kSegRing) & 1u, abort_flag, p.a.status, where));
        if (!ok) return false;
        const int4* from = reinterpret_cast<const int4*>(sm + L::seg + (seg % kSegRing) * 64);
        const int4 a = from[0], b = from[1], c = from[2], d = from[3];
        g.tiles = a.x; g.head = a.y; g.first = a.z; g.n_q = a.w; g.len = b.x; g.r0 = b.y; g.n_rows = b.z; g.t0 = b.w; g.lo_max = c.x; g.hi_min = c.y; g.whole = c.z; g.from_start = c.w;
        g.q_row = d.x; g.block0 = d.y;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(L::seg_empty, seg % kSegRing));
        return g.tiles > 0;
    };

    // (each branch sets its own count of registers: the compiler works by the smallest that reaches a place)
    if (warp >= kTmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kPlanWarp) {  // up to kSegRing segments ahead: finding one takes a handful of loads that wait for one another
        long long x0 = p.bound[me];
        const long long x_end = p.bound[me + 1];
        for (bool more = true; more; seg++) {
            int4 info[4] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
            more = x0 < x_end;
            if (more) {
                const int known = seg == 0 ? p.cut[2 * me + 1].z : -1;  // the pair that it begins in
                const Segment g = known >= 0 ? Segment(p, x0, x_end, known, p.cut[2 * me].z) : Segment(p, x0, x_end);
                info[0] = make_int4(g.c1 - g.c0, g.head, g.u.v.first, g.u.v.n_q);
                info[1] = make_int4(g.u.v.len, g.u.r0, g.u.n_rows, g.u.base + (g.u.j0 + g.c0) * kTileTokens);
                info[2] = make_int4(g.u.lo_max, g.u.hi_min, g.c0 == 0 && g.c1 == g.u.tiles, g.c0 == 0);
                info[3] = make_int4((int)(g.head * p.rows + (long long)g.u.v.first * p.a.group + g.u.r0), p.block_at[g.u.seq] + g.u.j0 + g.c0, 0, 0);
                x0 += g.c1 - g.c0;
            }
            if (seg >= kSegRing) ok = warp_all(mbar_wait(bar(L::seg_empty, seg % kSegRing), (seg / kSegRing - 1) & 1u, abort_flag, p.a.status, 84));
            if (!ok) break;
            if (lane == 0) {
                int4* to = reinterpret_cast<int4*>(sm + L::seg + (seg % kSegRing) * 64);
                for (int i = 0; i < 4; i++) to[i] = info[i];
                mbar_arrive(bar(L::seg_full, seg % kSegRing));
            }
            __syncwarp();
        }
    } else if (warp == kTmaWarp) {
        uint32_t n[2] = {0, 0}, tile = 0;  // copies of keys, of values; tiles so far
        SegmentInfo g;
        while (next_segment(g, 85)) {
            const bool two = g.n_rows > kTileRows;
            const uint32_t qb = seg % L::kQBufs;
            if (seg >= L::kQBufs) ok = warp_all(mbar_wait(bar(L::q_empty, qb), (seg / L::kQBufs - 1) & 1u, abort_flag, p.a.status, 71));
            if (!ok) break;
            if (elect_one()) {
                mbar_expect(bar(L::q_full, qb), two ? 2 * L::kQ : L::kQ);
                for (int i = 0; i < (two ? 2 : 1); i++)
#pragma unroll
                    for (int c = 0; c < D / 64; c++)
                        tma_load_2d(base + L::q + (kTiles * qb + i) * L::kQ + c * (kTileRows * 128), &map_q, c * 64, g.q_row + i * kTileRows, bar(L::q_full, qb));
            }
            __syncwarp();
            seg++;
            auto copy = [&](int kv, int j, uint32_t st, uint32_t round) {  // keys or values of tile j into stage st, its round-th use
                const int blk = min(g.block0 + j, p.cap_blocks - 1);  // (beyond: lengths above max_length)
                const int row = (int)(((long long)g.head * p.cap_blocks + blk) * kTileTokens);
                if (round) ok = warp_all(mbar_wait(bar(L::empty, st), (round - 1) & 1u, abort_flag, p.a.status, 72));
                if (!ok) return;
                if (elect_one()) {
                    const uint32_t to = base + L::stages + st * L::kStage;
                    mbar_expect(bar(L::full, st), L::kStage);
#pragma unroll
                    for (int c = 0; c < D / 64; c++) tma_load_2d(to + c * (kTileTokens * 128), kv ? &map_v : &map_k, c * 64, row, bar(L::full, st));
                    if (!kv) {  // (eight tiles are kept: keys of tile x are only asked for when the scores of tile x - 2 are there, so the rows are at x - 3 at least)
                        mbar_expect(bar(L::meta_full, (tile + j) % kMetaRing), 128);
                        bulk_load(base + L::meta + (tile + j) % kMetaRing * 128, p.meta + (row >> 4), 128, bar(L::meta_full, (tile + j) % kMetaRing));
                    }
                }
                __syncwarp();
                n[kv]++;
            };
            // in the order in which the products free the stages: keys and values in turn; with one row tile the scores, and so the keys, are a tile ahead
            if (kTiles == 2)
                for (int j = 0; j < g.tiles && ok; j++)
                    for (int kv = 0; kv < 2 && ok; kv++) copy(kv, j, (n[0] + n[1]) % kStages, (n[0] + n[1]) / kStages);
            else
                for (int j = -2; j < g.tiles && ok; j++) {  // K0 | V0 K1 | K2 V1 | K3 V2 ..: (j = -1: V0 needs no wait that K1 does)
                    if (j == -2) copy(0, 0, 0, n[0]);
                    else if (j == -1) {
                        copy(1, 0, 1, n[1]);
                        if (ok && g.tiles > 1) copy(0, 1, 0, n[0]);
                    } else {
                        if (j + 2 < g.tiles) copy(0, j + 2, 0, n[0]);
                        if (ok && j + 1 < g.tiles) copy(1, j + 1, 1, n[1]);
                    }
                }
            if (ok) tile += g.tiles;
            if (!ok) break;
        }
        if (!ok || warp_any(*abort_flag)) {  // copies on their way land before the block's shared memory becomes another's
            for (uint32_t i = seg > L::kQBufs ? seg - L::kQBufs : 0; i < seg; i++) wait_landed(bar(L::q_full, i % L::kQBufs), (i / L::kQBufs) & 1u);
            if (kTiles == 2)
                for (uint32_t all = n[0] + n[1], i = all > kStages ? all - kStages : 0; i < all; i++) wait_landed(bar(L::full, i % kStages), (i / kStages) & 1u);
            else
                for (int kv = 0; kv < 2; kv++)
                    if (n[kv]) wait_landed(bar(L::full, kv), (n[kv] - 1) & 1u);
            for (uint32_t i = n[0] > kMetaRing ? n[0] - kMetaRing : 0; i < n[0]; i++) wait_landed(bar(L::meta_full, i % kMetaRing), (i / kMetaRing) & 1u);
        }
    } else if (warp == kMmaWarp) {
        const uint32_t id_s = (1u << 4) | ((uint32_t)(kTileTokens >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);     // FP16 x FP16 -> FP32, both K-major
        const uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);  // B (the values) MN-major
        uint32_t n = 0, uses[2] = {0, 0};  // ring; weights taken of each tile
        SegmentInfo g;
        while (next_segment(g, 81)) {
            const int both = g.n_rows > kTileRows ? 2 : 1, tiles = g.tiles;
            const uint32_t qb = seg % L::kQBufs;
            ok = warp_all(mbar_wait(bar(L::q_full, qb), (seg / L::kQBufs) & 1u, abort_flag, p.a.status, 73));
            if (!ok) break;
            auto scores = [&](int i, uint32_t st, int place) {
                if (elect_one()) {
                    const uint64_t da = make_smem_desc(base + L::q + (kTiles * qb + i) * L::kQ, 16, 1024), db = make_smem_desc(base + L::stages + st * L::kStage, 16, 1024);
#pragma unroll
                    for (int kk = 0; kk < D / 16; kk++) {
                        const uint64_t off = (uint64_t)((kk / 4) * (kTileRows * 128 / 16) + (kk % 4) * 2);
                        tc_mma_f16(tmem + place * 128, da + off, db + off, id_s, kk > 0);
                    }
                    tc_commit(bar(L::s_full, place));
                }
                __syncwarp();
            };
            auto values = [&](int place, int i, uint32_t st, uint32_t parity, bool add) {  // as the weights come: those of the first 64 tokens, and the others
                const uint64_t dv = make_smem_desc(base + L::stages + st * L::kStage, kTileTokens * 128, 1024);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    ok = warp_all(mbar_wait(bar(h ? L::p_full : L::p_half, place), parity, abort_flag, p.a.status, 78));
                    if (!ok) return;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 4 * h; kk < 4 * h + 4; kk++)
                            tc_mma_f16_a_tmem(tmem + 256 + i * 128, tmem + place * 128 + kk * 8, dv + (uint64_t)(kk * 128), id_o, add || kk > 0);
                    }
                    __syncwarp();
                }
            };
            if constexpr (kTiles == 1) {
                // scores are a tile ahead of the weights: S0 S1 | P0 V0 S2 | P1 V1 S3 ..
                auto next_scores = [&]() {
                    ok = warp_all(mbar_wait(bar(L::full, 0), n & 1u, abort_flag, p.a.status, 74));
                    if (!ok) return;
                    tc_fence_after();
                    scores(0, 0, (int)(n & 1u));
                    if (elect_one()) tc_commit(bar(L::empty, 0));
                    __syncwarp();
                    n++;
                };
                next_scores();
                if (ok && seg) ok = warp_all(mbar_wait(bar(L::o_empty), (seg - 1) & 1u, abort_flag, p.a.status, 75));  // the segment in front of this one has read its sums
                for (int j = 0; j < tiles && ok; j++) {
                    if (j + 1 < tiles) next_scores();
                    if (ok) ok = warp_all(mbar_wait(bar(L::full, 1), uses[0] & 1u, abort_flag, p.a.status, 76));
                    if (ok) values((int)(uses[0] & 1u), 0, 1, (uses[0] >> 1) & 1u, j > 0);
                    if (!ok) break;
                    uses[0]++;
                    if (elect_one()) {
                        tc_commit(bar(L::empty, 1));
                        tc_commit(bar(L::pv_done));
                        if (j + 1 == tiles) { tc_commit(bar(L::o_full)); tc_commit(bar(L::q_empty, qb)); }
                    }
                    __syncwarp();
                }
                if (!ok) break;
                seg++;
                continue;
            }
            // keys of the first tile
            uint32_t st = n % kStages;
            ok = warp_all(mbar_wait(bar(L::full, st), (n / kStages) & 1u, abort_flag, p.a.status, 74));
            if (!ok) break;
            tc_fence_after();
            for (int i = 0; i < both; i++) scores(i, st, i);
            if (elect_one()) tc_commit(bar(L::empty, st));
            __syncwarp();
            n++;
            if (seg) ok = warp_all(mbar_wait(bar(L::o_empty), (seg - 1) & 1u, abort_flag, p.a.status, 75));  // the segment in front of this one has read its sums
            for (int j = 0; j < tiles && ok; j++) {
                const uint32_t sv = n % kStages, sk = (n + 1) % kStages;
                ok = warp_all(mbar_wait(bar(L::full, sv), (n / kStages) & 1u, abort_flag, p.a.status, 76));
                if (ok && j + 1 < tiles) ok = warp_all(mbar_wait(bar(L::full, sk), ((n + 1) / kStages) & 1u, abort_flag, p.a.status, 77));
                for (int i = 0; i < both && ok; i++) {
                    values(i, i, sv, uses[i] & 1u, j > 0);
                    if (!ok) break;
                    uses[i]++;
                    if (j + 1 < tiles) scores(i, sk, i);
                }
                if (!ok) break;
                if (elect_one()) {
                    tc_commit(bar(L::empty, sv));
                    if (j + 1 < tiles) tc_commit(bar(L::empty, sk));
                    else { tc_commit(bar(L::o_full)); tc_commit(bar(L::q_empty, qb)); }
                }
                __syncwarp();
                n += j + 1 < tiles ? 2 : 1;
            }
            if (!ok) break;
            seg++;
        }
        if (!ok) {  // products on their way end before the block's memory becomes another's: a commit of its own behind them
            if (elect_one()) {
                tc_commit(bar(L::drain));
                wait_landed(bar(L::drain), 0);
            }
            __syncwarp();
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsRows));
      if (warp < 4 * kTiles) {
        const int i = warp >> 2, row = (warp & 3) * 32 + lane;  // tile, row
        const uint32_t t_warp = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_o = t_warp + 256 + i * 128;
        uint32_t uses = 0, tile = 0, turn = 0;  // scores of this row tile, tiles of tokens, tiles of tokens that both row tiles had
        SegmentInfo g;
        while (next_segment(g, 82)) {
            const bool works = i * kTileRows < g.n_rows, mine = i * kTileRows + row < g.n_rows;  // the tile, this row
            const int r = g.r0 + min(i * kTileRows + row, g.n_rows - 1), qi = r / p.a.group;
            SeqView v;
            v.first = g.first; v.n_q = g.n_q; v.len = g.len;
            float m = kNegInf, l = 0.f;
            bool far = false;  // a maximum that an FMA cannot take off exactly
            if (works) {
                const int hi = min(v.len, hi_of(p.a, v, qi)), lo = lo_of(p.a, v, qi);
                const float mul = p.q_mul[g.head * p.rows + (long long)g.first * p.a.group + r];
                int t0 = g.t0;
                for (int j = 0; j < g.tiles; j++, t0 += kTileTokens) {
                    const uint32_t mt = base + L::meta + ((tile + j) % kMetaRing) * 128;
                    const int place = kTiles == 2 ? i : (int)(uses & 1u);  // of the scores
                    const uint32_t t_s = t_warp + place * 128;
                    ok = warp_all(mbar_wait(bar(L::s_full, place), (kTiles == 2 ? uses : uses >> 1) & 1u, abort_flag, p.a.status, 79) &&
                                  mbar_wait(bar(L::meta_full, (tile + j) % kMetaRing), ((tile + j) / kMetaRing) & 1u, abort_flag, p.a.status, 83));
                    if (!ok) break;
                    uses++;
                    tc_fence_after();
                    uint32_t sr[128];
#pragma unroll
                    for (int c = 0; c < 4; c++) tmem_ld_x32(t_s + 32 * c, sr + 32 * c);
                    float f[8], minus_ev[8], weight[8];  // of 16 tokens: factor of a score, -e_v, 2^e_v
#pragma unroll
                    for (int x = 0; x < 8; x++) {
                        const float4 k = lds_f4(mt + 16 * x);
                        f[x] = score_factor(mul, k.z); minus_ev[x] = k.x; weight[x] = k.y;
                    }
                    tmem_ld_wait();
                    float least = minus_ev[0];
#pragma unroll
                    for (int x = 1; x < 8; x++) least = fminf(least, minus_ev[x]);
                    if (t0 < g.lo_max || t0 + kTileTokens > g.hi_min || least == kNegInf) {  // some row does not see some token (of no page: an infinite query makes NaN of its zeros)
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            const uint32_t there = (minus_ev[2 * c] == kNegInf ? 0u : 0xFFFFu) | (minus_ev[2 * c + 1] == kNegInf ? 0u : 0xFFFF0000u);
                            const int lo_c = max(0, min(32, lo - t0 - 32 * c)), hi_c = max(0, min(32, hi - t0 - 32 * c));
                            const uint32_t seen = there & (uint32_t)((1ull << hi_c) - 1ull) & ~(uint32_t)((1ull << lo_c) - 1ull);  // (a bit a column: one test each)
#pragma unroll
                            for (int y = 0; y < 32; y++)
                                if (!(seen & (1u << y))) sr[32 * c + y] = __float_as_uint(kNegInf);
                        }
                    }
                    float top = kNegInf;
#pragma unroll
                    for (int x = 0; x < 8; x++) {
                        auto a = [&](int y) { return __uint_as_float(sr[16 * x + y]); };
                        const float b0 = max3(a(0), a(1), a(2)), b1 = max3(a(3), a(4), a(5)), b2 = max3(a(6), a(7), a(8)), b3 = max3(a(9), a(10), a(11)), b4 = max3(a(12), a(13), a(14));
                        const float c = max3(max3(b0, b1, a(15)), max3(b2, b3, b4), kNegInf);
                        top = fmaxf(top, fmaf(c, f[x], minus_ev[x]));
                    }
                    const bool grows = top > m + kLazy || (m == kNegInf && top > kNegInf);
                    if (__any_sync(0xFFFFFFFFu, grows)) {
                        const float next = grows ? top : m, h = grows ? part_factor(m, next) : 1.f;
                        if (kTiles == 1 && j > 0) {  // (with two row tiles the scores' barrier says so)
                            ok = warp_all(mbar_wait(bar(L::pv_done), uses & 1u, abort_flag, p.a.status, 86));  // products with values of tile uses - 2 (uses counts this one)
                            if (!ok) break;
                            tc_fence_after();
                        }
                        if (j > 0) {
#pragma unroll 1
                            for (int c = 0; c < D / 16; c++) {
                                uint32_t o[16];
                                tmem_ld_x16(t_o + 16 * c, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int y = 0; y < 16; y++) o[y] = __float_as_uint(__uint_as_float(o[y]) * h);
                                tmem_st_x16(t_o + 16 * c, o);
                            }
                        }
                        l *= h;
                        m = next;
                        far = __any_sync(0xFFFFFFFFu, fabsf(m) > 131072.f && m != kNegInf);
                    }
                    const float base_m = m == kNegInf ? 0.f : m;
                    if (L::kTurns && g.n_rows > kTileRows) {
                        if (i || turn) ok = warp_all(mbar_wait(bar(L::turn, 4 * i + (warp & 3)), (i ? turn : turn - 1) & 1u, abort_flag, p.a.status, 87));
                        if (!ok) break;
                    }
                    if (far) {  // there -m + 4 - e would lose its last bits: the differences first
#pragma unroll
                        for (int x = 0; x < 8; x++) {
#pragma unroll
                            for (int y = 0; y < 16; y++) sr[16 * x + y] = __float_as_uint(fmaf(__uint_as_float(sr[16 * x + y]), f[x], minus_ev[x]) - base_m);
                            f[x] = 1.f; minus_ev[x] = base_m;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        uint32_t pr[16];
#pragma unroll
                        for (int x = 2 * c; x < 2 * c + 2; x++) {
                            const float add = minus_ev[x] - base_m + kShift;
                            const uint64_t f2 = pack2(f[x], f[x]), a2 = pack2(add, add);
                            uint64_t sum2 = 0;
#pragma unroll
                            for (int y = 0; y < 16; y += 2) {
                                float e0, e1;
                                unpack2(fma2(pack2(__uint_as_float(sr[16 * x + y]), __uint_as_float(sr[16 * x + y + 1])), f2, a2), e0, e1);
                                e0 = exp2_approx(e0);
                                e1 = exp2_approx(e1);
                                sum2 = y ? add2(sum2, pack2(e0, e1)) : pack2(e0, e1);
                                pr[8 * (x & 1) + y / 2] = pack_f16(e0, e1);
                            }
                            float u0, u1;
                            unpack2(sum2, u0, u1);
                            l = fmaf(u0 + u1, weight[x], l);
                        }
                        if (L::kTurns && c == 3 && g.n_rows > kTileRows) {
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar(L::turn, 4 * (1 - i) + (warp & 3)));
                            turn++;
                        }
                        if (c == 2) {  // the products with the first 64 tokens may start: their weights have landed while these were computed
                            tmem_st_wait();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar(L::p_half, place));
                        }
                        tmem_st_x16(t_s + 16 * c, pr);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(L::p_full, place));
                }
            }
            if (!ok) break;
            tile += g.tiles;
            ok = warp_all(mbar_wait(bar(L::o_full), seg & 1u, abort_flag, p.a.status, 80));
            if (!ok) break;
            tc_fence_after();
            if (works) {
                float* record = p.a.partial + (size_t)(2 * me + (g.from_start ? 1 : 0)) * Record<D>::floats;
                const int h = g.head * p.a.group + r - qi * p.a.group;
                const long long tok = g.first + qi;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                // (a part goes through shared memory, 32 elements of each of the warp's rows at a time: a store of its 32-bit values then takes 4 rows and not 32, and each line that it
                // touches is a cycle: 64 queries against 60000 tokens 162 -> 157 us; results gain nothing by it)
                const uint32_t stage = base + L::out + warp * 4096;
#pragma unroll 1
                for (int c = 0; c < D / 32; c++) {
                    uint32_t o[32];
                    tmem_ld_x32(t_o + 32 * c, o);
                    tmem_ld_wait();
                    if (!g.whole) {
#pragma unroll
                        for (int y = 0; y < 8; y++) sts_v4(stage + lane * 128 + ((y ^ (lane & 7)) << 4), make_uint4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]));
                        __syncwarp();
#pragma unroll
                        for (int y = 0; y < 8; y++) { const uint4 w = lds_v4(stage + (4 * y + (lane >> 3)) * 128 + (((lane & 7) ^ ((4 * y + (lane >> 3)) & 7)) << 4)); o[4 * y] = w.x; o[4 * y + 1] = w.y; o[4 * y + 2] = w.z; o[4 * y + 3] = w.w; }
#pragma unroll
                        for (int y = 0; y < 8; y++)
                            *reinterpret_cast<uint4*>(record + (size_t)(i * kTileRows + (warp & 3) * 32 + 4 * y + (lane >> 3)) * D + 32 * c + 4 * (lane & 7)) =
                                make_uint4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
                        __syncwarp();
                    } else if (mine) {
#pragma unroll
                        for (int y = 0; y < 32; y += 8) {
                            float x[8];
#pragma unroll
                            for (int z = 0; z < 8; z++) x[z] = __uint_as_float(o[y + z]) * inv;
                            store_out8<DT>(p.a, tok * p.a.out_token + (long long)h * p.a.out_head + 32 * c + y, x);
                        }
                    }
                }
                if (mine) {
                    if (!g.whole) *reinterpret_cast<float2*>(record + (size_t)Record<D>::kRows * D + 2 * (i * kTileRows + row)) = make_float2(m, l);
                    else if (p.a.lse) p.a.lse[tok * p.a.heads + h] = lse_of(m, l, kShift);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(L::o_empty));
            seg++;
        }
      }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Joins the unit that the boundary between blocks b - 1 and b cuts first; a block of threads takes 16 of its rows.
constexpr int kJoinRows = 16;
template <int D, int DT>
__global__ void __launch_bounds__(kThreads) cache_attention_join_kernel(const PrefillParams p)
{
    __shared__ int s_record[kMaxBlocks], s_parts;
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int b = (int)blockIdx.x + 1, lane = threadIdx.x & 31;
    if (b >= p.blocks) return;
    constexpr int kSteps = (kMaxBlocks + 31) / 32;
    long long from[kSteps], to[kSteps];  // (all loads at once)
#pragma unroll
    for (int k = 0; k < kSteps; k++) { from[k] = p.bound[min(b + 32 * k + lane, p.blocks)]; to[k] = p.bound[min(b + 32 * k + lane + 1, p.blocks)]; }
    const long long x = p.bound[b], all = p.bound[p.blocks], x_before = p.bound[b - 1];
    const int4 cut = p.cut[2 * b], of = p.cut[2 * b + 1];  // (of a block that begins behind all tiles: not looked at)
    if (x >= all) return;
    const long long begin = x - cut.x, end = begin + cut.y;
    if (cut.x == 0 || x_before > begin) return;
    const int head = cut.z, r0 = cut.w, first = of.x, n_rows = of.y;
    if ((int)blockIdx.y * kJoinRows >= n_rows) return;
    if (threadIdx.x < 32) {  // the blocks that have tiles of the unit: the one in front of the boundary, whose part is its last, and those behind it, whose parts are their first
        int n = 1;
        if (lane == 0) s_record[0] = 2 * (b - 1) + 1;
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
            const bool in = from[k] < end && to[k] > from[k];
            const uint32_t any = __ballot_sync(0xFFFFFFFFu, in);
            if (in) s_record[n + __popc(any & ((1u << lane) - 1u))] = 2 * (b + 32 * k + lane);
            n += __popc(any);
        }
        if (lane == 0) s_parts = n;
    }
    __syncthreads();
    const int parts = s_parts;
    for (int i = threadIdx.x; i < kJoinRows * (D / 4); i += kThreads) {
        const int row = (int)blockIdx.y * kJoinRows + i / (D / 4), d = i % (D / 4) * 4;
        if (row >= n_rows) continue;
        auto record = [&](int j) -> const float* { return p.a.partial + (size_t)s_record[j] * Record<D>::floats; };
        float top = kNegInf, den = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int j = 0; j < parts; j++) top = fmaxf(top, record(j)[(size_t)Record<D>::kRows * D + 2 * row]);
#pragma unroll 4
        for (int j = 0; j < parts; j++) {
            const float2 ml = *reinterpret_cast<const float2*>(record(j) + (size_t)Record<D>::kRows * D + 2 * row);
            const float4 a = *reinterpret_cast<const float4*>(record(j) + (size_t)row * D + d);
            const float h = part_factor(ml.x, top);
            den += ml.y * h;
            o[0] += a.x * h; o[1] += a.y * h; o[2] += a.z * h; o[3] += a.w * h;
        }
        const int r = r0 + row, qi = r / p.a.group, h = head * p.a.group + r - qi * p.a.group;
        const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
        for (int y = 0; y < 4; y++) o[y] *= inv;
        store_out4<DT>(p.a, (long long)(first + qi) * p.a.out_token + (long long)h * p.a.out_head + d, o);
        if (p.a.lse && d == 0) p.a.lse[(long long)(first + qi) * p.a.heads + h] = lse_of(top, den, kShift);
    }
}

// ---------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------
constexpr size_t kMostWorkspace = (size_t)16 << 30;  // beyond, the few-rows kernel takes the call

struct Sizes {
    int cap_blocks, pairs;
    size_t cut, bound, block_at, tiles_at, units_at, pair_seq, partial, meta, q_mul, kx, vx, qx, total;  // offsets
};
Sizes sizes_of(int n_seqs, int n_q, int max_length, int heads, int kv_heads, int dim)
{
    Sizes z;
    const int group = heads / kv_heads, unit_rows = dim == 256 ? TileShape<256>::kUnitRows : TileShape<128>::kUnitRows;
    const long long cap = (long long)n_seqs * (((long long)max_length + kTileTokens - 1) / kTileTokens + 1);
    z.cap_blocks = (int)(cap < 0x7FFFFFFF ? cap : 0x7FFFFFFF);  // (refused by its size long before)
    z.pairs = (int)((long long)n_q * group / unit_rows) + n_seqs;  // (n_q * group is below 2^30)
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round_up_256(bytes); return here; };
    z.cut = take((size_t)kMaxBlocks * 32);
    z.bound = take((size_t)(kMaxBlocks + 1) * 8);
    z.block_at = take((size_t)(n_seqs + 1) * 4);
    z.tiles_at = take((size_t)(z.pairs + 1) * 8);
    z.units_at = take((size_t)z.pairs * 4);
    z.pair_seq = take((size_t)z.pairs * 4);
    z.partial = take((size_t)2 * kMaxBlocks * unit_rows * (dim + 2) * 4);
    z.meta = take((size_t)kv_heads * z.cap_blocks * 8 * 16);
    z.q_mul = take((size_t)n_q * heads * 4);
    z.kx = take((size_t)kv_heads * z.cap_blocks * kTileTokens * dim * 2);
    z.vx = take((size_t)kv_heads * z.cap_blocks * kTileTokens * dim * 2);
    z.qx = take((size_t)n_q * heads * dim * 2);
    z.total = at;
    return z;
}

struct PrefillSetup { cudaError_t rc; };
PerDevice<PrefillSetup> g_prefill_setup;

bool fp16_map(CUtensorMap* map, const void* at, int dim, long long rows)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)dim, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)dim * 2};
    const cuuint32_t box[2] = {64, 128}, one[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(at), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int DT>
cudaError_t launch_of(const PrefillParams& p, int sms, cudaStream_t st)
{
    cudaError_t rc = launch_pdl_threads(kPlanThreads, cache_plan_kernel, dim3(1), st, p);
    if (rc != cudaSuccess) return rc;
    const long long units = 2ll * p.cap_blocks * p.a.c.heads + ((long long)p.a.n_q * p.a.heads * D + 8191) / 8192, most = 6ll * sms;  // (six blocks fit on an SM)
    rc = launch_pdl(cache_expand_kernel<D, DT>, dim3((unsigned)(units < most ? units : most)), st, p);
    if (rc != cudaSuccess) return rc;
    CUtensorMap mq, mk, mv;
    const long long kv_rows = (long long)p.a.c.heads * p.cap_blocks * kTileTokens;
    if (!fp16_map(&mq, p.qx, D, p.rows * p.a.c.heads) || !fp16_map(&mk, p.kx, D, kv_rows) || !fp16_map(&mv, p.vx, D, kv_rows)) return cudaErrorInvalidValue;
    const int blocks = p.blocks;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreadsA);
    cfg.dynamicSmemBytes = PrefillSmem<D>::kBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    rc = cudaLaunchKernelEx(&cfg, cache_attention_tiles_kernel<D, DT>, mq, mk, mv, p);
    if (rc != cudaSuccess) return rc;
    rc = launch_pdl(cache_attention_join_kernel<D, DT>, dim3((unsigned)(blocks > 1 ? blocks - 1 : 1), TileShape<D>::kUnitRows / kJoinRows), st, p);
    g_launches.fetch_add(4, std::memory_order_relaxed);
    return rc;
}

}  // namespace

// From 64 rows of a key head on.  us, few-rows kernel / this, with 48, 64 and 96 rows (four heads to a key head, 8 key heads):
//   heads of 128: 16 sequences of up to 2000 tokens 62 / 65, 76 / 65, 104 / 66; 4 of up to 16000 95 / 110, 120 / 111, 165 / 111; one of 8000 40.8 / 41.9, 41.7 / 42.3, 51.5 / 42.2
//   heads of 64:  16 of up to 2000 41.8 / 48.3, 49.4 / 48.1, 66 / 49; 4 of up to 16000 62 / 82, 76 / 82, 102 / 81; one of 1000 16.8 / 20.5, 17.7 / 20.9, 19.6 / 21.0
//   heads of 256: 16 of up to 2000 137 / 99, 177 / 100, 256 / 103; one of 1000 27 / 31, 29 / 31, 33 / 32
// (Few and long sequences of heads of 64 lose a little at 64 rows, and heads of 256 would gain from fewer rows on.)
size_t prefill_workspace_bytes(int n_seqs, int n_q, int max_q, int max_length, int heads, int kv_heads, int dim)
{
    if ((long long)max_q * (heads / kv_heads) < 64) return 0;
    const Sizes z = sizes_of(n_seqs, n_q, max_length, heads, kv_heads, dim);
    // (rows of a tensor map; and no call is asked for more memory than a good part of a device's: the few-rows kernel then takes it)
    if ((long long)kv_heads * z.cap_blocks * kTileTokens > 0x7FFFFFFF || (long long)n_q * heads > 0x7FFFFFFF || z.total > kMostWorkspace) return 0;
    return z.total;
}

cudaError_t launch_prefill(AttentionParams a, int dtype, int max_length, uint8_t* ws, int sms, cudaStream_t st)
{
    int dev = 0;
    cudaError_t rc = cudaGetDevice(&dev);
    if (rc != cudaSuccess) return rc;
    const PrefillSetup* setup = g_prefill_setup.get(dev, [](int, PrefillSetup* o) {
        const void* k[6] = {(const void*)cache_attention_tiles_kernel<64, HIF8_BF16>, (const void*)cache_attention_tiles_kernel<64, HIF8_F16>,
                            (const void*)cache_attention_tiles_kernel<128, HIF8_BF16>, (const void*)cache_attention_tiles_kernel<128, HIF8_F16>,
                            (const void*)cache_attention_tiles_kernel<256, HIF8_BF16>, (const void*)cache_attention_tiles_kernel<256, HIF8_F16>};
        const int bytes[6] = {(int)PrefillSmem<64>::kBytes, (int)PrefillSmem<64>::kBytes, (int)PrefillSmem<128>::kBytes, (int)PrefillSmem<128>::kBytes, (int)PrefillSmem<256>::kBytes,
                              (int)PrefillSmem<256>::kBytes};
        o->rc = cudaSuccess;
        for (int i = 0; i < 6 && o->rc == cudaSuccess; i++) o->rc = cudaFuncSetAttribute(k[i], cudaFuncAttributeMaxDynamicSharedMemorySize, bytes[i]);
    });
    if (!setup || setup->rc != cudaSuccess) return cudaErrorInvalidValue;
    PrefillParams p;
    p.a = a;
    const Sizes z = sizes_of(a.n_seqs, a.n_q, max_length, a.heads, a.c.heads, a.c.dim);
    p.specials = a.special_flag;
    p.cut = reinterpret_cast<int4*>(ws + z.cut);
    p.block_at = reinterpret_cast<int*>(ws + z.block_at);
    p.tiles_at = reinterpret_cast<long long*>(ws + z.tiles_at);
    p.pair_seq = reinterpret_cast<int*>(ws + z.pair_seq);
    p.units_at = reinterpret_cast<int*>(ws + z.units_at);
    p.bound = reinterpret_cast<long long*>(ws + z.bound);
    p.a.partial = reinterpret_cast<float*>(ws + z.partial);
    p.meta = reinterpret_cast<float4*>(ws + z.meta);
    p.q_mul = reinterpret_cast<float*>(ws + z.q_mul);
    p.kx = reinterpret_cast<__half*>(ws + z.kx);
    p.vx = reinterpret_cast<__half*>(ws + z.vx);
    p.qx = reinterpret_cast<__half*>(ws + z.qx);
    p.cap_blocks = z.cap_blocks;
    p.pairs = z.pairs;
    p.blocks = sms < kMaxBlocks ? sms : kMaxBlocks;
    p.rows = (long long)a.n_q * a.group;
    p.unit_rows = a.c.dim == 256 ? TileShape<256>::kUnitRows : TileShape<128>::kUnitRows;
    if (a.c.dim == 64) return dtype == HIF8_BF16 ? launch_of<64, HIF8_BF16>(p, sms, st) : launch_of<64, HIF8_F16>(p, sms, st);
    if (a.c.dim == 128) return dtype == HIF8_BF16 ? launch_of<128, HIF8_BF16>(p, sms, st) : launch_of<128, HIF8_F16>(p, sms, st);
    return dtype == HIF8_BF16 ? launch_of<256, HIF8_BF16>(p, sms, st) : launch_of<256, HIF8_F16>(p, sms, st);
}

}  // namespace hif8
