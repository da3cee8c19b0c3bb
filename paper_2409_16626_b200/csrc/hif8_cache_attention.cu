// Attention over the HiF8 key/value cache.
//
//   s_ij = scale * sum_d q_i[d] k_j[d],   out_i = sum_j softmax_j(s_i) v_j,   lse_i = ln sum_j exp(s_ij)
//
// over the cached tokens j that query i may look at.  A code's value has at most 4 significant bits and an exponent in [-22, 15], so it is exact
// in FP16 (the smallest ones as FP16 subnormals), and codes are multiplied as they are: the block exponents of K go into the factor of a score and
// those of V into the softmax.  With x_ij = s_ij / ln 2 - e_v(j), e_v(j) the exponent of the block that v_j lies in, and m_i = max_j x_ij,
//   P_ij = 2^(x_ij - m_i + 8),   out_i = sum_j P_ij code_v(j) / sum_j P_ij 2^(e_v(j)),
// so P <= 2^8 whatever the blocks' spreads are (2^14 while m_i is a maximum of earlier tokens), and nothing is rounded but P (to FP16, 11 bits; products and
// sums are FP32).  The 2^8 keeps P in the normal range of FP16 down to 2^-22 of the largest.  Exponents lie within +-48, so the denominator stays far inside FP32.
//
// Few query rows of a key head are in this file, chunks of prompts in hif8_cache_prefill.cu.
#include "hif8_cache_attention.cuh"

namespace hif8 {
namespace {

constexpr float kPShift = 8.f, kPLimit = 14.f;  // weights are 2^(x - m + 8) with m an earlier maximum, up to 2^14 of FP16's 2^16

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
// ---------------------------------------------------------------------------------------------------------
// Few query rows (decoding, drafted tokens): bound by reading the cache once.
//
// A warp multiplies 16 tokens at a time on mma.sync with the tokens as the 16 rows of the A operand and up to 8 NT query rows as columns: S^T = K Q^T,
// O^T += V^T P^T.  Bytes come through a ring of TMA copies of the warp's own, and from there through the lookup into the operands: a table of the 256 FP16
// values with a copy for every lane takes a byte permute and a conflict-free lookup a code.  The tensor-memory path would write every decoded value to
// shared memory and read it again, and shared-memory traffic is what comes next after DRAM here.  (Loads straight into registers, a tile ahead, did not
// cover the latency: 8 sequences of up to 131072 tokens, 64/8 heads of 128: 480 us, 400 of them without any lookup.)
// Measured (us, of the measured copy bandwidth): those sequences 311 (4.8 TB/s, 73 %), 64 of up to 4096 tokens, 32/8 heads 74 (4.0 TB/s, 60 %; heads of 64 57, of 256 145).  Of a tile's 220 cycles an SM the
// shared-memory pipe is busy 165 (128 lookups and 32 wavefronts of bytes); 430 instructions a tile and warp leave the schedulers busy 62 % of the time.
// Which of the 16 tokens or the elements meet in a product is the operands' own business as long as both agree: a thread's bytes are read 16 at a time, and
// tokens and pieces are dealt to the threads so that the reads of a swizzled tile never meet in a bank (see token_of_row, piece_of).
//
// Chunks of 64 tokens of a (sequence, key head, row tile) are dealt out evenly: group g of four warps takes the chunks [T g / G, T (g + 1) / G) of all
// T, in order.  A unit whose chunks lie in several groups leaves partial sums in the workspace, which a second kernel adds in a fixed order.
// WIDE: short units are not cut: all warps of a block are one group, which takes whole units, and there is no second kernel (see whole_units).
// ---------------------------------------------------------------------------------------------------------
constexpr uint32_t kLutBytes = 65536;  // rows of 256 bytes on a 64 KiB boundary: the address is one byte permute away from the code

// groups of a block: what registers and shared memory leave room for (128 elements, NT = 1: three groups of 168 registers a thread 351 us where four take 341)
constexpr int groups_of(int dim, int nt) { return dim == 256 ? 2 : dim == 128 && nt == 2 ? 3 : 4; }

// Shared memory: [prefix sums, maxima and denominators, barriers, rings] table [rings].  The table lies on a 64 KiB boundary; a block's memory begins
// 1 KiB behind one.  The upper halves of the table's rows hold the warps' sums while a segment's are joined, a few query rows at a time: the rings
// go on with the next segment's tiles meanwhile.
template <int D, int NT, bool WIDE>
struct RowsShape {
    static constexpr int kWarps = 4 * groups_of(D, NT), kThreads = kWarps * 32, kGroupWarps = WIDE ? kWarps : 4, kGroups = kWarps / kGroupWarps, kChunk = 16 * kGroupWarps;
    static constexpr int kRows = 8 * NT;
    static constexpr int kStages = D == 64 ? 4 : 2;
    static constexpr uint32_t kTile = 16 * D;                            // bytes of 16 tokens of K or V
    static constexpr uint32_t kRing = kStages * 2 * kTile;               // of a warp
    static constexpr int kBackWarps = 98304 / kRing, kFrontWarps = kWarps > kBackWarps ? kWarps - kBackWarps : 0;  // rings behind / in front of the table
    static constexpr int kGapRows = 256 / kWarps, kJoinRows = D == 64 ? 8 : 4;  // rows of the table whose upper halves are a warp's; query rows that fit there
    static constexpr int kRecord = kRows * (D + 2);                      // floats of a partial result: sums, maxima, denominators
    // offsets from the block's first byte, which is 1024 modulo 65536
    static constexpr uint32_t kMl = (HIF8_CACHE_MAX_SEQS + 2) * 8, kScan = kMl + kWarps * kRows * 8, kBars = kScan + 32 * 8, kFlag = kBars + kWarps * kStages * 8,
                              kMul = (kFlag + 16 + 15) / 16 * 16, kQuery = (kMul + kGroups * kRows * 4 + 15) / 16 * 16,
                              kQueryBytes = kRows * D * 2;
    static constexpr uint32_t kFrontRing = kLutBytes - 1024 - kFrontWarps * kRing, kLut = kLutBytes - 1024, kBackRing = kLut + kLutBytes;
    static constexpr uint32_t kSmem = kBackRing + (kWarps < kBackWarps ? kWarps : kBackWarps) * kRing;
    static_assert(kQuery + kGroups * kQueryBytes <= kFrontRing && kSmem <= 227 * 1024 && kJoinRows * D * 4 <= kGapRows * 128, "shared memory");
    __device__ static uint32_t ring(uint32_t raw, int w) { return raw + (w < kBackWarps ? kBackRing + w * kRing : kFrontRing + (w - kBackWarps) * kRing); }
    // offset of float4 number f of query row `row` (of the kJoinRows) in warp w's sums: neither writing them from the products' layout nor reading rows meets in a bank
    __device__ static uint32_t sum_at(int w, int row, int f)
    {
        const int i = row * (D / 4) + (f ^ ((row >> 1) & 3) ^ (((f >> (D == 64 ? 1 : 4)) & 1) << 2));
        return kLut + (uint32_t)(w * kGapRows + (i >> 3)) * 256 + 128 + (uint32_t)(i & 7) * 16;
    }
};

// token (of a tile's 16) in row r of the A operand: with rows 2 t and 2 t + 1 the tokens that thread t of a column of threads reads V of
template <int D> __device__ __forceinline__ int token_of_row(int r)
{
    const int x = (r & 7) >> 1;
    return D == 64 ? (x & 1) + 4 * (x >> 1) + 2 * (r & 1) + (r & 8) : x + 4 * (r & 1) + (r & 8);
}
// piece of a value row (16 bytes, 8 for D = 64) that the threads of operand row g take
template <int D> __device__ __forceinline__ int piece_of(int g) { return D == 64 ? g : (g >> 1) | (g & 1) << 2; }
// byte offset of a 16-byte chunk of a token in a swizzled tile (rows of 128 bytes; of 64 for D = 64; halves of 128 bytes one behind the other for D = 256)
template <int D> __device__ __forceinline__ uint32_t chunk_at(int token, int chunk)
{
    if (D == 64) return (uint32_t)(token * 64 + ((chunk ^ ((token >> 1) & 3)) << 4));
    return (uint32_t)((chunk >> 3) * 2048 + token * 128 + (((chunk & 7) ^ (token & 7)) << 4));
}
__device__ __forceinline__ void group_sync(int group, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory"); }
// ... and whether `any` holds in one of the group's threads
__device__ __forceinline__ bool group_any(int group, int threads, bool any)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbarrier.cta.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(group + 1), "r"(threads), "r"((uint32_t)any) : "memory");
    return r != 0;
}

// Inf and NaN among the values that a query sees reach its result whatever their weights are.  Products with Inf tell that one is there, and which where the weights are not zero; a weight
// that is (below FP16's range, or of a score of -Inf) makes NaN of it.  So where a result is NaN and its denominator is not, the column is read again: four elements of query `tok` of the
// batch, from d on, x what the products gave.  NaN, or Inf of both signs, ends the search.  (In a function of its own: there is hardly ever anything to do.  8 sequences of 131072 tokens whose
// values are all Inf, most weights 0: 33 ms instead of 0.4; all NaN: 0.43.)
__device__ __noinline__ float4 seen_specials(const AttentionParams& p, int tok, int head, int d, float4 x)
{
    const uint32_t need = (x.x != x.x ? 0xFFu : 0u) | (x.y != x.y ? 0xFF00u : 0u) | (x.z != x.z ? 0xFF0000u : 0u) | (x.w != x.w ? 0xFF000000u : 0u);
    int s = 0;
    for (int n = p.n_seqs; n > 1;) {  // the last sequence that starts at or before the query
        const int half = n >> 1;
        if (start_at(p.q_start, s + half, p.n_q) <= tok) { s += half; n -= half; }
        else n = half;
    }
    const SeqView v = seq_view(p, s);
    const int lo = lo_of(p, v, tok - v.first), hi = min(v.len, hi_of(p, v, tok - v.first)), mask = (1 << p.c.shift) - 1;
    uint32_t inf = 0u, minus = 0u, nan = 0u;
    for (int t = lo; t < hi && need & ~(nan | (inf & minus));) {
        const int page = p.c.page_of(s, t >> p.c.shift), n = min(hi - t, mask + 1 - (t & mask));
        if (page >= 0) {
            const uint8_t* at = p.c.v + p.c.block_at(page, head) + (long long)(t & mask) * p.c.dim + d;
#pragma unroll 8
            for (int i = 0; i < n; i++) {
                const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(at + i * p.c.dim));
                inf |= __vcmpeq4(w, 0x6F6F6F6Fu); minus |= __vcmpeq4(w, 0xEFEFEFEFu); nan |= __vcmpeq4(w, 0x80808080u);
            }
        }
        t += n;
    }
    nan |= inf & minus;
    auto result = [&](float y, int shift) -> float {
        if (!(need >> shift & 1u) || nan >> shift & 1u) return y;
        return inf >> shift & 1u ? -kNegInf : minus >> shift & 1u ? kNegInf : y;
    };
    return make_float4(result(x.x, 0), result(x.y, 8), result(x.z, 16), result(x.w, 24));
}
__device__ __forceinline__ void resolve_specials(const AttentionParams& p, int tok, int head, int d, float den, float (&x)[4])
{
    const float any = (x[0] + x[1]) + (x[2] + x[3]);
    if (any != any && den == den) {
        const float4 y = seen_specials(p, tok, head, d, make_float4(x[0], x[1], x[2], x[3]));
        x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
    }
}

// The work of one sequence in chunks
struct SeqChunks {
    int lo, per_unit, tiles;  // first token (on a chunk), chunks of a unit, row tiles
    __device__ SeqChunks(const AttentionParams& p, const SeqView& v, int rows, int chunk)
    {
        lo = v.n_q ? lo_of(p, v, 0) / chunk * chunk : 0;
        per_unit = max(1, (v.len - lo + chunk - 1) / chunk);
        tiles = (int)(((long long)v.n_q * p.group + rows - 1) / rows);
    }
};

template <int D, int NT, int DT, bool WIDE>
__global__ void __launch_bounds__(RowsShape<D, NT, WIDE>::kThreads, 1)
cache_attention_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttentionParams p)
{
    using S = RowsShape<D, NT, WIDE>;
    constexpr int GW = S::kGroupWarps, kChunk = S::kChunk;
    constexpr int J = D / 64;                       // blocks of 64 elements of a key
    constexpr int VB = D / 8;                       // bytes of a value row that a thread takes
    constexpr int MT = D / 16;                      // m16 tiles of the output
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    long long* s_prefix = reinterpret_cast<long long*>(smem_raw);
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int grp = warp / GW, gw = warp % GW;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + S::kFlag);
    if ((raw & (kLutBytes - 1)) != 1024) {  // (the same answer in every thread of the grid)
        pdl_wait_prior_grid();
        if (blockIdx.x == 0 && threadIdx.x == 0) { *p.status = 7; *p.chunks = 0; }
        return;
    }
    {
        uint32_t* lut_words = reinterpret_cast<uint32_t*>(smem_raw + S::kLut);
        for (int i = threadIdx.x; i < 256 * 8; i += S::kThreads) {
            const uint32_t v = g_f16_of_code.v[i >> 3];
            *reinterpret_cast<uint4*>(lut_words + (i >> 3) * 64 + (i & 7) * 4) = make_uint4(v, v, v, v);
        }
    }
    const uint32_t bars = raw + S::kBars + warp * S::kStages * 8;
    if (lane == 0) {
        for (int x = 0; x < S::kStages; x++) mbar_init(bars + 8 * x, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) *abort_flag = 0;
    pdl_wait_prior_grid();
    pdl_launch_dependents();

    // chunks in front of each sequence: every thread takes consecutive sequences
    {
        long long* s_warp = reinterpret_cast<long long*>(smem_raw + S::kScan);
        const int each = (p.n_seqs + S::kThreads - 1) / S::kThreads, s0 = min(p.n_seqs, (int)threadIdx.x * each), s1 = min(p.n_seqs, s0 + each);
        long long mine = 0;
        for (int s = s0; s < s1; s++) {
            const SeqView v = seq_view(p, s);
            const SeqChunks k(p, v, S::kRows, kChunk);
            s_prefix[s] = mine;
            mine += (long long)k.tiles * p.c.heads * (WIDE ? 1 : k.per_unit);
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
        if (blockIdx.x == 0 && threadIdx.x == 0) { *p.chunks = s_prefix[p.n_seqs]; *p.status = 0; }
    }
    const long long chunks = s_prefix[p.n_seqs];
    const int groups = (int)min((long long)gridDim.x * S::kGroups, chunks);
    const int me = (int)blockIdx.x + grp * (int)gridDim.x;  // (few chunks: a group on every SM before a second one)
    if (me >= groups) return;
    long long x0 = share_of(chunks, me, groups);
    const long long x_end = share_of(chunks, me + 1, groups);
    const uint32_t lut = raw + S::kLut + 4u * lane;
    const uint32_t ring = S::ring(raw, warp);
    float2* all_ml = reinterpret_cast<float2*>(smem_raw + S::kMl) + grp * GW * S::kRows;
    const int slot_mask = (1 << p.c.shift) - 1;
    // where this thread reads its bytes of a tile: keys of operand rows g and g + 8, the 16-byte chunks t, t + 4, ..; values of four tokens
    const int tok_k = token_of_row<D>(g), piece = piece_of<D>(g);
    uint32_t use = 0;  // uses of the ring by this warp: stage use % kStages, parity (use / kStages) & 1
    bool ok = true;
    const uint32_t magic = 65536u / (uint32_t)p.group + 1u;  // x / group = x magic >> 16 for the x < group + 16 that come up

    // ---- a segment: chunks c0 .. c1 of a unit.  The first one is looked for; the others begin at the next unit, which takes no search and hardly a division.  (Looked
    // for by every warp, a segment took as many instructions as 18 tiles.)
    struct Segment {
        SeqView v;
        int s, head, r0, n_rows, q0, h0, c0, c1, per_unit, lo_chunk, hi_min, hi_max, lo_min, lo_max;  // q0, h0: query and head of the first row
    };
    Segment e0{};
    long long left = x_end - x0;  // chunks (units: WIDE) of this group from the segment's first on
    auto enter = [&]() {          // e0.s: its tokens
        e0.v = seq_view(p, e0.s);
        const SeqChunks k(p, e0.v, S::kRows, kChunk);
        e0.per_unit = k.per_unit; e0.lo_chunk = k.lo;
    };
    auto limits = [&]() {
        e0.c1 = WIDE ? e0.per_unit : (int)min((long long)e0.per_unit, e0.c0 + left);
        e0.n_rows = min(S::kRows, e0.v.n_q * p.group - e0.r0);
        e0.q0 = e0.r0 ? e0.r0 / p.group : 0; e0.h0 = e0.r0 - e0.q0 * p.group;
        const int qb = e0.q0 + (int)((uint32_t)(e0.h0 + e0.n_rows - 1) * magic >> 16);
        e0.hi_min = min(e0.v.len, hi_of(p, e0.v, e0.q0)); e0.hi_max = min(e0.v.len, hi_of(p, e0.v, qb)); e0.lo_min = lo_of(p, e0.v, e0.q0); e0.lo_max = lo_of(p, e0.v, qb);
    };
    auto locate = [&]() {
        e0.s = 0;
        for (int n = p.n_seqs; n > 1;) {  // last sequence that starts at or before x0 (those without chunks share their start with the next)
            const int half = n >> 1;
            if (s_prefix[e0.s + half] <= x0) { e0.s += half; n -= half; }
            else n = half;
        }
        enter();
        const long long in_seq = x0 - s_prefix[e0.s], unit = WIDE ? in_seq : div_small(in_seq, e0.per_unit);
        const int tiles = (int)(((long long)e0.v.n_q * p.group + S::kRows - 1) / S::kRows);
        e0.c0 = WIDE ? 0 : (int)(in_seq - unit * e0.per_unit);
        e0.head = (int)div_small(unit, tiles); e0.r0 = (int)(unit - (long long)e0.head * tiles) * S::kRows;
        limits();
    };
    auto advance = [&]() -> bool {  // to the next segment; false: there is none
        left -= WIDE ? 1 : e0.c1 - e0.c0;
        if (left <= 0) return false;
        e0.r0 += S::kRows;
        if (e0.r0 >= e0.v.n_q * p.group) {
            e0.r0 = 0;
            if (++e0.head == p.c.heads) {
                e0.head = 0;
                do { e0.s++; enter(); } while (e0.v.n_q == 0 && e0.s + 1 < p.n_seqs);
            }
        }
        e0.c0 = 0;
        limits();
        return true;
    };
    auto step_of = [&](int h0, int row) -> int { return (int)((uint32_t)(h0 + row) * magic >> 16); };  // queries from the first row's to row `row`'s

    // ---- the copies: tiles of this warp, kStages ahead of the products.  Lane n holds pool row and exponents of the warp's tile in the n-th chunk of a batch of 32;
    // a tile without a page, or with no token that a row sees, is left out.  `ahead` holds first tokens and exponents of those on their way.
    int b_row = -1, b_exps = 0, b_first = 0;
    uint32_t b_live = 0;
    int ahead_t0[S::kStages], ahead_exps[S::kStages];
    auto load_batch = [&](int c) {
        b_first = c;
        const int at = e0.lo_chunk + (c + lane) * kChunk + 16 * gw;  // (below 2^31: a length, at most 2^30, and less than 2^14 more)
        const int page = c + lane < e0.c1 && at < e0.hi_max && at + 16 > e0.lo_min ? p.c.page_of(e0.s, at >> p.c.shift) : -1;
        const long long e = (long long)max(page, 0) * p.c.heads + e0.head;
        b_exps = page >= 0 ? (clamp_cache_exp(p.c.k_exp[e]) & 0xFF) | clamp_cache_exp(p.c.v_exp[e]) << 8 : 0;
        b_row = (int)(e << p.c.shift) + (at & slot_mask);  // (rows of a pool number less than 2^31)
        b_live = __ballot_sync(0xFFFFFFFFu, page >= 0);
    };
    auto ask = [&](uint32_t n, int& t0, int& exps) {  // the next tile into the place of use n; t0 = -1: there is none
        while (!b_live && b_first + 32 < e0.c1) load_batch(b_first + 32);
        t0 = -1;
        if (!b_live || !ok) return;
        const int i = __ffs(b_live) - 1, row = __shfl_sync(0xFFFFFFFFu, b_row, i);
        t0 = e0.lo_chunk + (b_first + i) * kChunk + 16 * gw;
        b_live &= b_live - 1;
        const uint32_t st = n % S::kStages, at = ring + st * 2 * S::kTile, bar = bars + 8 * st;
        __syncwarp();  // every lane has read what the stage held
        if (elect_one()) {
            mbar_expect(bar, 2 * S::kTile);
            tma_load_2d(at, &map_k, 0, row, bar);
            if (D == 256) tma_load_2d(at + 2048, &map_k, 128, row, bar);
            tma_load_2d(at + S::kTile, &map_v, 0, row, bar);
            if (D == 256) tma_load_2d(at + S::kTile + 2048, &map_v, 128, row, bar);
        }
        __syncwarp();
        exps = __shfl_sync(0xFFFFFFFFu, b_exps, i);  // (behind the copies, which need not wait for them)
    };
    // ---- the queries of a segment: the group's warps load (behind the first tiles) and convert a share of the rows each, D / 8 lanes to a row
    constexpr int kRowLanes = D / 8, kRowsStep = GW * 32 / kRowLanes, kSteps = (S::kRows + kRowsStep - 1) / kRowsStep;
    unsigned char* queries = smem_raw + S::kQuery + grp * S::kQueryBytes;
    float* muls = reinterpret_cast<float*>(smem_raw + S::kMul) + grp * S::kRows;
    uint4 q_raw[kSteps];
    const int q_row = (gw * 32 + lane) / kRowLanes, q_piece = lane % kRowLanes;  // first row, eight elements of it
    auto begin = [&]() {
        load_batch(e0.c0);
#pragma unroll
        for (int x = 0; x < S::kStages; x++) ask(use + x, ahead_t0[x], ahead_exps[x]);
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int row = q_row + i * kRowsStep;
            q_raw[i] = make_uint4(0, 0, 0, 0);
            if (row < e0.n_rows) {
                const int step = step_of(e0.h0, row);
                const unsigned short* src = reinterpret_cast<const unsigned short*>(p.q) + (long long)(e0.v.first + e0.q0 + step) * p.q_token +
                                            (long long)(e0.head * p.group + e0.h0 + row - step * p.group) * p.q_head + 8 * q_piece;
                if (p.vectors) q_raw[i] = __ldg(reinterpret_cast<const uint4*>(src));
                else q_raw[i] = make_uint4((uint32_t)src[0] | (uint32_t)src[1] << 16, (uint32_t)src[2] | (uint32_t)src[3] << 16, (uint32_t)src[4] | (uint32_t)src[5] << 16, (uint32_t)src[6] | (uint32_t)src[7] << 16);
            }
        }
    };
    auto convert_queries = [&]() {
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int row = q_row + i * kRowsStep;
            int e = 0;
            if (DT == HIF8_BF16) {  // FP16 queries are multiplied as they are
                float a = amax_value<DT>(amax_vector<DT>(0u, q_raw[i]));
#pragma unroll
                for (int d = 1; d < kRowLanes; d *= 2) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, d));
                e = query_exp(a);
                const float f = pow2f(e);
                auto both = [&](uint32_t w) { return pack_f16(q_value<DT>(w & 0xFFFFu) * f, q_value<DT>(w >> 16) * f); };
                q_raw[i] = make_uint4(both(q_raw[i].x), both(q_raw[i].y), both(q_raw[i].z), both(q_raw[i].w));
            }
            if (row < S::kRows) {
                *reinterpret_cast<uint4*>(queries + row * D * 2 + 16 * q_piece) = q_raw[i];
                if (q_piece == 0) muls[row] = query_factor(p.scale_log2, e);
            }
        }
    };
    locate();
    begin();
    convert_queries();
    group_sync(grp, GW * 32);
    // (what the joining kernel has to know of the unit that this group's first chunk lies in)
    if (!WIDE && gw == 0 && lane == 0) {
        int4* cut = p.cut + 2 * me;
        cut[0] = make_int4(e0.head, e0.r0, e0.c0, e0.per_unit);
        cut[1] = make_int4(e0.v.first, e0.n_rows, 0, 0);
    }

    while (true) {
        const SeqView v = e0.v;
        const int n_rows = e0.n_rows, hi_min = e0.hi_min, hi_max = e0.hi_max, lo_min = e0.lo_min, lo_max = e0.lo_max;
        auto query_of = [&](int row) -> int { return e0.q0 + step_of(e0.h0, row); };

        // queries: column g of n8 tile i is row r0 + 8 i + g; a thread takes the elements 64 j + 16 t .. + 15
        uint32_t qb[NT][J][4][2];
        float row_mul[NT][2];
#pragma unroll
        for (int i = 0; i < NT; i++) {
#pragma unroll
            for (int j = 0; j < J; j++) {
                const uint4* from = reinterpret_cast<const uint4*>(queries + (8 * i + g) * D * 2 + 128 * j + 32 * t);
                const uint4 a = from[0], b = from[1];
                qb[i][j][0][0] = a.x; qb[i][j][0][1] = a.y; qb[i][j][1][0] = a.z; qb[i][j][1][1] = a.w;
                qb[i][j][2][0] = b.x; qb[i][j][2][1] = b.y; qb[i][j][3][0] = b.z; qb[i][j][3][1] = b.w;
            }
#pragma unroll
            for (int b = 0; b < 2; b++) row_mul[i][b] = muls[8 * i + 2 * t + b];  // the scores' columns of this thread: rows 2 t and 2 t + 1 of the tile
        }

        // base: the maximum that the weights refer to, 0 before there is one; limit: what an argument may be without a new one; far: a base that an FMA cannot take
        float m[NT][2], l[NT][2], base[NT][2], limit[NT][2], o[NT][MT][4];
        bool far = false;
#pragma unroll
        for (int i = 0; i < NT; i++) {
            m[i][0] = m[i][1] = kNegInf;
            l[i][0] = l[i][1] = base[i][0] = base[i][1] = 0.f;
            limit[i][0] = limit[i][1] = kNegInf;
#pragma unroll
            for (int x = 0; x < MT; x++)
#pragma unroll
                for (int y = 0; y < 4; y++) o[i][x][y] = 0.f;
        }

        while (ahead_t0[0] >= 0) {
            const int t0 = ahead_t0[0], exps = ahead_exps[0];
            const uint32_t st = use % S::kStages, parity = (use / S::kStages) & 1u, at_k = ring + st * 2 * S::kTile, at_v = at_k + S::kTile, bar = bars + 8 * st;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag, p.status, 61));
            if (!ok) break;
            // scores, transposed: operand row g (+ 8) x rows 2 t, 2 t + 1.  (Two sums, so that a product does not wait for the one in front of it.)
            float sc[NT][4], sd[NT][4];
#pragma unroll
            for (int i = 0; i < NT; i++) {
                sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
                sd[i][0] = sd[i][1] = sd[i][2] = sd[i][3] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < J; j++) {
                const uint4 ka = lds_v4(at_k + chunk_at<D>(tok_k, 4 * j + t)), kb = lds_v4(at_k + chunk_at<D>(tok_k + 8, 4 * j + t));
                const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const uint32_t a0 = __byte_perm(lds_u32(__byte_perm(wa[q], lut, 0x7604)), lds_u32(__byte_perm(wa[q], lut, 0x7614)), 0x5410);
                    const uint32_t a2 = __byte_perm(lds_u32(__byte_perm(wa[q], lut, 0x7624)), lds_u32(__byte_perm(wa[q], lut, 0x7634)), 0x5410);
                    const uint32_t a1 = __byte_perm(lds_u32(__byte_perm(wb[q], lut, 0x7604)), lds_u32(__byte_perm(wb[q], lut, 0x7614)), 0x5410);
                    const uint32_t a3 = __byte_perm(lds_u32(__byte_perm(wb[q], lut, 0x7624)), lds_u32(__byte_perm(wb[q], lut, 0x7634)), 0x5410);
#pragma unroll
                    for (int i = 0; i < NT; i++) mma_16816_f16(q & 1 ? sd[i] : sc[i], a0, a1, a2, a3, qb[i][j][q][0], qb[i][j][q][1]);
                }
            }
            const bool whole = t0 >= lo_max && t0 + 16 <= hi_min;  // every row sees every token
            const int ke = (int)(signed char)(exps & 0xFF), ve = exps >> 8;
            const float k_mul = pow2f(kMulShift - ke);
            float v_mul = pow2f(ve), v_add = (float)-ve;
            auto factor = [&](int i, int b) -> float { return score_factor(row_mul[i][b], k_mul); };
            // Arguments of the exponentials, x - base + 8 in one FMA; the maximum is only looked for when one of them has outgrown the weights' range in FP16
            // by now (x > base + 6), or there was none before.
            auto argument = [&](int i, int h, int b, float f) -> float {
                const float y = sc[i][2 * h + b];
                return far ? fmaf(y, f, v_add) - base[i][b] + kPShift : fmaf(y, f, v_add - base[i][b] + kPShift);  // (for large scores base - 8 is not exact, the difference is)
            };
            float e[NT][4];
            bool grows = false;
#pragma unroll
            for (int i = 0; i < NT; i++) {
#pragma unroll
                for (int b = 0; b < 2; b++) {
                    const float f = factor(i, b);
#pragma unroll
                    for (int h = 0; h < 2; h++) sc[i][2 * h + b] += sd[i][2 * h + b];
                    if (!whole) {
                        const int row = 8 * i + 2 * t + b, qi = query_of(min(row, n_rows - 1));
                        const int hi = row < n_rows ? min(v.len, hi_of(p, v, qi)) : v.len, lo = row < n_rows ? lo_of(p, v, qi) : 0;  // (nobody reads columns without a row)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const int tok = t0 + tok_k + 8 * h;
                            if (tok < lo || tok >= hi) sc[i][2 * h + b] = kNegInf;
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        e[i][2 * h + b] = argument(i, h, b, f);
                        grows |= e[i][2 * h + b] > limit[i][b];
                    }
                }
            }
            if (__any_sync(0xFFFFFFFFu, grows)) {
                // A tile whose values are zeros has no say in what the weights refer to: they count as values of the largest exponent.  (What it adds to the sums is 0 in any case;
                // zeros have exponent 0, which would push the weights of small values in other blocks out of FP16.)
                uint32_t some = 0u;
#pragma unroll
                for (int y = 0; y < D / 32; y++) {
                    const int tok = t0 + (D == 64 ? 8 * y + (lane >> 2) : (4 * y + (lane >> 3)) & 15);
                    const uint4 w = lds_v4(at_v + 512 * y + 16 * lane);
                    if (tok >= lo_min && tok < hi_max) some |= w.x | w.y | w.z | w.w;
                }
                if (!__any_sync(0xFFFFFFFFu, some != 0u)) {
                    v_add = -(float)HIF8_CACHE_EXP_MAX;
                    v_mul = pow2f(HIF8_CACHE_EXP_MAX);
                }
                bool large = false;
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int b = 0; b < 2; b++) {
                        const float f = factor(i, b);
                        float a = fmaxf(fmaf(sc[i][b], f, v_add), fmaf(sc[i][2 + b], f, v_add));
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 4));
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 8));
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 16));
                        const float n = fmaxf(m[i][b], a), g0 = part_factor(m[i][b], n);
                        m[i][b] = n;
                        base[i][b] = n == kNegInf ? 0.f : n;
                        limit[i][b] = n == kNegInf ? kNegInf : kPLimit;
                        large |= fabsf(base[i][b]) > 131072.f;
                        l[i][b] *= g0;
#pragma unroll
                        for (int x = 0; x < MT; x++) { o[i][x][b] *= g0; o[i][x][2 + b] *= g0; }
                    }
                far = __any_sync(0xFFFFFFFFu, large);
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int b = 0; b < 2; b++)
#pragma unroll
                        for (int h = 0; h < 2; h++) e[i][2 * h + b] = argument(i, h, b, factor(i, b));
            }
            uint32_t pb[NT][2];
#pragma unroll
            for (int i = 0; i < NT; i++) {
#pragma unroll
                for (int y = 0; y < 4; y++) e[i][y] = exp2_approx(e[i][y]);
#pragma unroll
                for (int b = 0; b < 2; b++) l[i][b] = fmaf(e[i][b] + e[i][2 + b], v_mul, l[i][b]);
                pb[i][0] = transpose_8x8(pack_f16(e[i][0], e[i][1]));
                pb[i][1] = transpose_8x8(pack_f16(e[i][2], e[i][3]));
            }
            uint32_t vw[4][VB / 4];  // of the tokens in operand rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
            for (int h = 0; h < 4; h++) {
                const int tok = token_of_row<D>(2 * t + (h & 1) + 8 * (h >> 1));
                if (D == 64) {
                    const uint2 a = lds_v2(at_v + chunk_at<D>(tok, piece >> 1) + 8 * (piece & 1));
                    vw[h][0] = a.x; vw[h][1] = a.y;
                } else {
#pragma unroll
                    for (int y = 0; y < VB / 16; y++) {
                        const uint4 a = lds_v4(at_v + chunk_at<D>(tok, 8 * y + piece));
                        vw[h][4 * y] = a.x; vw[h][4 * y + 1] = a.y; vw[h][(4 * y + 2) % (VB / 4)] = a.z; vw[h][(4 * y + 3) % (VB / 4)] = a.w;
                    }
                }
                // What no row sees is not there; of what some rows see and others do not, Inf and NaN are left out, since 0 times them would reach the
                // others: cache_attention_specials_kernel adds them to the rows that do see them.
                if (!whole) {
                    const bool in = t0 + tok >= lo_min && t0 + tok < hi_max;
                    const bool mixed = t0 + tok >= hi_min || t0 + tok < lo_max;
#pragma unroll
                    for (int y = 0; y < VB / 4; y++) vw[h][y] = !in ? 0u : mixed ? finite_codes(vw[h][y]) : vw[h][y];
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
                        const uint32_t sel = 0x7604u + 0x10u * (uint32_t)(2 * (x & 1) + b);
                        a[2 * h + b] = __byte_perm(lds_u32(__byte_perm(vw[2 * h][wd], lut, sel)), lds_u32(__byte_perm(vw[2 * h + 1][wd], lut, sel)), 0x5410);
                    }
#pragma unroll
                for (int i = 0; i < NT; i++) mma_16816_f16(o[i][x], a[0], a[1], a[2], a[3], pb[i][0], pb[i][1]);
            }
#pragma unroll
            for (int x = 0; x + 1 < S::kStages; x++) { ahead_t0[x] = ahead_t0[x + 1]; ahead_exps[x] = ahead_exps[x + 1]; }
            ask(use + S::kStages, ahead_t0[S::kStages - 1], ahead_exps[S::kStages - 1]);
            use++;
        }
        if (!ok) {  // copies on their way land before the block's shared memory becomes another's
#pragma unroll
            for (int x = 0; x < S::kStages; x++)
                if (ahead_t0[x] >= 0) wait_landed(bars + 8 * ((use + x) % S::kStages), ((use + x) / S::kStages) & 1u);
            __syncwarp();
        }

        // ---- the four warps' sums of the segment (all warps': WIDE); the next segment's first tiles and queries are asked for meanwhile
        const int done_q0 = e0.q0, done_h0 = e0.h0, done_head = e0.head;
        bool more = false;
        const bool is_whole = e0.c0 == 0 && e0.c1 == e0.per_unit;
        float* record = p.partial + (size_t)(2 * me + (e0.c0 == 0 ? 1 : 0)) * S::kRecord;
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int b = 0; b < 2; b++) {
                l[i][b] += __shfl_xor_sync(0xFFFFFFFFu, l[i][b], 4);
                l[i][b] += __shfl_xor_sync(0xFFFFFFFFu, l[i][b], 8);
                l[i][b] += __shfl_xor_sync(0xFFFFFFFFu, l[i][b], 16);
                if (g == 0) all_ml[gw * S::kRows + 8 * i + 2 * t + b] = make_float2(m[i][b], l[i][b]);
            }
#pragma unroll
        for (int x = 0; x < S::kStages; x++) ahead_t0[x] = -1;
#pragma unroll
        for (int pass = 0; pass < S::kRows / S::kJoinRows; pass++) {
            if (pass * S::kJoinRows >= n_rows) break;  // (the same in the whole group)
            if (pass) group_sync(grp, GW * 32);
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int b = 0; b < 2; b++) {
                    const int row = 8 * i + 2 * t + b;
                    if (row / S::kJoinRows == pass) {
#pragma unroll
                        for (int x = 0; x < MT; x += 2) {
                            const int d = D == 64 ? 8 * piece + 2 * x : 128 * (x / 8) + 16 * piece + 2 * (x % 8);
                            *reinterpret_cast<float4*>(smem_raw + S::sum_at(warp, row % S::kJoinRows, d / 4)) = make_float4(o[i][x][b], o[i][x][2 + b], o[i][x + 1][b], o[i][x + 1][2 + b]);
                        }
                    }
                }
            group_sync(grp, GW * 32);
            if (pass == 0) {
                more = advance();
                if (more) begin();
            }
            const int rows = min(S::kJoinRows, n_rows - pass * S::kJoinRows);
            for (int i = gw * 32 + lane; i < rows * (D / 4); i += GW * 32) {
                const int in_pass = i / (D / 4), row = pass * S::kJoinRows + in_pass, f = i % (D / 4);
                float2 ml[GW];
                float top = kNegInf, den = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < GW; w++) { ml[w] = all_ml[w * S::kRows + row]; top = fmaxf(top, ml[w].x); }
#pragma unroll
                for (int w = 0; w < GW; w++) {
                    const float h = part_factor(ml[w].x, top);
                    den += ml[w].y * h;
                    const float4 a = *reinterpret_cast<const float4*>(smem_raw + S::sum_at(grp * GW + w, in_pass, f));
                    x[0] += a.x * h; x[1] += a.y * h; x[2] += a.z * h; x[3] += a.w * h;
                }
                if (is_whole) {
                    const int step = step_of(done_h0, row), h = done_head * p.group + done_h0 + row - step * p.group;
                    const long long tok = v.first + done_q0 + step;
                    const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
                    for (int y = 0; y < 4; y++) x[y] *= inv;
                    resolve_specials(p, (int)tok, done_head, 4 * f, den, x);
                    store_out4<DT>(p, tok * p.out_token + (long long)h * p.out_head + 4 * f, x);
                    if (p.lse && f == 0) p.lse[tok * p.heads + h] = lse_of(top, den, kPShift);
                } else {
                    *reinterpret_cast<float4*>(record + row * D + 4 * f) = make_float4(x[0], x[1], x[2], x[3]);
                    if (f == 0) *reinterpret_cast<float2*>(record + S::kRows * D + 2 * row) = make_float2(top, den);
                }
            }
        }
        if (more) convert_queries();
        if (group_any(grp, GW * 32, !ok) || !more) break;
    }
    if (!ok || *abort_flag) {
#pragma unroll
        for (int x = 0; x < S::kStages; x++)
            if (ahead_t0[x] >= 0) wait_landed(bars + 8 * ((use + x) % S::kStages), ((use + x) / S::kStages) & 1u);
    }
}

// Block b - 1 joins the unit that the boundary between groups b - 1 and b cuts, if that is the first one to do so; the parts are added in the groups' order.
// A unit may lie in all groups: the parts' factors come first, then threads share the parts of a result out among them.
constexpr int kCombineThreads = 512;
template <int D, int NT, int DT>
__global__ void __launch_bounds__(kCombineThreads) cache_attention_combine_kernel(const __grid_constant__ AttentionParams p, int all_groups)
{
    using S = RowsShape<D, NT, false>;
    constexpr int kMostGroups = kMaxBlocks * S::kGroups, kItems = S::kRows * (D / 4);
    static_assert(kItems <= kCombineThreads, "a thread for every four results");
    __shared__ float s_factor[kMostGroups * S::kRows];
    __shared__ float s_top[S::kRows], s_den[S::kRows];
    __shared__ float4 s_part[kCombineThreads];
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int b = (int)blockIdx.x + 1;
    const long long chunks = *p.chunks;
    const int4 cut = p.cut[2 * b], of = p.cut[2 * b + 1];  // (of a group that has no chunks: not looked at)
    const int groups = (int)min((long long)all_groups, chunks);
    if (b >= groups) return;
    const long long begin = share_of(chunks, b, groups) - cut.z, end = begin + cut.w;
    if (cut.z == 0 || share_of(chunks, b - 1, groups) > begin) return;
    const int parts = owner_of(chunks, end - 1, groups) - (b - 1) + 1;  // groups b - 1 .. b - 2 + parts
    const int head = cut.x, r0 = cut.y, first = of.x, n_rows = of.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto record = [&](int i) -> const float* { return p.partial + (size_t)(2 * (b - 1 + i) + (i == 0 ? 1 : 0)) * S::kRecord; };
    for (int row = warp; row < n_rows; row += kCombineThreads / 32) {
        float top = kNegInf, den = 0.f;
        for (int j = lane; j < parts; j += 32) top = fmaxf(top, record(j)[S::kRows * D + 2 * row]);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        for (int j = lane; j < parts; j += 32) {
            const float2 ml = *reinterpret_cast<const float2*>(record(j) + S::kRows * D + 2 * row);
            const float h = part_factor(ml.x, top);
            s_factor[j * S::kRows + row] = h;
            den += ml.y * h;
        }
#pragma unroll
        for (int d = 1; d < 32; d *= 2) den += __shfl_xor_sync(0xFFFFFFFFu, den, d);
        if (lane == 0) { s_top[row] = top; s_den[row] = den; }
    }
    __syncthreads();
    const int items = n_rows * (D / 4), shares = kCombineThreads / items, item = (int)threadIdx.x % items, share = (int)threadIdx.x / items;
    const int row = item / (D / 4), f = item % (D / 4);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (share < shares) {
#pragma unroll 4
        for (int j = share; j < parts; j += shares) {
            const float4 a = *reinterpret_cast<const float4*>(record(j) + row * D + 4 * f);
            const float h = s_factor[j * S::kRows + row];
            o.x += a.x * h; o.y += a.y * h; o.z += a.z * h; o.w += a.w * h;
        }
        s_part[threadIdx.x] = o;
    }
    __syncthreads();
    if (share != 0) return;
    for (int j = 1; j < shares; j++) {
        const float4 a = s_part[j * items + item];
        o.x += a.x; o.y += a.y; o.z += a.z; o.w += a.w;
    }
    const int r = r0 + row, qi = r / p.group, h = head * p.group + r - qi * p.group;
    const float den = s_den[row], inv = den == 0.f ? 0.f : 1.f / den;
    float x[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    resolve_specials(p, first + qi, head, 4 * f, den, x);
    store_out4<DT>(p, (long long)(first + qi) * p.out_token + (long long)h * p.out_head + 4 * f, x);
    if (p.lse && f == 0) p.lse[(long long)(first + qi) * p.heads + h] = lse_of(s_top[row], den, kPShift);
}

// Inf and NaN among the values of tokens that only some of a sequence's queries see: the rows that do see them get them here.  (Those that all queries
// see take the ordinary way with few rows; chunks leave all of them out of the products, and set a flag where there are some.)  A block looks through `slices` pieces of 16 elements of a key head's value rows, 256 pieces at a time, and keeps a bit for each token,
// element and kind of what it finds; there is hardly ever anything to do, and if there is, a result takes a few words to look at, however much was found.  Without
// a window only the first of a kind in an element counts (whoever sees a later one sees that as well): a cache full of NaN does not make the work quadratic.
template <int DT>
__global__ void __launch_bounds__(kThreads) cache_attention_specials_kernel(const AttentionParams p, int slices)
{
    constexpr int kWords = kThreads;  // (16 slices by words of tokens: 128, and 256 where 16 slices leave half of each word)
    __shared__ uint32_t s_found[3][kWords];  // Inf, -Inf, NaN: [elements][tokens / 32]
    __shared__ uint32_t s_before[256];       // kinds that an element held in earlier rounds
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    if (p.special_flag && !*p.special_flag) return;
    const int head = blockIdx.y, s = blockIdx.z;
    const SeqView v = seq_view(p, s);
    if (v.n_q < (p.special_flag ? 1 : 2)) return;
    // tokens that the last query sees or the first, and not both (chunks: that any sees): [a0, a1) and [b0, b1), number k being a0 + k, and b0 + k - n_a from n_a on
    const int hi1 = min(v.len, hi_of(p, v, v.n_q - 1)), lo0 = lo_of(p, v, 0), hi0 = p.special_flag ? lo0 : min(v.len, hi_of(p, v, 0)), lo1 = p.special_flag ? lo0 : lo_of(p, v, v.n_q - 1);
    const int a0 = lo0, a1 = min(lo1, hi1), b0 = max(hi0, a1), b1 = hi1, n_a = max(0, a1 - a0), n = n_a + max(0, b1 - b0);
    const int step = kThreads / slices, words = (step + 31) / 32, width = 16 * slices;  // tokens at a time
    for (int i = threadIdx.x; i < 3 * kWords; i += kThreads) s_found[i / kWords][i % kWords] = 0u;
    s_before[threadIdx.x] = 0u;  // (kThreads == 256, the most elements)
    __syncthreads();
    auto token = [&](int k) -> int { return k < n_a ? a0 + k : b0 + (k - n_a); };
    for (int k0 = 0; k0 < n; k0 += step) {
        const int kk = (int)threadIdx.x / slices, k = k0 + kk, d0 = ((int)threadIdx.x - kk * slices) * 16;
        bool any = false;
        if (k < n) {
            const int tok = token(k), page = p.c.page_of(s, tok >> p.c.shift);
            uint4 w = make_uint4(0, 0, 0, 0);
            if (page >= 0)
                w = __ldg(reinterpret_cast<const uint4*>(p.c.v + p.c.block_at(page, head) + (long long)(tok & ((1 << p.c.shift) - 1)) * p.c.dim + (int)blockIdx.x * width + d0));
            if (finite_codes(w.x) != w.x || finite_codes(w.y) != w.y || finite_codes(w.z) != w.z || finite_codes(w.w) != w.w)
                for (int d = 0; d < 16; d++) {
                    const uint32_t c = ((d < 4 ? w.x : d < 8 ? w.y : d < 12 ? w.z : w.w) >> (8 * (d & 3))) & 0xFFu;
                    const int kind = c == 0x6Fu ? 0 : c == 0xEFu ? 1 : 2;
                    if ((c == 0x80u || (c & 0x7Fu) == 0x6Fu) && !(s_before[d0 + d] >> kind & 1u)) {
                        atomicOr(&s_found[kind][(d0 + d) * words + (kk >> 5)], 1u << (kk & 31));
                        any = true;
                    }
                }
        }
        if (!__syncthreads_or(any)) continue;
        // rows of queries that see any of the round's tokens
        const int tok0 = token(k0), tok1 = token(min(k0 + step, n) - 1), i0 = p.causal ? max(0, tok0 - v.pos(0)) : 0, i1 = p.window ? (int)min((long long)v.n_q, (long long)tok1 + p.window - v.pos(0)) : v.n_q;
        const long long work = (long long)i1 * p.group * width;
        for (long long x = (long long)i0 * p.group * width + threadIdx.x; x < work; x += kThreads) {
            const int r = (int)(x / width), d = (int)(x - (long long)r * width), qi = r / p.group, h = head * p.group + r - qi * p.group;
            const int hi = min(v.len, hi_of(p, v, qi)), lo = lo_of(p, v, qi);
            // the numbers it sees, from this round's first: of [a0, a1), of [b0, b1)
            const int from[2] = {max(lo - a0, 0) - k0, max(lo - b0 + n_a, n_a) - k0}, to[2] = {min(hi - a0, n_a) - k0, hi - b0 + n_a - k0};
            uint32_t seen[3] = {0u, 0u, 0u};
            for (int y = 0; y < words; y++) {
                uint32_t mask = 0u;
                for (int z = 0; z < 2; z++) {
                    const int f = max(0, min(32, from[z] - 32 * y)), t = max(0, min(32, to[z] - 32 * y));
                    if (f < t) mask |= (uint32_t)((1ull << t) - (1ull << f));
                }
                for (int z = 0; z < 3; z++) seen[z] |= s_found[z][d * words + y] & mask;
            }
            if (seen[0] | seen[1] | seen[2]) {
                const float add = seen[2] || (seen[0] && seen[1]) ? __uint_as_float(0x7FC00000u) : seen[0] ? -kNegInf : kNegInf;
                unsigned short* out = reinterpret_cast<unsigned short*>(p.out) + (long long)(v.first + qi) * p.out_token + (long long)h * p.out_head + (int)blockIdx.x * width + d;
                *out = (unsigned short)to_bits<DT>(q_value<DT>(*out) + add);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 3 * width * words; i += kThreads) {
            const int z = i / (width * words), j = i - z * width * words;
            if (s_found[z][j] && !p.window) atomicOr(&s_before[j / words], 1u << z);
            s_found[z][j] = 0u;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------
constexpr size_t kHeadBytes = 256;  // status word, flag of specials, chunks in all

// n8 tiles of query rows that a warp takes: two where the rows fill more than one and the registers allow it
int row_tiles_of(int max_q, int group, int dim) { return (long long)max_q * group > 8 && dim <= 128 ? 2 : 1; }

size_t partial_bytes(int dim, int nt)
{
    const size_t groups = (size_t)kMaxBlocks * groups_of(dim, nt);
    return round_up_256(groups * 32) + round_up_256(2 * groups * 8 * nt * (dim + 2) * 4);
}

// The pool of K or V as rows of head_dim bytes, boxes of 16 tokens (128 bytes of each at most), swizzled.  Encoded anew in every call: it holds no more than
// the address and the sizes.
bool pool_map(CUtensorMap* map, const void* pool, const CacheView& c)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c.dim, (cuuint64_t)c.pages * c.heads << c.shift}, strides[1] = {(cuuint64_t)c.dim};
    const cuuint32_t box[2] = {(cuuint32_t)(c.dim < 128 ? c.dim : 128), 16}, one[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(pool), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              c.dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct DeviceSetup {
    cudaError_t rc;
};
PerDevice<DeviceSetup> g_setup;

template <int D, int NT, int DT>
cudaError_t allow_shared()
{
    const cudaError_t e = cudaFuncSetAttribute((const void*)cache_attention_rows_kernel<D, NT, DT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RowsShape<D, NT, false>::kSmem);
    return e != cudaSuccess ? e : cudaFuncSetAttribute((const void*)cache_attention_rows_kernel<D, NT, DT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RowsShape<D, NT, true>::kSmem);
}
template <int DT>
cudaError_t allow_shared_of()
{
    cudaError_t e[5] = {allow_shared<64, 1, DT>(), allow_shared<64, 2, DT>(), allow_shared<128, 1, DT>(), allow_shared<128, 2, DT>(), allow_shared<256, 1, DT>()};
    for (cudaError_t x : e)
        if (x != cudaSuccess) return x;
    return cudaSuccess;
}

// Whether units are taken whole by all warps of a block, without a second kernel: where every unit has a block of its own and a warp two tiles of 16 tokens at most.
// us a call in a graph, 8 key heads of 128, BF16, cut / whole: 1 sequence of 100 tokens 9.1 / 6.6, 16 of up to 500 16.3 / 10.6; three tiles a warp: 1 of 517 10.6 / 11.0, two
// rounds of blocks: 64 of up to 300 20.3 / 28.9, 32 of up to 100, 4 key heads and 32 heads to each 16.1 / 21.4.  Heads of 256, whose blocks have two groups of warps and not four, four rounds
// too unless all tokens are one chunk of a group: 16 sequences, 8 key heads, 16 heads to each (two rounds), of up to 60 tokens 12.6 / 15.4, 100 20.2 / 15.7, 250 25.8 / 19.9; 32 (four) of up to
// 250 38.9 / 36.2, 48 (six) 51.8 / 51.1.  (Units and lengths are the host's upper bounds.)
bool whole_units(const AttentionParams& p, int max_q, int max_length, int rows, int warps, int blocks)
{
    // (row tiles of all sequences: as many as the longest has for each, or one more for each than full ones)
    const long long each = ((long long)max_q * p.group + rows - 1) / rows * p.n_seqs, full = (long long)p.n_q * p.group / rows + p.n_seqs;
    const long long units = (each < full ? each : full) * p.c.heads;
    const long long tokens = p.window && p.window + (long long)max_q < max_length ? p.window + (long long)max_q : max_length;
    return units <= (p.c.dim == 256 && tokens > 64 ? 4ll : 1ll) * blocks && tokens <= 32 * warps;
}

template <int D, int NT, int DT, bool WIDE>
cudaError_t launch_rows_form(const AttentionParams& p, int blocks, cudaStream_t st)
{
    using S = RowsShape<D, NT, WIDE>;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CUtensorMap map_k, map_v;
    if (!pool_map(&map_k, p.c.k, p.c) || !pool_map(&map_v, p.c.v, p.c)) return cudaErrorInvalidValue;
    g_launches.fetch_add(WIDE ? 1 : 2, std::memory_order_relaxed);
    const cudaError_t rc = cudaLaunchKernelEx(&cfg, cache_attention_rows_kernel<D, NT, DT, WIDE>, map_k, map_v, p);
    if (WIDE || rc != cudaSuccess) return rc;
    const int groups = blocks * S::kGroups;
    return launch_pdl_threads(kCombineThreads, cache_attention_combine_kernel<D, NT, DT>, dim3((unsigned)(groups - 1)), st, p, groups);
}
template <int D, int NT, int DT>
cudaError_t launch_rows(const AttentionParams& p, int max_q, int max_length, int sms, cudaStream_t st)
{
    const int blocks = sms < kMaxBlocks ? sms : kMaxBlocks;
    if (whole_units(p, max_q, max_length, 8 * NT, RowsShape<D, NT, true>::kWarps, blocks)) return launch_rows_form<D, NT, DT, true>(p, blocks, st);
    return launch_rows_form<D, NT, DT, false>(p, blocks, st);
}
template <int DT>
cudaError_t launch_rows_of(const AttentionParams& p, int nt, int max_q, int max_length, int sms, cudaStream_t st)
{
    if (p.c.dim == 64) return nt == 2 ? launch_rows<64, 2, DT>(p, max_q, max_length, sms, st) : launch_rows<64, 1, DT>(p, max_q, max_length, sms, st);
    if (p.c.dim == 128) return nt == 2 ? launch_rows<128, 2, DT>(p, max_q, max_length, sms, st) : launch_rows<128, 1, DT>(p, max_q, max_length, sms, st);
    return launch_rows<256, 1, DT>(p, max_q, max_length, sms, st);
}

}  // namespace
}  // namespace hif8

using namespace hif8;

extern "C" size_t hif8_cache_attention_workspace_bytes(int n_seqs, int n_q, int max_q, int max_length, int heads, int kv_heads, int head_dim)
{
    if (n_seqs < 0 || n_q < 0 || max_q < 0 || max_length < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || (head_dim != 64 && head_dim != 128 && head_dim != 256)) return 0;
    const size_t rows = partial_bytes(head_dim, row_tiles_of(max_q, heads / kv_heads, head_dim)), tiles = prefill_workspace_bytes(n_seqs, n_q, max_q, max_length, heads, kv_heads, head_dim);
    return kHeadBytes + (rows > tiles ? rows : tiles);
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
    if ((int64_t)n_q * (heads / kv_heads) > 0x3FFFFFFF || ((int64_t)n_pages * kv_heads << p.c.shift) > 0x7FFFFFFF) return HIF8_ERR_SHAPE;
    if (n_seqs == 0 || n_q == 0) return HIF8_OK;
    if (n_pages == 0) return HIF8_ERR_SHAPE;
    if (!q || !out || !d_q_start || !d_lengths) return HIF8_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 1u) return HIF8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(d_q_start) | reinterpret_cast<uintptr_t>(d_lengths) | reinterpret_cast<uintptr_t>(lse)) & 3u) return HIF8_ERR_ALIGN;
    // rows of the result must not share elements: tokens outermost, or heads
    const int64_t inner = out_token_stride < out_head_stride ? out_token_stride : out_head_stride, outer = out_token_stride < out_head_stride ? out_head_stride : out_token_stride;
    const int64_t n_inner = out_token_stride < out_head_stride ? n_q : heads, n_outer = out_token_stride < out_head_stride ? heads : n_q;
    if ((n_inner > 1 && inner < head_dim) || (n_outer > 1 && outer < (n_inner - 1) * inner + head_dim)) return HIF8_ERR_SHAPE;
    const size_t q_bytes = ((size_t)(n_q - 1) * (size_t)q_token_stride + (size_t)(heads - 1) * (size_t)q_head_stride + (size_t)head_dim) * 2;
    const size_t out_bytes = ((size_t)(n_q - 1) * (size_t)out_token_stride + (size_t)(heads - 1) * (size_t)out_head_stride + (size_t)head_dim) * 2;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HIF8_ERR_WORKSPACE;
    const int group = heads / kv_heads;
    int nt = row_tiles_of(max_q, group, head_dim);
    if (workspace_bytes < kHeadBytes + partial_bytes(head_dim, nt)) nt = row_tiles_of(1, group, head_dim);  // (the workspace of single tokens takes any call)
    if (workspace_bytes < kHeadBytes + partial_bytes(head_dim, nt)) return HIF8_ERR_WORKSPACE;
    const size_t tiles = prefill_workspace_bytes(n_seqs, n_q, max_q, max_length, heads, kv_heads, head_dim);
    const bool chunk = tiles && workspace_bytes >= kHeadBytes + tiles;
    const size_t pool = p.c.pool_bytes(), exps = p.c.exp_bytes();
    if (written_over({{out, out_bytes}, {lse, lse ? (size_t)n_q * (size_t)heads * 4 : 0}, {workspace, kHeadBytes + (chunk ? tiles : partial_bytes(head_dim, nt))}},
                     {{q, q_bytes}, {k_pages, pool}, {v_pages, pool}, {k_exp, exps}, {v_exp, exps}, {page_table, p.c.table_bytes(n_seqs)}, {d_q_start, (size_t)(n_seqs + 1) * 4},
                      {d_lengths, (size_t)n_seqs * 4}}))
        return HIF8_ERR_OVERLAP;
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
    p.scale_log2 = fminf(softmax_scale * kLog2e, 3.0e38f); p.causal = causal != 0; p.window = window < 1 << 30 ? window : 1 << 30;  // (lengths and queries stay below 2^30: positions minus a window stay inside an int)
    p.out = out; p.out_token = out_token_stride; p.out_head = out_head_stride; p.lse = lse;
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
    p.status = reinterpret_cast<int*>(ws);
    p.chunks = reinterpret_cast<long long*>(ws + 8);
    p.cut = reinterpret_cast<int4*>(ws + kHeadBytes);
    p.partial = reinterpret_cast<float*>(ws + kHeadBytes + round_up_256((size_t)kMaxBlocks * groups_of(head_dim, nt) * 32));
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t rc;
    p.special_flag = nullptr;
    if (chunk) {
        p.special_flag = p.status + 1;
        rc = launch_prefill(p, dtype, max_length, ws + kHeadBytes, sms, st);
    } else rc = dtype == HIF8_BF16 ? launch_rows_of<HIF8_BF16>(p, nt, max_q, max_length, sms, st) : launch_rows_of<HIF8_F16>(p, nt, max_q, max_length, sms, st);
    if (rc == cudaSuccess && (p.special_flag || (max_q > 1 && (p.causal || p.window)))) {
        const int slices = p.special_flag ? 1 : head_dim / 16;  // (few rows: few tokens to look at)
        const dim3 grid((unsigned)(head_dim / 16 / slices), (unsigned)kv_heads, (unsigned)n_seqs);
        rc = dtype == HIF8_BF16 ? launch_pdl(cache_attention_specials_kernel<HIF8_BF16>, grid, st, p, slices) : launch_pdl(cache_attention_specials_kernel<HIF8_F16>, grid, st, p, slices);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    note_status_word(st, p.status);
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}
