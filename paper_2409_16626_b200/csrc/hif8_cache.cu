// The HiF8 key/value cache: new tokens into its pages (append), tokens back out (read), sequences that continue from another's
// pages (fork), and live pages moved together (compact).  Attention over the cache is in hif8_cache_attention.cu.
//
// All four are bound by the bytes they move; small calls by launches and by how many loads wait for one another.  Measured (us, of the measured copy bandwidth):
// 27.7 K tokens of prompts, 8 heads of 128, BF16, appended and read back 71 (73 %; alone 41 and 38), FP32 57 and 67 (76 and 65 %), 128 single tokens 8.4 on the device for both calls; 512
// samples forked, pages of 128 tokens 26 (82 %); 3.6 K pages of 64 tokens moved 170 (84 %).
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "hif8.h"
#include "hif8_cache.cuh"
#include "hif8_device.cuh"
#include "hif8_internal.cuh"

namespace hif8 {
extern std::atomic<uint64_t> g_launches;
namespace {

// ---------------------------------------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------------------------------------
struct AppendParams {
    CacheView c;
    const void* src[2];  // K, V
    long long token_stride, head_stride;
    const int* start;
    const int* lengths;
    int n_seqs, n_new;
    long long units;  // pieces x heads x 2
    int vectors;      // 16-byte loads
    int target_exp;
    unsigned flags;
};

// A block of a cache (one page's tokens of one head of K or V) is converted by TEAM threads: their part of it stays in registers between the
// reduction of its largest magnitude and the conversion, so the source is read once, and the next block's part is on its way meanwhile; what a block has beyond what
// they hold is read twice, the second time from L2.  A warp holds 2 KiB of a 16-bit source and 4 KiB of FP32, 256 threads 16 KiB and
// 32 KiB (64 tokens of 128 elements), 512 threads 64 KiB: the smallest team that holds a block of the call takes it (27.7 K tokens of 8 heads, BF16, with the reading call, us: pages of 64 x 128
// by 256 threads 70; of 128 x 128 by 256 / 512: 108 / 92; of 16 x 64 by 256 threads / a warp: 108 / 44).
template <int SRC, int TEAM> struct AppendShape {
    static constexpr int kBlock = TEAM > kThreads ? TEAM : kThreads;                       // threads of a block
    static constexpr int kHeld = TEAM > kThreads || SRC == HIF8_F32 ? 8 : 4;               // vectors of a unit in a thread's registers
};
template <int MODE, int SRC, int TEAM>
__global__ void __launch_bounds__(AppendShape<SRC, TEAM>::kBlock) cache_append_kernel(const AppendParams p)
{
    constexpr int PV = SrcTraits<SRC>::kPerVec, kHeld = AppendShape<SRC, TEAM>::kHeld, kBlock = AppendShape<SRC, TEAM>::kBlock;
    __shared__ SmemTables s;
    __shared__ uint32_t s_part[2][kBlock / 32];
    setup_tables<true, MODE != HIF8_RND_TA, false, MODE, SRC, kBlock>(s, p.flags);
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, member = threadIdx.x % TEAM;
    const int row_vecs = p.c.dim / PV, row_shift = 31 - __clz(row_vecs);
    UnitWalk walk(p.units, 2 * p.c.heads, (long long)blockIdx.x * (kBlock / TEAM) + threadIdx.x / TEAM, (long long)gridDim.x * (kBlock / TEAM));
    // the unit that is loaded, in a thread's registers; the one before it is being converted
    Piece pc;
    int page = -1, n_vec = 0, n_units = 0;
    const char* src = nullptr;
    auto load = [&](const char* from, int i) -> uint4 {
        const int t = i >> row_shift;
        const long long e = (long long)t * p.token_stride + (long long)(i - (t << row_shift)) * PV;
        if (p.vectors) return __ldcs(reinterpret_cast<const uint4*>(from + e * (16 / PV)));
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; j++)
            w[j] = SRC == HIF8_F32 ? reinterpret_cast<const uint32_t*>(from)[e + j]
                                   : (uint32_t)reinterpret_cast<const unsigned short*>(from)[e + 2 * j] | ((uint32_t)reinterpret_cast<const unsigned short*>(from)[e + 2 * j + 1] << 16);
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    uint4 held[kHeld];
    auto begin = [&]() {  // the next unit that there is something of; n_vec = 0: there is none
        n_vec = 0;
        for (; walk.left > 0; walk.next()) {
            if (walk.fresh || n_units == 0) {
                pc = find_piece(walk.number, p.start, p.lengths, p.n_seqs, p.n_new, p.c.shift, lane);
                page = pc.count ? p.c.page_of(pc.seq, pc.pos >> p.c.shift) : -1;
            }
            n_units++;
            if (page < 0) continue;  // (the same answer in the whole team)
            n_vec = pc.count << row_shift;
            src = reinterpret_cast<const char*>(p.src[walk.part & 1]) + ((long long)pc.token * p.token_stride + (long long)(walk.part >> 1) * p.head_stride) * (16 / PV);
#pragma unroll
            for (int j = 0; j < kHeld; j++) held[j] = member + j * TEAM < n_vec ? load(src, member + j * TEAM) : make_uint4(0, 0, 0, 0);
            return;
        }
    };
    begin();
    int parity = 0;
    while (n_vec > 0) {
        uint4 mine[kHeld];
#pragma unroll
        for (int j = 0; j < kHeld; j++) mine[j] = held[j];
        const int count = n_vec, slot = pc.pos & ((1 << p.c.shift) - 1), head = walk.part >> 1;
        const bool is_v = walk.part & 1;
        const char* from = src;
        int* exps = (is_v ? p.c.v_exp : p.c.k_exp) + ((long long)page * p.c.heads + head);
        uint8_t* dst = (is_v ? p.c.v : p.c.k) + p.c.block_at(page, head) + (long long)slot * p.c.dim;
        walk.next();
        begin();
        int e;
        if (slot) e = clamp_cache_exp(*exps);  // the block's first tokens set its exponent
        else {
            uint32_t acc = 0;
#pragma unroll
            for (int j = 0; j < kHeld; j++) acc = amax_vector<SRC>(acc, mine[j]);
            for (int i = member + kHeld * TEAM; i < count; i += TEAM) acc = amax_vector<SRC>(acc, load(from, i));
            uint32_t a = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(amax_value<SRC>(acc)));
            if (TEAM > 32) {  // (two places in turn: whoever is still reading one is waited for at the other's barrier)
                if (lane == 0) s_part[parity][threadIdx.x >> 5] = a;
                __syncthreads();
                a = __reduce_max_sync(0xFFFFFFFFu, lane < TEAM / 32 ? s_part[parity][lane] : 0u);
                parity ^= 1;
            }
            e = clamp_cache_exp(scale_exp_from_amax(a, p.target_exp));
            if (member == 0) *exps = e;
        }
        const float scale = pow2f(e);
        uint32_t scale2[4];
        float scales[8];
#pragma unroll
        for (int j = 0; j < 4; j++) scale2[j] = bf16x2_of_pow2(scale);
#pragma unroll
        for (int j = 0; j < 8; j++) scales[j] = scale;
        auto convert = [&](int i, const uint4& v) {
            uint2 w;
            if (MODE == HIF8_RND_TA) w = encode_vector_ta<SRC>(v, scale2, scales, s.ta);
            else {
                uint32_t c[8];
#pragma unroll
                for (int k = 0; k < PV; k++) {
                    float x; uint32_t raw;
                    unpack<SRC>(v, k, x, raw);
                    c[k] = encode_one<MODE, SRC>(x, raw, scale, s.ta, s.thr, 0u);
                }
                w.x = c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24);
                if (PV == 8) w.y = c[4] | (c[5] << 8) | (c[6] << 16) | (c[7] << 24);
            }
            if (PV == 8) *reinterpret_cast<uint2*>(dst + (long long)i * 8) = w;
            else *reinterpret_cast<uint32_t*>(dst + (long long)i * 4) = w.x;
        };
#pragma unroll
        for (int j = 0; j < kHeld; j++)
            if (member + j * TEAM < count) convert(member + j * TEAM, mine[j]);
        for (int i = member + kHeld * TEAM; i < count; i += TEAM) convert(i, load(from, i));
    }
}

template <int MODE, int SRC, int TEAM>
void launch_append_team(const AppendParams& p, int sms, cudaStream_t st)
{
    constexpr int kBlock = AppendShape<SRC, TEAM>::kBlock;
    const long long blocks = (p.units * TEAM + kBlock - 1) / kBlock, most = (long long)sms * 4;
    launch_pdl_threads(kBlock, cache_append_kernel<MODE, SRC, TEAM>, dim3((unsigned)(blocks < most ? blocks : most)), st, p);
}
// tokens: what a sequence has in the mean, up to a page
template <int MODE, int SRC>
void launch_append(const AppendParams& p, int tokens, int sms, cudaStream_t st)
{
    const int vecs = tokens * p.c.dim / SrcTraits<SRC>::kPerVec;
    if (vecs <= 32 * AppendShape<SRC, 32>::kHeld) launch_append_team<MODE, SRC, 32>(p, sms, st);
    else if (vecs <= 256 * AppendShape<SRC, 256>::kHeld) launch_append_team<MODE, SRC, 256>(p, sms, st);
    else launch_append_team<MODE, SRC, 512>(p, sms, st);
}
template <int MODE>
void launch_append_of(int dtype, const AppendParams& p, int tokens, int sms, cudaStream_t st)
{
    if (dtype == HIF8_F32) launch_append<MODE, HIF8_F32>(p, tokens, sms, st);
    else if (dtype == HIF8_BF16) launch_append<MODE, HIF8_BF16>(p, tokens, sms, st);
    else launch_append<MODE, HIF8_F16>(p, tokens, sms, st);
}

// ---------------------------------------------------------------------------------------------------------
// Read
// ---------------------------------------------------------------------------------------------------------
struct ReadParams {
    CacheView c;
    void* dst[2];
    long long token_stride, head_stride;
    const int* start;
    const int* first;
    int n_seqs, n_out;
    long long units;
    int vectors;
};

template <int DT> struct OutVec;  // 16 bytes of results
template <> struct OutVec<HIF8_F32> { static constexpr int n = 4; };
template <> struct OutVec<HIF8_BF16> { static constexpr int n = 8; };
template <> struct OutVec<HIF8_F16> { static constexpr int n = 8; };

// Codes are looked up in a table that every lane has a copy of (see fill_lane_table), as BF16 for BF16 results, which a packed product with the
// block's power of two then finishes, and as FP32 otherwise.  A warp takes a unit; tokens of an entry that names no page read as zeros.
template <int DT>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const ReadParams p)
{
    __shared__ __align__(16) uint32_t table[kLaneTableWords];
    const uint32_t f = decode_bits_f32(threadIdx.x);  // kThreads == 256 codes
    fill_lane_table(table, DT == HIF8_BF16 ? f >> 16 : f);
    __syncthreads();
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    constexpr int N = OutVec<DT>::n;
    const int lane = threadIdx.x & 31;
    const uint32_t lane4 = 4u * lane;
    const int row_vecs = p.c.dim / N;
    UnitWalk walk(p.units, 2 * p.c.heads, (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), (long long)gridDim.x * (kThreads / 32));
    Piece pc;
    int page = -1;
    for (; walk.left > 0; walk.next()) {
        const int head = walk.part >> 1;
        const bool is_v = walk.part & 1;
        if (walk.fresh) {
            pc = find_piece(walk.number, p.start, p.first, p.n_seqs, p.n_out, p.c.shift, lane);
            page = pc.count ? p.c.page_of(pc.seq, pc.pos >> p.c.shift) : -1;
        }
        if (!pc.count) continue;
        const int slot = pc.pos & ((1 << p.c.shift) - 1), n_vec = pc.count * row_vecs;
        const int e = page < 0 ? 0 : clamp_cache_exp((is_v ? p.c.v_exp : p.c.k_exp)[(long long)page * p.c.heads + head]);
        const float back = pow2f(-e);
        const uint32_t back2 = bf16x2_of_pow2(back);
        const uint8_t* src = (is_v ? p.c.v : p.c.k) + (page < 0 ? 0ll : p.c.block_at(page, head) + (long long)slot * p.c.dim);
        char* dst = reinterpret_cast<char*>(p.dst[is_v]);
        constexpr int kStep = 4;
        for (int i0 = lane; i0 < n_vec; i0 += 32 * kStep) {
            uint32_t w[kStep][N / 4];
#pragma unroll
            for (int j = 0; j < kStep; j++) {
                const int i = i0 + 32 * j;
#pragma unroll
                for (int x = 0; x < N / 4; x++) w[j][x] = 0u;
                if (i < n_vec && page >= 0) {
                    if (N == 8) {
                        const uint2 a = __ldg(reinterpret_cast<const uint2*>(src + (long long)i * 8));
                        w[j][0] = a.x; w[j][N / 4 - 1] = a.y;
                    } else w[j][0] = __ldg(reinterpret_cast<const uint32_t*>(src + (long long)i * 4));
                }
            }
#pragma unroll
            for (int j = 0; j < kStep; j++) {
                const int i = i0 + 32 * j;
                if (i >= n_vec) break;
                uint32_t o[4];
                if (DT == HIF8_BF16) {
#pragma unroll
                    for (int x = 0; x < N / 4; x++) {
                        const uint2 a = lane_lookup4(table, w[j][x], lane4);
                        o[2 * x] = mul_bf16x2(a.x, back2); o[(2 * x + 1) & 3] = mul_bf16x2(a.y, back2);
                    }
                } else {
                    float v[N];
#pragma unroll
                    for (int x = 0; x < N / 4; x++) {
                        v[4 * x] = __uint_as_float(lane_lookup<0>(table, w[j][x], lane4)) * back; v[4 * x + 1] = __uint_as_float(lane_lookup<1>(table, w[j][x], lane4)) * back;
                        v[4 * x + 2] = __uint_as_float(lane_lookup<2>(table, w[j][x], lane4)) * back; v[4 * x + 3] = __uint_as_float(lane_lookup<3>(table, w[j][x], lane4)) * back;
                    }
#pragma unroll
                    for (int x = 0; x < 4; x++)
                        o[x] = DT == HIF8_F32 ? to_bits<HIF8_F32>(v[x]) : (to_bits<HIF8_F16>(v[(2 * x) % N]) | (to_bits<HIF8_F16>(v[(2 * x + 1) % N]) << 16));
                }
                const int t = i / row_vecs;
                const long long at = (long long)(pc.token + t) * p.token_stride + (long long)head * p.head_stride + (long long)(i - t * row_vecs) * N;
                if (p.vectors) __stcs(reinterpret_cast<uint4*>(dst + at * (16 / N)), make_uint4(o[0], o[1], o[2], o[3]));
                else {
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        if (DT == HIF8_F32) reinterpret_cast<uint32_t*>(dst)[at + x] = o[x];
                        else {
                            reinterpret_cast<unsigned short*>(dst)[at + 2 * x] = (unsigned short)o[x];
                            reinterpret_cast<unsigned short*>(dst)[at + 2 * x + 1] = (unsigned short)(o[x] >> 16);
                        }
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------
// Copies of whole pages
// ---------------------------------------------------------------------------------------------------------
// Eight loads in flight a thread, eight blocks an SM (3.6 K pages of 64 tokens, 8 heads of 128, moved, us: two loads 191, four 176, eight 174; four blocks 186).
constexpr int kCopyUnroll = 8;
constexpr int kCopyBytes = kThreads * 16 * kCopyUnroll;  // 32 KiB: what a block copies at a time

// part `part` of page `from` to page `to`: parts of kCopyBytes of K, then of V; the first one also takes the exponents
__device__ __forceinline__ void copy_page_part(const CacheView& c, int from, int to, int part, int parts)
{
    const long long bytes = c.page_bytes();
    uint8_t* pool = 2 * part < parts ? c.k : c.v;
    const long long at = (long long)(2 * part < parts ? part : part - parts / 2) * kCopyBytes;
    const uint4* src = reinterpret_cast<const uint4*>(pool + from * bytes + at);
    uint4* dst = reinterpret_cast<uint4*>(pool + to * bytes + at);
    const int n = (int)(min((long long)kCopyBytes, bytes - at) / 16);
    uint4 v[kCopyUnroll];
#pragma unroll
    for (int j = 0; j < kCopyUnroll; j++)
        if ((int)threadIdx.x + j * kThreads < n) v[j] = src[threadIdx.x + j * kThreads];
#pragma unroll
    for (int j = 0; j < kCopyUnroll; j++)
        if ((int)threadIdx.x + j * kThreads < n) dst[threadIdx.x + j * kThreads] = v[j];
    if (part == 0)
        for (int i = threadIdx.x; i < 2 * c.heads; i += kThreads) {
            int* e = i < c.heads ? c.k_exp : c.v_exp;
            const int h = i < c.heads ? i : i - c.heads;
            e[(long long)to * c.heads + h] = e[(long long)from * c.heads + h];
        }
}
int copy_parts(const CacheView& c) { return 2 * (int)((c.page_bytes() + kCopyBytes - 1) / kCopyBytes); }

struct ForkParams {
    CacheView c;
    const int* lengths;
    const int* parent;
    const int* new_page;
    int* table_out;
    long long out_stride;
    int* lengths_out;
    int n_seqs, n_children, parts;
};

// A block takes a part of a child's copied page; that of the first part also writes the child's row and length.
__global__ void __launch_bounds__(kThreads) cache_fork_kernel(const ForkParams p)
{
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int child = blockIdx.x, part = blockIdx.y;
    const int par = p.parent[child];
    const bool ok = (unsigned)par < (unsigned)p.n_seqs;
    const int len = ok ? min(p.c.length(p.lengths[par]), (int)min((long long)p.c.capacity(), p.out_stride << p.c.shift)) : 0;
    const int used = (len + (1 << p.c.shift) - 1) >> p.c.shift, last = used - 1;
    int page = p.new_page ? p.new_page[child] : -1;
    const int from = used ? p.c.page_of(par, last) : -1;
    bool copies = (len & ((1 << p.c.shift) - 1)) && from >= 0 && (unsigned)page < (unsigned)p.c.pages && page != from;
    // a page that an earlier child names as well is that one's
    int taken = 0;
    if (copies)
        for (int i = threadIdx.x; i < child; i += kThreads) taken |= p.new_page[i] == page;
    copies = !__syncthreads_or(taken) && copies;
    if (part == 0) {
        const int* row = p.c.table + (ok ? (long long)par * p.c.table_stride : 0ll);
        int* out = p.table_out + (long long)child * p.out_stride;
        for (long long i = threadIdx.x; i < p.out_stride; i += kThreads) out[i] = i >= used ? -1 : (i == last && copies ? page : row[i]);
        if (threadIdx.x == 0) p.lengths_out[child] = len;
    }
    if (copies) copy_page_part(p.c, from, page, part, p.parts);
}

// ---------------------------------------------------------------------------------------------------------
// Compaction
// ---------------------------------------------------------------------------------------------------------
struct CompactParams {
    CacheView c;
    int* table;
    const int* lengths;
    int n_seqs, move, parts;
    uint32_t* live;    // a bit a page
    int* counts;       // live pages, pages that move
    int* to;           // [pages] new number of a page that moves
    int* movers;       // [pages] those pages in order
    int* holes;        // [pages] free pages below the live count, in order
    int* n_live_out;
    int* free_out;
    int words;
    int mark_here;     // the ranking block marks, in its shared memory
};
constexpr int kRankThreads = 1024;
// Up to that many table entries and pages one block marks and ranks, a launch instead of three; beyond, its single SM takes longer to read the table
// than the other launches cost (us a call that moves nothing, one launch / three: 2048 entries and 1024 pages 5.9 / 6.3, 4096 and 2048 6.7 / 6.7, 8192 and 4096 9.5 / 8.3, 65536 and 32768
// 50 / 28).
constexpr long long kMarkHereEntries = 1 << 12;
constexpr int kMarkHereWords = 8192;

__device__ __forceinline__ void mark_entry(const CompactParams& p, long long e, uint32_t* bits)
{
    const int seq = (int)(e / p.c.table_stride), i = (int)(e - (long long)seq * p.c.table_stride);
    if (((long long)i << p.c.shift) >= p.c.length(p.lengths[seq])) return;
    const int page = p.c.page_of(seq, i);
    if (page >= 0) atomicOr(bits + (page >> 5), 1u << (page & 31));
}

__global__ void __launch_bounds__(kThreads) cache_clear_kernel(const CompactParams p)
{
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < p.words; i += gridDim.x * kThreads) p.live[i] = 0u;
}

__global__ void __launch_bounds__(kThreads) cache_mark_kernel(const CompactParams p)
{
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const long long n = (long long)p.n_seqs * p.c.table_stride;
    for (long long e = (long long)blockIdx.x * kThreads + threadIdx.x; e < n; e += (long long)gridDim.x * kThreads) mark_entry(p, e, p.live);
}

// sum of v over the threads in front of this one; *total: over all of them
__device__ __forceinline__ int block_prefix(int v, int* total, int* s_warp)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    int w = s_warp[lane];  // (kRankThreads / 32 == 32 warps)
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, w, d);
        if (lane >= d) w += y;
    }
    *total = __shfl_sync(0xFFFFFFFFu, w, 31);
    const int before = warp ? __shfl_sync(0xFFFFFFFFu, w, warp - 1) : 0;
    return before + x - v;
}

// One block: counts the live pages, then ranks those that have to move, the holes that take them, and the free pages.  A thread takes
// consecutive words, so ranks follow from one sum over the block.
__global__ void __launch_bounds__(kRankThreads) cache_rank_kernel(const CompactParams p)
{
    __shared__ uint32_t s_live[kMarkHereWords];
    __shared__ int s_warp[32];
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const uint32_t* live = p.live;
    if (p.mark_here) {
        for (int i = threadIdx.x; i < p.words; i += kRankThreads) s_live[i] = 0u;
        __syncthreads();
        const long long n = (long long)p.n_seqs * p.c.table_stride;
        for (long long e = threadIdx.x; e < n; e += kRankThreads) mark_entry(p, e, s_live);
        __syncthreads();
        live = s_live;
    }
    const int each = (p.words + kRankThreads - 1) / kRankThreads, w0 = min(p.words, (int)threadIdx.x * each), w1 = min(p.words, w0 + each);
    int mine = 0, n_live, dummy;
    for (int w = w0; w < w1; w++) mine += __popc(live[w]);
    block_prefix(mine, &n_live, s_warp);
    // the word's pages at and beyond the live count / below it
    auto above = [&](int w) -> uint32_t { const int b = n_live - 32 * w; return b <= 0 ? 0xFFFFFFFFu : b >= 32 ? 0u : 0xFFFFFFFFu << b; };
    auto exist = [&](int w) -> uint32_t { const int b = p.c.pages - 32 * w; return b >= 32 ? 0xFFFFFFFFu : (1u << b) - 1u; };
    int movers = 0, holes = 0, free_pages = 0;
    for (int w = w0; w < w1; w++) {
        const uint32_t x = live[w], f = ~x & exist(w);
        movers += __popc(x & above(w)); holes += __popc(f & ~above(w)); free_pages += __popc(f);
    }
    int n_move;
    int rm = block_prefix(movers, &n_move, s_warp), rh = block_prefix(holes, &dummy, s_warp), rf = block_prefix(free_pages, &dummy, s_warp);
    for (int w = w0; w < w1; w++) {
        const uint32_t x = live[w];
        for (uint32_t m = x & above(w); m; m &= m - 1) {
            const int page = 32 * w + __ffs(m) - 1;
            p.movers[rm] = page;
            p.to[page] = rm++;
        }
        for (uint32_t m = ~x & exist(w) & ~above(w); m; m &= m - 1) p.holes[rh++] = 32 * w + __ffs(m) - 1;
        if (!p.move)
            for (uint32_t m = ~x & exist(w); m; m &= m - 1) p.free_out[rf++] = 32 * w + __ffs(m) - 1;
    }
    const int n_free = p.c.pages - n_live;
    for (int i = threadIdx.x; i < p.c.pages; i += kRankThreads) {
        if (i >= n_free) p.free_out[i] = -1;
        else if (p.move) p.free_out[i] = n_live + i;
    }
    if (threadIdx.x == 0) { *p.n_live_out = n_live; p.counts[0] = n_live; p.counts[1] = n_move; }
}

// moves the pages, and rewrites the entries that name them
__global__ void __launch_bounds__(kThreads) cache_move_kernel(const CompactParams p)
{
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int n_live = p.counts[0], n_move = p.counts[1];
    const long long work = (long long)n_move * p.parts;
    for (long long i = blockIdx.x; i < work; i += gridDim.x) {
        const int r = (int)(i / p.parts);
        copy_page_part(p.c, p.movers[r], p.holes[r], (int)(i - (long long)r * p.parts), p.parts);
    }
    const long long n = n_move ? (long long)p.n_seqs * p.c.table_stride : 0;
    for (long long e = (long long)blockIdx.x * kThreads + threadIdx.x; e < n; e += (long long)gridDim.x * kThreads) {
        const int seq = (int)(e / p.c.table_stride), j = (int)(e - (long long)seq * p.c.table_stride);
        if (((long long)j << p.c.shift) >= p.c.length(p.lengths[seq])) continue;
        const int page = p.c.page_of(seq, j);
        if (page >= n_live) p.table[e] = p.holes[p.to[page]];
    }
}

size_t round_up_256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace
}  // namespace hif8

using namespace hif8;

static bool aligned_rows(const void* a, const void* b, int64_t token_stride, int64_t head_stride, size_t item)
{
    return !((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15u) && !((token_stride * (int64_t)item) & 15) && !((head_stride * (int64_t)item) & 15);
}
// Whether a row of one result and a row of another of the same strides, `delta` elements apart, share an element (slices of one tensor do not): for each
// distance in heads the tokens' distance that comes closest.
static bool rows_meet(int64_t delta, int64_t token_stride, int64_t head_stride, int n, int heads, int dim)
{
    for (int h = 1 - heads; h < heads; h++) {
        const int64_t rest = delta + h * head_stride;
        int64_t t = token_stride ? -rest / token_stride : 0;
        for (int64_t x = t - 1; x <= t + 1; x++) {
            const int64_t y = x < 1 - n ? 1 - n : x > n - 1 ? n - 1 : x, gap = rest + y * token_stride;
            if (gap > -dim && gap < dim) return true;
        }
    }
    return false;
}
static bool ints_aligned(const void* a, const void* b = nullptr, const void* c = nullptr, const void* d = nullptr)
{
    return !((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c) | reinterpret_cast<uintptr_t>(d)) & 3u);
}
static int finish_launch(int n)
{
    g_launches.fetch_add((uint64_t)n, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}

extern "C" int hif8_cache_append(const void* k, const void* v, int src_dtype, int64_t token_stride, int64_t head_stride, const int* d_new_start, const int* d_lengths,
                                 int n_seqs, int n_new, uint8_t* k_pages, uint8_t* v_pages, int* k_exp, int* v_exp, int n_pages, int kv_heads, int page_tokens,
                                 int head_dim, const int* page_table, int64_t table_stride, int target_exp, int rnd, unsigned flags, hif8_stream_t stream)
{
    if (src_dtype != HIF8_F32 && src_dtype != HIF8_BF16 && src_dtype != HIF8_F16) return HIF8_ERR_DTYPE;
    if (rnd != HIF8_RND_TA && rnd != HIF8_RND_HR && rnd != HIF8_RND_SSR && rnd != HIF8_RND_TE) return HIF8_ERR_ROUND;
    if (flags & ~3u) return HIF8_ERR_FLAGS;
    if (target_exp < -22 || target_exp > 15) return HIF8_ERR_SCALE_RANGE;
    if (n_seqs < 0 || n_seqs > HIF8_CACHE_MAX_SEQS || n_new < 0 || token_stride < 0 || head_stride < 0) return HIF8_ERR_SHAPE;
    AppendParams p;
    if (int rc = check_cache(k_pages, v_pages, k_exp, v_exp, n_pages, kv_heads, page_tokens, head_dim, page_table, table_stride, &p.c)) return rc;
    if (n_seqs == 0 || n_new == 0) return HIF8_OK;
    if (!k || !v || !d_new_start || !d_lengths) return HIF8_ERR_NULL;
    const size_t item = dtype_bytes(src_dtype);
    if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & (item - 1) || !ints_aligned(d_new_start, d_lengths)) return HIF8_ERR_ALIGN;
    const size_t src_bytes = ((size_t)(n_new - 1) * (size_t)token_stride + (size_t)(kv_heads - 1) * (size_t)head_stride + (size_t)head_dim) * item;
    const size_t pool = p.c.pool_bytes(), exps = p.c.exp_bytes();
    if (written_over({{k_pages, pool}, {v_pages, pool}, {k_exp, exps}, {v_exp, exps}},
                     {{k, src_bytes}, {v, src_bytes}, {page_table, p.c.table_bytes(n_seqs)}, {d_new_start, (size_t)(n_seqs + 1) * 4}, {d_lengths, (size_t)n_seqs * 4}}))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.src[0] = k; p.src[1] = v; p.token_stride = token_stride; p.head_stride = head_stride; p.start = d_new_start; p.lengths = d_lengths;
    p.n_seqs = n_seqs; p.n_new = n_new; p.target_exp = target_exp; p.flags = flags;
    p.units = piece_numbers(n_new, n_seqs, p.c.shift) * kv_heads * 2;
    p.vectors = aligned_rows(k, v, token_stride, head_stride, item);
    const int mean = (n_new + n_seqs - 1) / n_seqs, tokens = mean < page_tokens ? mean : page_tokens;
    cudaStream_t st = (cudaStream_t)stream;
    switch (rnd) {
        case HIF8_RND_TA: launch_append_of<HIF8_RND_TA>(src_dtype, p, tokens, sms, st); break;
        case HIF8_RND_HR: launch_append_of<HIF8_RND_HR>(src_dtype, p, tokens, sms, st); break;
        case HIF8_RND_SSR: launch_append_of<HIF8_RND_SSR>(src_dtype, p, tokens, sms, st); break;
        default: launch_append_of<HIF8_RND_TE>(src_dtype, p, tokens, sms, st); break;
    }
    return finish_launch(1);
}

extern "C" int hif8_cache_read(const uint8_t* k_pages, const uint8_t* v_pages, const int* k_exp, const int* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim,
                               const int* page_table, int64_t table_stride, const int* d_first, const int* d_out_start, int n_seqs, int n_out, void* k, void* v,
                               int dst_dtype, int64_t token_stride, int64_t head_stride, hif8_stream_t stream)
{
    if (dst_dtype != HIF8_F32 && dst_dtype != HIF8_BF16 && dst_dtype != HIF8_F16) return HIF8_ERR_DTYPE;
    if (n_seqs < 0 || n_seqs > HIF8_CACHE_MAX_SEQS || n_out < 0 || token_stride < 0 || head_stride < 0) return HIF8_ERR_SHAPE;
    ReadParams p;
    if (int rc = check_cache(k_pages, v_pages, k_exp, v_exp, n_pages, kv_heads, page_tokens, head_dim, page_table, table_stride, &p.c)) return rc;
    if (n_seqs == 0 || n_out == 0) return HIF8_OK;
    if (!k || !v || !d_first || !d_out_start) return HIF8_ERR_NULL;
    // rows must not share elements: tokens outermost, or heads
    const int64_t inner = token_stride < head_stride ? token_stride : head_stride, outer = token_stride < head_stride ? head_stride : token_stride;
    const int64_t n_inner = token_stride < head_stride ? n_out : kv_heads, n_outer = token_stride < head_stride ? kv_heads : n_out;
    if ((n_inner > 1 && inner < head_dim) || (n_outer > 1 && outer < (n_inner - 1) * inner + head_dim)) return HIF8_ERR_SHAPE;
    const size_t item = dtype_bytes(dst_dtype);
    if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & (item - 1) || !ints_aligned(d_first, d_out_start)) return HIF8_ERR_ALIGN;
    const size_t dst_bytes = ((size_t)(n_out - 1) * (size_t)token_stride + (size_t)(kv_heads - 1) * (size_t)head_stride + (size_t)head_dim) * item;
    const size_t pool = p.c.pool_bytes(), exps = p.c.exp_bytes();
    if (rows_meet(((intptr_t)v - (intptr_t)k) / (intptr_t)item, token_stride, head_stride, n_out, kv_heads, head_dim)) return HIF8_ERR_OVERLAP;
    for (const void* d : {k, v})
        if (written_over({{d, dst_bytes}}, {{k_pages, pool}, {v_pages, pool}, {k_exp, exps}, {v_exp, exps}, {page_table, p.c.table_bytes(n_seqs)}, {d_first, (size_t)n_seqs * 4},
                                            {d_out_start, (size_t)(n_seqs + 1) * 4}}))
            return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.dst[0] = k; p.dst[1] = v; p.token_stride = token_stride; p.head_stride = head_stride; p.start = d_out_start; p.first = d_first;
    p.n_seqs = n_seqs; p.n_out = n_out;
    p.units = piece_numbers(n_out, n_seqs, p.c.shift) * kv_heads * 2;
    p.vectors = aligned_rows(k, v, token_stride, head_stride, item);
    const long long blocks = (p.units + kThreads / 32 - 1) / (kThreads / 32), most = (long long)sms * 6;  // (six tables fit in an SM's shared memory)
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    cudaStream_t st = (cudaStream_t)stream;
    if (dst_dtype == HIF8_F32) launch_pdl(cache_read_kernel<HIF8_F32>, grid, st, p);
    else if (dst_dtype == HIF8_BF16) launch_pdl(cache_read_kernel<HIF8_BF16>, grid, st, p);
    else launch_pdl(cache_read_kernel<HIF8_F16>, grid, st, p);
    return finish_launch(1);
}

extern "C" int hif8_cache_fork(uint8_t* k_pages, uint8_t* v_pages, int* k_exp, int* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim, const int* page_table,
                               int64_t table_stride, const int* d_lengths, int n_seqs, const int* d_parent, const int* d_new_page, int n_children, int* table_out,
                               int64_t table_out_stride, int* d_lengths_out, hif8_stream_t stream)
{
    if (n_seqs < 0 || n_children < 0 || n_children > HIF8_CACHE_MAX_SEQS || table_out_stride < 1) return HIF8_ERR_SHAPE;
    ForkParams p;
    if (int rc = check_cache(k_pages, v_pages, k_exp, v_exp, n_pages, kv_heads, page_tokens, head_dim, page_table, table_stride, &p.c)) return rc;
    if (n_children == 0) return HIF8_OK;
    if ((n_seqs && !d_lengths) || !d_parent || !table_out || !d_lengths_out) return HIF8_ERR_NULL;
    if (!ints_aligned(d_lengths, d_parent, d_new_page, table_out) || !ints_aligned(d_lengths_out)) return HIF8_ERR_ALIGN;
    const size_t pool = d_new_page ? p.c.pool_bytes() : 0, exps = d_new_page ? p.c.exp_bytes() : 0, each = (size_t)n_children * 4;
    if (written_over({{table_out, each * (size_t)table_out_stride}, {d_lengths_out, each}, {k_pages, pool}, {v_pages, pool}, {k_exp, exps}, {v_exp, exps}},
                     {{page_table, p.c.table_bytes(n_seqs)}, {d_lengths, (size_t)n_seqs * 4}, {d_parent, each}, {d_new_page, d_new_page ? each : 0}}))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.lengths = d_lengths; p.parent = d_parent; p.new_page = d_new_page; p.table_out = table_out; p.out_stride = table_out_stride; p.lengths_out = d_lengths_out;
    p.n_seqs = n_seqs; p.n_children = n_children; p.parts = copy_parts(p.c);
    launch_pdl(cache_fork_kernel, dim3((unsigned)n_children, (unsigned)(d_new_page ? p.parts : 1)), (cudaStream_t)stream, p);
    return finish_launch(1);
}

extern "C" size_t hif8_cache_compact_workspace_bytes(int n_pages)
{
    const size_t n = n_pages > 0 ? (size_t)n_pages : 0;
    return 256 + round_up_256((n + 31) / 32 * 4) + 3 * round_up_256(4 * n);
}

extern "C" int hif8_cache_compact(uint8_t* k_pages, uint8_t* v_pages, int* k_exp, int* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim, int* page_table,
                                  int64_t table_stride, const int* d_lengths, int n_seqs, int move, int* d_n_live, int* d_free_pages, void* workspace,
                                  size_t workspace_bytes, hif8_stream_t stream)
{
    if (n_seqs < 0 || n_seqs > HIF8_CACHE_MAX_SEQS) return HIF8_ERR_SHAPE;
    CompactParams p;
    if (int rc = check_cache(k_pages, v_pages, k_exp, v_exp, n_pages, kv_heads, page_tokens, head_dim, page_table, table_stride, &p.c)) return rc;
    if ((n_seqs && !d_lengths) || !d_n_live || (n_pages && !d_free_pages)) return HIF8_ERR_NULL;
    if (!ints_aligned(d_lengths, d_n_live, d_free_pages)) return HIF8_ERR_ALIGN;
    if (!workspace || workspace_bytes < hif8_cache_compact_workspace_bytes(n_pages) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HIF8_ERR_WORKSPACE;
    const size_t pool = move ? p.c.pool_bytes() : 0, exps = move ? p.c.exp_bytes() : 0, table = p.c.table_bytes(n_seqs), lengths = (size_t)n_seqs * 4;
    if (written_over({{d_n_live, 4}, {d_free_pages, (size_t)n_pages * 4}, {workspace, hif8_cache_compact_workspace_bytes(n_pages)}, {k_pages, pool}, {v_pages, pool}, {k_exp, exps}, {v_exp, exps},
                      {page_table, move ? table : 0}},
                     {{page_table, move ? 0 : table}, {d_lengths, lengths}}))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.table = page_table; p.lengths = d_lengths; p.n_seqs = n_seqs; p.move = move != 0; p.parts = copy_parts(p.c);
    p.words = (n_pages + 31) / 32;
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
    p.counts = reinterpret_cast<int*>(ws); ws += 256;
    p.live = reinterpret_cast<uint32_t*>(ws); ws += round_up_256((size_t)p.words * 4);
    p.to = reinterpret_cast<int*>(ws); ws += round_up_256((size_t)n_pages * 4);
    p.movers = reinterpret_cast<int*>(ws); ws += round_up_256((size_t)n_pages * 4);
    p.holes = reinterpret_cast<int*>(ws);
    p.n_live_out = d_n_live; p.free_out = d_free_pages;
    const long long entries = (long long)n_seqs * table_stride;
    p.mark_here = entries <= kMarkHereEntries && p.words <= kMarkHereWords;
    cudaStream_t st = (cudaStream_t)stream;
    int launches = 1;
    if (!p.mark_here) {
        const unsigned most = (unsigned)sms * 8;
        const unsigned clear_blocks = (unsigned)((p.words + kThreads - 1) / kThreads);
        launch_pdl(cache_clear_kernel, dim3(clear_blocks < 1 ? 1 : clear_blocks < most ? clear_blocks : most), st, p);
        const long long mark_blocks = (entries + kThreads - 1) / kThreads;
        launch_pdl(cache_mark_kernel, dim3(mark_blocks < 1 ? 1 : (unsigned)(mark_blocks < most ? mark_blocks : most)), st, p);
        launches += 2;
    }
    launch_pdl_threads(kRankThreads, cache_rank_kernel, dim3(1), st, p);
    if (p.move) {
        const long long want = (long long)n_pages / 2 * p.parts, most = (long long)sms * 8;  // (no more pages move than stay)
        launch_pdl(cache_move_kernel, dim3(want < 1 ? 1 : (unsigned)(want < most ? want : most)), st, p);
        launches++;
    }
    return finish_launch(launches);
}
