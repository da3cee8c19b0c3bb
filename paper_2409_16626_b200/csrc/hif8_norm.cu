// Root-mean-square norm in front of a block-scaled product, with the residual's addition and HiF8 codes as its result, and its gradient.
//
//   h = x + residual (rounded to their type),  r = 1 / sqrt(mean(h^2) + eps),  y = h r w  ->  codes with a scale for each 1 x 128
//   dx = r (w dy - u mean(w dy u)) + dh,  u = h r;     dw_j = sum_i dy_ij u_ij
//
// Both are bound by memory.  A row is held in registers between its sum and its results (16 to 1024 threads per row, up to 32 elements a
// thread), so every tensor is read or written once.  Sums, the norm's factor and the weight's gradient are FP32.
#include "hif8_block.cuh"
#include "hif8_host_cache.h"

namespace hif8 {
namespace {

constexpr int kNormEights = 4;  // groups of eight elements that a thread holds of a row

struct NormParams {
    const void* x;
    const void* residual;  // or null
    const void* weight;
    void* h;               // or null
    float* rstd;           // or null
    long long ld_x, ld_res, ld_h, rows, cols;
    float eps;
    BlockCodes m;
    int gs, lg;            // threads of a row, and their log2 in blocks of 256
    int target_exp;
    unsigned flags;
    bool late;             // the next launch may start at the end: its blocks sit unevenly when they come under launches of several rounds
};

// How a row is shared out: ALONE, one block to a row, any number `gs` of threads in whole warps; otherwise 1 << lg threads of a block of 256, 16 of them only where HALF.
// Sum over a row's threads, the same bits in each of them; `s_part`: one of two sets of a word per warp, used in turn, so nobody still reads it from the use before the last
// one, which the barrier of the last one stands behind; words of no warp are zero.
template <bool ALONE, bool HALF>
__device__ __forceinline__ float row_sum(float v, float* s_part, int gs, int lg, int group, bool alone)
{
    if (HALF && lg == 4) {
#pragma unroll
        for (int d = 8; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        return v;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if (!ALONE && lg == 5) return v;
    if ((threadIdx.x & 31u) == 0) s_part[threadIdx.x >> 5] = v;
    if (alone) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(1 << lg) : "memory");
    const int n = ALONE ? gs >> 5 : 1 << (lg - 5);
    const float* part = ALONE ? s_part : s_part + (group << (lg - 5));
    if (!ALONE && n == 2) return part[0] + part[1];
    v = 0.f;
    for (int i = 0; i < n; i += 4) {
        const float4 q = *reinterpret_cast<const float4*>(part + i);
        v += (q.x + q.y) + (q.z + q.w);
    }
    return v;
}
// Eights of a row: neighbouring elements of a thread where rows lie on 16-byte boundaries and have whole eights (WHOLE), otherwise spread over a warp (see load_spread)
template <bool WHOLE> __device__ __forceinline__ int first_column(int j, int gs, int t) { return WHOLE ? (j * gs + t) * 8 : (j * gs + (t & ~31)) * 8 + (t & 31); }
template <int DT, bool WHOLE, bool KEEP = false> __device__ __forceinline__ Eight<DT> load_row(const void* row, int c, int end)
{
    if constexpr (WHOLE) return load_eight<DT, KEEP, true>(row, c, end, true);
    else return load_spread<DT, KEEP>(row, c, end);
}
// The same where NOW, with its place among the code's loads: the compiler puts a load that is used behind a barrier behind it, where it has only one (8192 x 8192 BF16 115 -> 100 us).
template <int DT, bool WHOLE, bool NOW> __device__ __forceinline__ Eight<DT> load_row_now(const void* row, int c, int end)
{
    if constexpr (WHOLE && NOW) {
        Eight<DT> e;
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row) + (unsigned)c * (DT == HIF8_F32 ? 4u : 2u));
        const int in = c < end;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(e.v) / 16); i++)
            asm volatile("{ .reg .pred q; setp.ne.s32 q, %5, 0; mov.u32 %0, 0; mov.u32 %1, 0; mov.u32 %2, 0; mov.u32 %3, 0; @q ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4]; }"
                         : "=&r"(e.v[i].x), "=&r"(e.v[i].y), "=&r"(e.v[i].z), "=&r"(e.v[i].w) : "l"(p + i), "r"(in));
        return e;
    } else return load_row<DT, WHOLE>(row, c, end);
}
template <int DT, bool WHOLE> __device__ __forceinline__ void store_row(const char* row, int c, int end, const Eight<DT>& e)
{
    if constexpr (WHOLE) store_eight<DT, true>(const_cast<char*>(row), c, end, true, e);
    else store_spread<DT>(const_cast<char*>(row), c, end, e);
}

template <int DT> __device__ __forceinline__ const char* row_at(const void* base, long long row, long long ld)
{
    return reinterpret_cast<const char*>(base) + (size_t)row * (size_t)ld * (DT == HIF8_F32 ? 4 : 2);
}

// x + residual, rounded once.  (16-bit types packed: the sum in FP32 rounded to them is the same, since a sum that FP32 rounds has one term far below half a step of the other.)
template <int DT> __device__ __forceinline__ uint32_t add_word(uint32_t a, uint32_t b)
{
    uint32_t d;
    if (DT == HIF8_F32) return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    if (DT == HIF8_BF16) asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <int DT> __device__ __forceinline__ Eight<DT> add_eight(const Eight<DT>& a, const Eight<DT>& b)
{
    Eight<DT> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.v) / 16); i++)
        r.v[i] = make_uint4(add_word<DT>(a.v[i].x, b.v[i].x), add_word<DT>(a.v[i].y, b.v[i].y), add_word<DT>(a.v[i].z, b.v[i].z), add_word<DT>(a.v[i].w, b.v[i].w));
    return r;
}

__device__ __forceinline__ uint32_t half_max(uint32_t m)  // of the sixteen threads of a block of 128
{
    const unsigned mask = 0xFFFFu << (threadIdx.x & 16u);
#pragma unroll
    for (int d = 8; d; d >>= 1) m = max(m, __shfl_xor_sync(mask, m, d));
    return m;
}

// Issue slots are what a row costs beside its bytes: columns behind the row's end are zeros already when they are loaded, a block's maximum leaves Inf out only where there is
// one, and the code table is read with the sign.
// WHOLE: every row on a 16-byte boundary (codes: 8), columns a multiple of 8.  NV: eights of a thread; 1 for short rows, of which a block then has more.
constexpr int norm_blocks(int dtype, int block, int nv) { return nv > 1 && dtype == HIF8_F32 ? (block < 512 ? 512 / block : 1) : 1024 / block; }
template <int DT, int MODE, int BLOCK, int NV, bool WHOLE>
__global__ void __launch_bounds__(BLOCK, norm_blocks(DT, BLOCK, NV)) norm_encode_kernel(const NormParams p)
{
    __shared__ SmemTables sm;
    __shared__ __align__(16) float s_part[2][32];
    if (threadIdx.x < 64) s_part[threadIdx.x >> 5][threadIdx.x & 31u] = 0.f;
    setup_tables<true, MODE != HIF8_RND_TA, false, MODE, HIF8_F32, BLOCK == kThreads ? kThreads : kThreads + 1>(sm, p.flags);  // (blocks of more threads may have any number)
    pdl_wait_prior_grid();
    if (!p.late) pdl_launch_dependents();
    constexpr bool kAlone = BLOCK > 256;
    const int gs = kAlone ? p.gs : 1 << p.lg, group = kAlone ? 0 : threadIdx.x >> p.lg, t = kAlone ? threadIdx.x : threadIdx.x & (gs - 1), groups = kAlone ? 1 : BLOCK >> p.lg;
    int turn = 0;
    for (long long row = (long long)blockIdx.x * groups + group; row - group < p.rows; row += (long long)gridDim.x * groups, turn ^= 1) {
        const bool live = row < p.rows;  // a group behind the last row only takes part in the exchanges
        const int end = live ? (int)p.cols : 0;
        Eight<DT> h[NV];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++) h[j] = load_row<DT, WHOLE>(row_at<DT>(p.x, row, p.ld_x), first_column<WHOLE>(j, gs, t), end);
        if (p.residual) {
            Eight<DT> r[NV];
#pragma unroll
            for (int j = 0; j < NV; j++) r[j] = load_row<DT, WHOLE>(row_at<DT>(p.residual, row, p.ld_res), first_column<WHOLE>(j, gs, t), end);
#pragma unroll
            for (int j = 0; j < NV; j++) h[j] = add_eight<DT>(h[j], r[j]);
        }
        if (p.h) {
#pragma unroll
            for (int j = 0; j < NV; j++) store_row<DT, WHOLE>(row_at<DT>(p.h, row, p.ld_h), first_column<WHOLE>(j, gs, t), end, h[j]);
        }
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float v = value_of_eight<DT>(h[j], i);
                sum = fmaf(v, v, sum);
            }
        sum = row_sum<kAlone, NV == 1>(sum, s_part[turn], gs, p.lg, group, kAlone || groups == 1);
        const float rstd = __frsqrt_rn(sum / (float)p.cols + p.eps);
        if (p.rstd && t == 0 && live) p.rstd[row] = rstd;
        uint8_t* codes = p.m.codes + (size_t)row * (size_t)p.m.ld;
        int* exps = p.m.exps + (size_t)row * (size_t)p.m.exp_stride;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = first_column<WHOLE>(j, gs, t);
            if ((WHOLE ? c & ~127 : c - (t & 31)) >= end) continue;  // (WHOLE: the same for a block's sixteen threads, and so is what follows for half a warp; else for a warp)
            const Eight<DT> w = load_row<DT, WHOLE, true>(p.weight, c, (int)p.cols);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = value_of_eight<DT>(h[j], i) * rstd * value_of_eight<DT>(w, i);
            // WHOLE: the eight elements lie in one block, of sixteen threads; else four each in the two blocks of a warp
            float top[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; i++) top[WHOLE ? 0 : i >> 2] = fmaxf(top[WHOLE ? 0 : i >> 2], fabsf(y[i]));  // (a NaN is passed over)
            auto largest = [&](float v) { return WHOLE ? half_max(__float_as_uint(v)) : __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v)); };
            uint32_t m[2] = {largest(top[0]), WHOLE ? 0u : largest(top[1])};
            if (max(m[0], m[1]) >= 0x7F800000u) {
                top[0] = top[1] = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) top[WHOLE ? 0 : i >> 2] = amax_step(top[WHOLE ? 0 : i >> 2], y[i]);
                m[0] = largest(top[0]);
                if (!WHOLE) m[1] = largest(top[1]);
            }
            const int se0 = block_exp_from_amax(m[0], p.target_exp), se1 = WHOLE ? se0 : block_exp_from_amax(m[1], p.target_exp);
            if (WHOLE) {
                if ((t & 15) == 0) exps[c >> 7] = se0;
            } else if ((t & 31) == 0) {
                exps[c >> 7] = se0;
                if (c + 128 < end) exps[(c >> 7) + 1] = se1;
            }
            const float scale0 = pow2f(se0), scale1 = pow2f(se1);
            uint32_t k[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float scale = i < 4 ? scale0 : scale1;
                if (MODE == HIF8_RND_TA) k[i] = sm.ta[__float_as_uint(y[i] * scale) >> 19];
                else k[i] = encode_one<MODE, HIF8_F32>(y[i], __float_as_uint(y[i]), scale, sm.ta, sm.thr, 0u);
            }
            const uint2 word = make_uint2(__byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410),
                                          __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410));
            if (!WHOLE) store_codes_spread(codes, c, end, word);
            else if (c < end) *reinterpret_cast<uint2*>(codes + c) = word;
        }
    }
    if (p.late) pdl_launch_dependents();
}

// ------------------------------------------------------------------------------------------------
// gradient
// ------------------------------------------------------------------------------------------------
struct NormBackwardParams {
    const void* dy;
    const void* h;
    const void* dh;      // or null
    const void* weight;
    const float* rstd;
    void* dx;
    float* part;         // [blocks][cols] shares of the weight's gradient, or null
    long long ld_dy, ld_h, ld_dh, ld_dx, rows, cols;
    int gs, lg;
};

// Its values are unpacked again behind this: kept unpacked over a barrier they take registers that the kernels do not have.
template <int DT> __device__ __forceinline__ void packed_again(Eight<DT>& e)
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(e.v) / 16); i++) asm volatile("" : "+r"(e.v[i].x), "+r"(e.v[i].y), "+r"(e.v[i].z), "+r"(e.v[i].w));
}

// element i of eight FP32 values
__device__ __forceinline__ void set_value(Eight<HIF8_F32>& e, int i, float v)
{
    uint4& q = e.v[i >> 2];
    ((i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w) = __float_as_uint(v);
}

// A thread has the same columns of every row it works on, so it keeps their sums of dy u: in registers (NV up to 2), of rows beyond 16384 columns (NV = 4, 1024 threads with 64
// registers each) in shared memory.
template <int DT, int BLOCK, int NV, bool WHOLE>
__global__ void __launch_bounds__(BLOCK, 1024 / BLOCK) norm_backward_kernel(const NormBackwardParams p)
{
    constexpr bool kFar = NV > 2;
    extern __shared__ __align__(16) float s_acc[];  // BLOCK x 8 NV: kFar: the threads' sums; blocks of 256: to join their groups
    constexpr bool kLate = DT == HIF8_F32 && NV > 1;  // dh is loaded behind the mean: no registers for it in front
    constexpr bool kInPlace = DT == HIF8_F32 && !kFar;  // w dy and u in the places of dy and h over the mean (8192 x 8192 197 -> 185 us; of 32768 columns 309 and 329)
    __shared__ __align__(16) float s_part[2][BLOCK / 32];
    if (BLOCK > 256) {
        if (threadIdx.x < BLOCK / 16) s_part[0][threadIdx.x] = 0.f;
        __syncthreads();
    }
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    constexpr bool kAlone = BLOCK > 256;
    const int gs = kAlone ? p.gs : 1 << p.lg, group = kAlone ? 0 : threadIdx.x >> p.lg, t = kAlone ? threadIdx.x : threadIdx.x & (gs - 1), groups = kAlone ? 1 : BLOCK >> p.lg;
    float acc[kFar ? 1 : NV][8];
    if (!kFar) {
#pragma unroll
        for (int j = 0; j < (kFar ? 1 : NV); j++)
#pragma unroll
            for (int i = 0; i < 8; i++) acc[j][i] = 0.f;
    } else {
        for (int k = 0; k < NV * 8; k++) s_acc[k * BLOCK + threadIdx.x] = 0.f;
    }
    const float inv = 1.f / (float)p.cols;
    int turn = 0;
    for (long long row = (long long)blockIdx.x * groups + group; row - group < p.rows; row += (long long)gridDim.x * groups, turn ^= 1) {
        const bool live = row < p.rows;
        const int end = live ? (int)p.cols : 0;
        Eight<DT> dy[NV], h[NV], dh[NV];
#pragma unroll
        for (int j = 0; j < NV; j++) dy[j] = load_row_now<DT, WHOLE, kAlone>(row_at<DT>(p.dy, row, p.ld_dy), first_column<WHOLE>(j, gs, t), end);
#pragma unroll
        for (int j = 0; j < NV; j++) h[j] = load_row_now<DT, WHOLE, kAlone>(row_at<DT>(p.h, row, p.ld_h), first_column<WHOLE>(j, gs, t), end);
        const float rstd = live ? __ldg(p.rstd + row) : 0.f;
        if (!kLate && p.dh) {
#pragma unroll
            for (int j = 0; j < NV; j++) dh[j] = load_row_now<DT, WHOLE, kAlone>(row_at<DT>(p.dh, row, p.ld_dh), first_column<WHOLE>(j, gs, t), end);
        } else {
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int i = 0; i < (int)(sizeof(dh[j].v) / 16); i++) dh[j].v[i] = make_uint4(0, 0, 0, 0);
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const Eight<DT> w = load_row<DT, WHOLE, true>(p.weight, first_column<WHOLE>(j, gs, t), (int)p.cols);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                // (u first: near 1 whatever h is, where dy h and dy r might leave FP32)
                const float d = value_of_eight<DT>(dy[j], i), u = value_of_eight<DT>(h[j], i) * rstd;
                const float wdy = d * value_of_eight<DT>(w, i);
                sum = fmaf(wdy, u, sum);
                if constexpr (kInPlace) {
                    set_value(h[j], i, u);
                    set_value(dy[j], i, wdy);
                }
                if (!kFar) acc[j % (kFar ? 1 : NV)][i] = fmaf(d, u, acc[j % (kFar ? 1 : NV)][i]);
                else s_acc[(j * 8 + i) * BLOCK + threadIdx.x] = fmaf(d, u, s_acc[(j * 8 + i) * BLOCK + threadIdx.x]);
            }
        }
        const float mean = row_sum<kAlone, NV == 1>(sum, s_part[turn], gs, p.lg, group, kAlone || groups == 1) * inv, factor = kInPlace ? -mean : -rstd * mean;
        const void* weight = p.weight;
        asm volatile("" : "+l"(weight));
#pragma unroll
        for (int j = 0; j < NV; j++) {
            packed_again<DT>(dy[j]);
            packed_again<DT>(h[j]);
            if (kLate && p.dh) dh[j] = load_row_now<DT, WHOLE, kAlone>(row_at<DT>(p.dh, row, p.ld_dh), first_column<WHOLE>(j, gs, t), end);
            Eight<DT> w;
            if (!kInPlace) w = load_row<DT, WHOLE, true>(weight, first_column<WHOLE>(j, gs, t), (int)p.cols);
            float g[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {  // r (w dy - u mean) + dh
                const float wdy = kInPlace ? value_of_eight<DT>(dy[j], i) : value_of_eight<DT>(dy[j], i) * value_of_eight<DT>(w, i);
                g[i] = fmaf(rstd, fmaf(factor, value_of_eight<DT>(h[j], i), wdy), value_of_eight<DT>(dh[j], i));
            }
            store_row<DT, WHOLE>(row_at<DT>(p.dx, row, p.ld_dx), first_column<WHOLE>(j, gs, t), end, pack_eight<DT>(g));
        }
    }
    if (!p.part) return;
    float* out = p.part + (size_t)blockIdx.x * (size_t)p.cols;
    if (kFar) {
        for (int k = 0; k < NV * 8; k++) {
            const int c = first_column<WHOLE>(k >> 3, gs, t) + (k & 7) * (WHOLE ? 1 : 32);
            if (c < p.cols) out[c] = s_acc[k * BLOCK + threadIdx.x];
        }
        return;
    }
    if (groups == 1) {
#pragma unroll
        for (int j = 0; j < (kFar ? 1 : NV); j++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int c = first_column<WHOLE>(j, gs, t) + i * (WHOLE ? 1 : 32);
                if (c < p.cols) out[c] = acc[j][i];
            }
        return;
    }
    // the groups' sums, in their order
    const int width = gs * NV * 8;
#pragma unroll
    for (int j = 0; j < (kFar ? 1 : NV); j++)
#pragma unroll
        for (int i = 0; i < 8; i += WHOLE ? 4 : 1) {
            float* to = s_acc + group * width + first_column<WHOLE>(j, gs, t) + i * (WHOLE ? 1 : 32);
            if (WHOLE) *reinterpret_cast<float4*>(to) = make_float4(acc[j][i], acc[j][i + 1], acc[j][i + 2], acc[j][i + 3]);
            else *to = acc[j][i];
        }
    __syncthreads();
    for (int c = threadIdx.x; c < width && c < p.cols; c += BLOCK) {
        float v = 0.f;
        for (int g = 0; g < groups; g++) v += s_acc[g * width + c];
        out[c] = v;
    }
}

// dweight_j (+)= the blocks' shares, in their order: 32 columns by 32 slices of the blocks
constexpr int kShareThreads = 1024;
__global__ void __launch_bounds__(kShareThreads) norm_weight_grad_kernel(const float* __restrict__ part, int blocks, long long cols, float* dweight, int accumulate)
{
    __shared__ float s_sum[32][33];
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, per = (blocks + 31) / 32;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < cols) {
        const int from = slice * per, to = min(blocks, from + per);
#pragma unroll 8
        for (int b = from; b < to; b++) v += part[(size_t)b * (size_t)cols + c];
    }
    s_sum[slice][lane] = v;
    __syncthreads();
    v = s_sum[lane][slice];  // a warp adds a column's 32 sums
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const long long own = (long long)blockIdx.x * 32 + slice;
    if (lane == 0 && own < cols) dweight[own] = accumulate ? dweight[own] + v : v;
}

int finish(int launches)
{
    g_launches.fetch_add((uint64_t)launches, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}

// How rows are shared out: nv eights a thread, 1 where a row is short, `most` where it is not; one block to a row of more than 256 threads, as many warps as it takes.
struct RowPlan {
    int nv, gs, lg, groups, threads;  // threads: of a block
    RowPlan(long long cols, int most, bool whole, bool alone)
    {
        const long long eights = (cols + 7) / 8;
        // (alone: few rows, whose time is that of one; 64 threads or fewer of a row do without the other eights' instructions: 524288 x 128 BF16, norm 295 -> 104 us,
        // its gradient 226 -> 105)
        nv = (alone && eights <= 1024) || eights <= 64 ? 1 : most;
        const long long want = (eights + nv - 1) / nv;
        lg = whole && nv == 1 ? 4 : 5;
        while ((1ll << lg) < want && lg < 8) lg++;
        gs = 1 << lg;
        if (gs < want) gs = (int)((want + 31) / 32 * 32);
        if (gs > 256) {
            groups = 1; threads = gs;
        } else {
            groups = 256 / gs; threads = 256;
        }
    }
};
constexpr int kFewRows = 148;

// The gradient's kernel: as many blocks as are resident.  (FP32 of up to 4096 columns, eight elements a thread: 16384 x 4096 181 -> 171 us, 65536 x 1024 170 -> 165.)
RowPlan backward_plan(long long cols, int dtype, bool whole) { return RowPlan(cols, dtype == HIF8_F32 && cols <= 4096 ? 1 : cols <= 16384 ? 2 : 4, whole, false); }
long long backward_blocks(long long rows, const RowPlan& plan)
{
    const long long need = (rows + plan.groups - 1) / plan.groups, most = 148ll * (1024 / plan.threads);
    return need < most ? need : most;
}
// of any type and alignment, which the shares of the weight's gradient in the workspace go by
long long backward_most(long long rows, long long cols)
{
    long long most = 0;
    for (int dtype : {HIF8_F32, HIF8_BF16})
        for (bool whole : {false, true}) {
            const long long blocks = backward_blocks(rows, backward_plan(cols, dtype, whole));
            if (blocks > most) most = blocks;
        }
    return most;
}

template <int DT, int MODE, bool WHOLE>
void launch_norm(NormParams p, int sms, cudaStream_t st)
{
    const RowPlan plan(p.cols, kNormEights, WHOLE, p.rows <= kFewRows);
    p.gs = plan.gs; p.lg = plan.lg;
    const int block = plan.threads <= 256 ? 256 : plan.threads <= 512 ? 512 : 1024;
    const long long need = (p.rows + plan.groups - 1) / plan.groups, most = (long long)sms * (norm_blocks(DT, block, plan.nv) * block / plan.threads);
    const dim3 grid((unsigned)(need < most ? need : most));
    p.late = need > most;
    if (plan.nv == 1) {
        if (block == 256) launch_pdl_threads(256, norm_encode_kernel<DT, MODE, 256, 1, WHOLE>, grid, st, p);
        else launch_pdl_threads(plan.threads, norm_encode_kernel<DT, MODE, 1024, kNormEights, WHOLE>, grid, st, p);
    } else if (block == 256) launch_pdl_threads(256, norm_encode_kernel<DT, MODE, 256, kNormEights, WHOLE>, grid, st, p);
    else if (block == 512) launch_pdl_threads(plan.threads, norm_encode_kernel<DT, MODE, 512, kNormEights, WHOLE>, grid, st, p);
    else launch_pdl_threads(plan.threads, norm_encode_kernel<DT, MODE, 1024, kNormEights, WHOLE>, grid, st, p);
}
template <int DT, int MODE>
void launch_norm(const NormParams& p, bool whole, int sms, cudaStream_t st)
{
    if (whole) launch_norm<DT, MODE, true>(p, sms, st);
    else launch_norm<DT, MODE, false>(p, sms, st);
}
template <int DT>
void launch_norm_mode(int rnd, const NormParams& p, bool whole, int sms, cudaStream_t st)
{
    switch (rnd) {
        case HIF8_RND_TA: return launch_norm<DT, HIF8_RND_TA>(p, whole, sms, st);
        case HIF8_RND_HR: return launch_norm<DT, HIF8_RND_HR>(p, whole, sms, st);
        case HIF8_RND_SSR: return launch_norm<DT, HIF8_RND_SSR>(p, whole, sms, st);
        default: return launch_norm<DT, HIF8_RND_TE>(p, whole, sms, st);
    }
}

template <int DT, int BLOCK, int NV, bool WHOLE>
bool launch_backward_block(const NormBackwardParams& p, int threads, long long blocks, cudaStream_t st)
{
    const size_t bytes = BLOCK == 256 || NV > 2 ? (size_t)BLOCK * NV * 8 * sizeof(float) : 0;
    if (bytes > 48 * 1024) {  // a fact of the device, set by its first such call
        static PerDevice<cudaError_t> ready;
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess) return false;
        const cudaError_t* rc = ready.get(dev, [&](int, cudaError_t* out) {
            *out = cudaFuncSetAttribute(norm_backward_kernel<DT, BLOCK, NV, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        });
        if (!rc || *rc != cudaSuccess) return false;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, norm_backward_kernel<DT, BLOCK, NV, WHOLE>, p) == cudaSuccess;
}
template <int DT, bool WHOLE>
bool launch_backward(NormBackwardParams p, long long blocks, cudaStream_t st)
{
    const RowPlan plan = backward_plan(p.cols, DT, WHOLE);
    p.gs = plan.gs; p.lg = plan.lg;
    if (plan.threads <= 256) {
        if (plan.nv == 1) return launch_backward_block<DT, 256, 1, WHOLE>(p, 256, blocks, st);
        if constexpr (DT != HIF8_F32) return launch_backward_block<DT, 256, 2, WHOLE>(p, 256, blocks, st);
    }
    if (plan.threads <= 512) {
        if constexpr (DT == HIF8_F32)
            if (plan.nv == 1) return launch_backward_block<DT, 512, 1, WHOLE>(p, plan.threads, blocks, st);
        return launch_backward_block<DT, 512, 2, WHOLE>(p, plan.threads, blocks, st);
    }
    return plan.nv == 2 ? launch_backward_block<DT, 1024, 2, WHOLE>(p, plan.threads, blocks, st) : launch_backward_block<DT, 1024, 4, WHOLE>(p, plan.threads, blocks, st);
}
template <int DT>
bool launch_backward(const NormBackwardParams& p, bool whole, long long blocks, cudaStream_t st)
{
    return whole ? launch_backward<DT, true>(p, blocks, st) : launch_backward<DT, false>(p, blocks, st);
}

// the same rows (a result in the place of an operand), or no byte in common
bool same_or_apart(const void* dst, size_t dst_bytes, long long ld_dst, const void* src, size_t src_bytes, long long ld_src, long long rows)
{
    return (dst == src && (ld_dst == ld_src || rows <= 1)) || !ranges_overlap(dst, dst_bytes, src, src_bytes);
}

}  // namespace
}  // namespace hif8

using namespace hif8;

extern "C" int hif8_rmsnorm_encode(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int dtype, const void* weight, float eps, int64_t rows, int64_t cols,
                                   void* h, int64_t ld_h, float* d_rstd, uint8_t* dst, int64_t ld_dst, int* d_exp, int64_t exp_stride, int target_exp, int rnd, unsigned flags,
                                   hif8_stream_t stream)
{
    if (bad_dtype(dtype)) return HIF8_ERR_DTYPE;
    if (rnd != HIF8_RND_TA && rnd != HIF8_RND_HR && rnd != HIF8_RND_SSR && rnd != HIF8_RND_TE) return HIF8_ERR_ROUND;
    if (flags & ~(unsigned)(HIF8_FLAG_SATURATE | HIF8_FLAG_NAN_TO_ZERO)) return HIF8_ERR_FLAGS;
    if (target_exp < -22 || target_exp > 15 || !(eps >= 0.f && eps <= 3.402823466e38f)) return HIF8_ERR_SCALE_RANGE;
    if (rows < 0 || cols < 0 || cols > HIF8_NORM_MAX_COLS || rows > 0x7FFFFFFFll * 32) return HIF8_ERR_SHAPE;
    NormParams p{};
    p.m = BlockCodes{dst, ld_dst, d_exp, exp_stride, rows, cols, 0};
    if (ld_x < cols || (residual && ld_residual < cols) || (h && ld_h < cols) || ld_dst < cols || exp_stride < p.m.blocks_across()) return HIF8_ERR_SHAPE;
    if (rows == 0 || cols == 0) return HIF8_OK;
    if (!x || !weight || !dst || !d_exp) return HIF8_ERR_NULL;
    const size_t item = dtype_bytes(dtype);
    if (!aligned_to(x, item) || !aligned_to(residual, item) || !aligned_to(weight, item) || !aligned_to(h, item) || !aligned_to(d_rstd, 4) || !aligned_to(d_exp, 4)) return HIF8_ERR_ALIGN;
    const size_t x_bytes = matrix_bytes(rows, cols, ld_x, item), r_bytes = residual ? matrix_bytes(rows, cols, ld_residual, item) : 0, h_bytes = h ? matrix_bytes(rows, cols, ld_h, item) : 0;
    const size_t w_bytes = (size_t)cols * item, rstd_bytes = d_rstd ? (size_t)rows * 4 : 0;
    if (written_over({{dst, p.m.code_bytes()}, {d_exp, p.m.exp_bytes()}, {d_rstd, rstd_bytes}}, {{x, x_bytes}, {residual, r_bytes}, {weight, w_bytes}, {h, h_bytes}}) ||
        written_over({{h, h_bytes}}, {{weight, w_bytes}}) || !same_or_apart(h, h_bytes, ld_h, x, x_bytes, ld_x, rows) ||
        !same_or_apart(h, h_bytes, ld_h, residual, r_bytes, ld_residual, rows))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.x = x; p.residual = residual; p.weight = weight; p.h = h; p.rstd = d_rstd; p.ld_x = ld_x; p.ld_res = ld_residual; p.ld_h = ld_h; p.rows = rows; p.cols = cols;
    p.eps = eps; p.target_exp = target_exp; p.flags = flags;
    // every row on a 16-byte boundary (codes: 8)
    const bool whole = (cols & 7) == 0 && vector_rows(x, rows, ld_x, item) && aligned_to(weight, 16) && aligned_to(dst, 8) && (rows <= 1 || (ld_dst & 7) == 0) &&
                       (!residual || vector_rows(residual, rows, ld_residual, item)) && (!h || vector_rows(h, rows, ld_h, item));
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == HIF8_F32) launch_norm_mode<HIF8_F32>(rnd, p, whole, sms, st);
    else if (dtype == HIF8_BF16) launch_norm_mode<HIF8_BF16>(rnd, p, whole, sms, st);
    else launch_norm_mode<HIF8_F16>(rnd, p, whole, sms, st);
    return finish(1);
}

extern "C" size_t hif8_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || cols > HIF8_NORM_MAX_COLS) return 0;
    return ((size_t)backward_most(rows, cols) * (size_t)cols * sizeof(float) + 255) & ~(size_t)255;
}

extern "C" int hif8_rmsnorm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* dh, int64_t ld_dh, int dtype, const void* weight, const float* d_rstd,
                                     int64_t rows, int64_t cols, void* dx, int64_t ld_dx, float* d_weight_grad, int accumulate, void* workspace, size_t workspace_bytes,
                                     hif8_stream_t stream)
{
    if (bad_dtype(dtype)) return HIF8_ERR_DTYPE;
    if (rows < 0 || cols < 0 || cols > HIF8_NORM_MAX_COLS || rows > 0x7FFFFFFFll * 32) return HIF8_ERR_SHAPE;
    if (ld_dy < cols || ld_h < cols || (dh && ld_dh < cols) || ld_dx < cols) return HIF8_ERR_SHAPE;
    if (cols == 0) return HIF8_OK;
    cudaStream_t st = (cudaStream_t)stream;
    if (!aligned_to(d_weight_grad, 4)) return HIF8_ERR_ALIGN;
    if (rows == 0) {  // no row: a gradient of zeros
        if (d_weight_grad && !accumulate && cudaMemsetAsync(d_weight_grad, 0, (size_t)cols * 4, st) != cudaSuccess) return HIF8_ERR_CUDA;
        return HIF8_OK;
    }
    if (!dy || !h || !weight || !d_rstd || !dx) return HIF8_ERR_NULL;
    const size_t item = dtype_bytes(dtype);
    if (!aligned_to(dy, item) || !aligned_to(h, item) || !aligned_to(dh, item) || !aligned_to(weight, item) || !aligned_to(dx, item) || !aligned_to(d_rstd, 4)) return HIF8_ERR_ALIGN;
    NormBackwardParams p{};
    const size_t need = d_weight_grad ? hif8_rmsnorm_backward_workspace_bytes(rows, cols) : 0;
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 256))) return HIF8_ERR_WORKSPACE;
    const size_t dy_bytes = matrix_bytes(rows, cols, ld_dy, item), h_bytes = matrix_bytes(rows, cols, ld_h, item), dh_bytes = dh ? matrix_bytes(rows, cols, ld_dh, item) : 0;
    const size_t dx_bytes = matrix_bytes(rows, cols, ld_dx, item), w_bytes = (size_t)cols * item, dw_bytes = d_weight_grad ? (size_t)cols * 4 : 0;
    if (written_over({{d_weight_grad, dw_bytes}, {workspace, need}},
                     {{dy, dy_bytes}, {h, h_bytes}, {dh, dh_bytes}, {weight, w_bytes}, {d_rstd, (size_t)rows * 4}, {dx, dx_bytes}}) ||
        written_over({{dx, dx_bytes}}, {{h, h_bytes}, {weight, w_bytes}, {d_rstd, (size_t)rows * 4}}) || !same_or_apart(dx, dx_bytes, ld_dx, dy, dy_bytes, ld_dy, rows) ||
        !same_or_apart(dx, dx_bytes, ld_dx, dh, dh_bytes, ld_dh, rows))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    p.dy = dy; p.h = h; p.dh = dh; p.weight = weight; p.rstd = d_rstd; p.dx = dx; p.part = d_weight_grad ? reinterpret_cast<float*>(workspace) : nullptr;
    p.ld_dy = ld_dy; p.ld_h = ld_h; p.ld_dh = ld_dh; p.ld_dx = ld_dx; p.rows = rows; p.cols = cols;
    const bool whole = (cols & 7) == 0 && vector_rows(dy, rows, ld_dy, item) && vector_rows(h, rows, ld_h, item) && vector_rows(dx, rows, ld_dx, item) && aligned_to(weight, 16) &&
                       (!dh || vector_rows(dh, rows, ld_dh, item));
    const long long blocks = backward_blocks(rows, backward_plan(cols, dtype, whole));
    const bool ok = dtype == HIF8_F32 ? launch_backward<HIF8_F32>(p, whole, blocks, st) : dtype == HIF8_BF16 ? launch_backward<HIF8_BF16>(p, whole, blocks, st) : launch_backward<HIF8_F16>(p, whole, blocks, st);
    if (!ok) return HIF8_ERR_CUDA;
    if (p.part)
        launch_pdl_threads(kShareThreads, norm_weight_grad_kernel, dim3((unsigned)((cols + 31) / 32)), st, reinterpret_cast<const float*>(workspace), (int)blocks, (long long)cols, d_weight_grad, accumulate);
    return finish(p.part ? 2 : 1);
}
