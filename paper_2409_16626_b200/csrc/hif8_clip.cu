// The global norm of many gradients, and clipping: what stands between the backward pass under a loss scale of 2^s and the optimizer's step.
//
//   norm = sqrt(sum g^2) 2^-s,   out = g 2^-s min(1, max_norm / norm)
//
// Two launches: sums of squares, a share of the list to a block, and the scaling, in front of which every block adds the shares up in the same order. Both are bound by
// memory.  A share is a stretch of the list of all elements, in which each tensor takes kTensorCost places more than it has elements, for what it costs to come to one: so
// neither many small tensors nor few large ones leave blocks idle.  A block fetches the descriptors of its tensors together, works on long pieces with all threads and on short ones
// with a warp each.  (Tensors one after the other, each with its descriptor's latency: 3000 tensors of 10 elements 362 us, 11.5; 2.7 M elements in 28 matrices and 9 vectors
// 21.5 us, 11.8.)  Squares are added in FP32 over 16 bytes and in FP64 from there on (vectors whose sum leaves FP32's comfortable range: in FP64 altogether): the
// norm is within 5 * 2^-24 of the exact one, and the squares of finite gradients do not overflow.  (FP64 from the first square on would take a conversion and an FP64 multiply-add
// for each element.)
#include "hif8_block.cuh"

namespace hif8 {
namespace {

constexpr int kClipBlocks = 1024;   // shares at most
// Blocks an SM, and words of 32 bytes that a thread has in flight: sums of squares, results.  (436000000 BF16 elements: so 403 us; 4, 2 and 2 440, which spilled; 2, 8 and 4 411;
// 2, 4 and 3 412; 2, 6 and 2 408.  20000000 16.9 and 18.9, 1000 5.6 and 6.4.)
constexpr int kClipPerSM = 2;
constexpr int kSquaresUnroll = 6, kScaleUnroll = 3;
constexpr long long kTensorCost = 1024, kShare = 2048;  // (a share's least length)
constexpr int kKeepWords = 7168;    // of a piece's end stay in L2 for the second launch, which begins there: 68 MB over the blocks
constexpr long long kLongPiece = 2048;                  // from so many elements on a piece is the whole block's

struct ClipParams {
    const uint64_t* src;
    const uint64_t* dst;
    const int* dtypes;
    const int64_t* start;
    int tensors;
    long long total, cost, per;   // elements; places of the list; places of a block's share
    const int* scale_exp;
    float max_norm;
    float* norm_out;
    int* found;
    double* part;
    int parts;
};

// Elements lo .. hi - 1 of a tensor (shares start on multiples of sixteen within it)
struct Piece16 {
    uint64_t src, dst;
    long long lo, hi;
    int dtype;
};

__device__ __forceinline__ long long start_of(const ClipParams& p, int t) { return max(0ll, min((long long)p.start[t], p.total)); }
__device__ __forceinline__ long long place_of(const ClipParams& p, int t) { return start_of(p, t) + kTensorCost * t; }

// the last tensor whose places start at or in front of `at` (a warp together, one probe a lane and round)
__device__ __forceinline__ int find_tensor(const ClipParams& p, long long at)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = p.tensors;
    while (n > 1) {
        const int step = (n + 31) >> 5, i = lo + lane * step;
        const bool below = lane * step < n && (lane == 0 || place_of(p, i) <= at);
        const int last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, below));
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}

// What of tensor t lies at the places from .. to - 1; false if its places start behind them
__device__ __forceinline__ bool piece_of(const ClipParams& p, int t, long long from, long long to, Piece16& s)
{
    if (t >= p.tensors) return false;
    const long long b = start_of(p, t), e = start_of(p, t + 1), n = max(0ll, e - b), first = b + kTensorCost * (t + 1);  // place of its first element
    s.src = p.src[t];
    s.dst = p.dst ? p.dst[t] : s.src;
    s.dtype = p.dtypes[t];
    s.lo = from <= first ? 0 : min(n, (from - first + 15) & ~15ll);
    s.hi = to <= first ? 0 : min(n, (to - first + 15) & ~15ll);
    if (!s.src || !s.dst || ((s.src | s.dst) & (s.dtype == HIF8_F32 ? 3u : 1u))) s.hi = s.lo;  // (no address of such elements: left out)
    return b + kTensorCost * t < to;
}

// f(piece, thread, threads) for the pieces of this block's share; first: find_tensor of its beginning
template <class F>
__device__ __forceinline__ void for_pieces(const ClipParams& p, long long from, long long to, int first, F&& f)
{
    __shared__ Piece16 s_piece[kThreads];
    for (int batch = first; batch < p.tensors; batch += kThreads) {
        Piece16 mine{};
        const bool in = piece_of(p, batch + (int)threadIdx.x, from, to, mine);
        if (!in) mine.hi = mine.lo;  // (starts that are in no order: nothing)
        s_piece[threadIdx.x] = mine;
        const int n = __syncthreads_count(in);  // (starts are in order: those in the share come first)
        const int warp = threadIdx.x >> 5;
#pragma unroll 1
        for (int i = 0; i < n + (kThreads / 32) * ((n + kThreads / 32 - 1) / (kThreads / 32)); i += i < n ? 1 : kThreads / 32) {  // long ones, then a warp's short ones
            const bool alone = i >= n;
            const int k = alone ? i - n + warp : i;
            if (k >= n) continue;
            const Piece16 s = s_piece[k];
            if ((s.hi - s.lo < kLongPiece) != alone) continue;
            f(s, alone ? (int)(threadIdx.x & 31u) : (int)threadIdx.x, alone ? 32 : kThreads);
        }
        if (n < kThreads) break;
        __syncthreads();
    }
}

// 32 bytes; `whole`: on a boundary of that many, and not of 16 only.  GONE: not to be kept in L2.  What the first launch reads in front of a piece's end and what the second one
// writes is not: 436000000 BF16 elements 454 -> 440 us, 20000000 20.3 -> 19.0 (with four blocks an SM; 40 to 130 MB kept: 441 to 443).
template <bool GONE> __device__ __forceinline__ void load_32(const void* from, uint4& a, uint4& b, bool whole)
{
    if (!whole) {
        a = reinterpret_cast<const uint4*>(from)[0];
        b = reinterpret_cast<const uint4*>(from)[1];
    } else if (GONE)
        asm volatile("ld.global.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(from));
    else
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(from));
}
__device__ __forceinline__ void store_32(void* to, const uint4& a, const uint4& b, bool whole)
{
    if (!whole) {
        reinterpret_cast<uint4*>(to)[0] = a;
        reinterpret_cast<uint4*>(to)[1] = b;
    } else
        asm volatile("st.global.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(to), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}

template <int DT> __device__ __forceinline__ double squares(const uint4& v)
{
    constexpr int PV = SrcTraits<DT>::kPerVec;
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < PV; k++) {
        float x; uint32_t raw;
        unpack<DT>(v, k, x, raw);
        q = fmaf(x, x, q);
    }
    if (q >= 8.673617379884035e-19f && q <= 1.329227995784916e36f) return (double)q;  // 2^-60 .. 2^120
    const uint32_t magnitude = DT == HIF8_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu;
    if (((v.x | v.y | v.z | v.w) & magnitude) == 0) return 0.0;
    double d = 0.0;
#pragma unroll 1
    for (int k = 0; k < PV; k++) {
        const uint32_t w = (k * 4 / PV) == 0 ? v.x : (k * 4 / PV) == 1 ? v.y : (k * 4 / PV) == 2 ? v.z : v.w;
        const uint32_t raw = DT == HIF8_F32 ? w : ((k & 1) ? w >> 16 : w & 0xFFFFu);
        const double x = DT == HIF8_F32 ? (double)__uint_as_float(raw) : DT == HIF8_BF16 ? (double)__uint_as_float(raw << 16) : (double)__half2float(__ushort_as_half((unsigned short)raw));
        d = fma(x, x, d);
    }
    return d;
}

template <int DT> __device__ __forceinline__ double piece_squares(const Piece16& s, int thread, int threads)
{
    constexpr int PW = 2 * SrcTraits<DT>::kPerVec;  // elements of 32 bytes
    double sum = 0.0;
    long long tail = s.lo;
    if ((s.src & 15u) == 0) {
        const bool whole = (s.src & 16u) == 0;
        const char* from = reinterpret_cast<const char*>(s.src);
        const long long end = s.hi / PW;
        for (long long base = s.lo / PW + thread; base < end; base += threads * kSquaresUnroll) {
            uint4 v[kSquaresUnroll][2];
#pragma unroll
            for (int j = 0; j < kSquaresUnroll; j++) {
                v[j][0] = v[j][1] = make_uint4(0, 0, 0, 0);
                if (base + j * threads >= end) continue;
                if (base < end - kKeepWords) load_32<true>(from + (base + j * threads) * 32, v[j][0], v[j][1], whole);
                else load_32<false>(from + (base + j * threads) * 32, v[j][0], v[j][1], whole);
            }
#pragma unroll
            for (int j = 0; j < kSquaresUnroll; j++) sum += squares<DT>(v[j][0]) + squares<DT>(v[j][1]);
        }
        tail = max(s.lo, end * PW);
    }
#pragma unroll 1
    for (long long i = tail + thread; i < s.hi; i += threads) {
        float x; uint32_t raw;
        load_scalar<DT>(reinterpret_cast<const void*>(s.src), (unsigned long long)i, x, raw);
        sum = fma((double)x, (double)x, sum);
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double v, double* s_part)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; w++) v += s_part[w];
    return v;
}

__global__ void __launch_bounds__(kThreads, kClipPerSM) grad_squares_kernel(const ClipParams p)
{
    __shared__ double s_part[kThreads / 32];
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const long long from = (long long)blockIdx.x * p.per, to = min(p.cost, from + p.per);
    double sum = 0.0;
    if (from < to)
        for_pieces(p, from, to, find_tensor(p, from), [&](const Piece16& s, int thread, int threads) {
            if (s.dtype == HIF8_F32) sum += piece_squares<HIF8_F32>(s, thread, threads);
            else if (s.dtype == HIF8_BF16) sum += piece_squares<HIF8_BF16>(s, thread, threads);
            else if (s.dtype == HIF8_F16) sum += piece_squares<HIF8_F16>(s, thread, threads);
        });
    sum = block_sum(sum, s_part);
    if (threadIdx.x == 0) p.part[blockIdx.x] = sum;
}

// x f p, p a power of two that is 1 unless f p is no normal FP32: one rounding to FP32 (below 2^-126, and only then, a second); a 16-bit tensor's type is the next
struct Factor {
    float f, p;
    __device__ __forceinline__ float of(float x) const { return x * f * p; }
};

template <int DT> __device__ __forceinline__ uint4 scaled(const uint4& v, const Factor& f)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if (DT == HIF8_F32) w[k] = __float_as_uint(f.of(__uint_as_float(w[k])));
        else if (DT == HIF8_BF16) {
            const float lo = f.of(__uint_as_float(w[k] << 16)), hi = f.of(__uint_as_float(w[k] & 0xFFFF0000u));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(hi), "f"(lo));
        } else {
            const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(f.of(x.y)), "f"(f.of(x.x)));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// (from its end, which the first launch read last)
template <int DT> __device__ __forceinline__ void scale_piece(const Piece16& s, const Factor& f, int thread, int threads)
{
    constexpr int PW = 2 * SrcTraits<DT>::kPerVec;
    long long tail = s.lo;
    if (((s.src | s.dst) & 15u) == 0) {
        const bool whole = ((s.src | s.dst) & 16u) == 0;
        const char* from = reinterpret_cast<const char*>(s.src);
        char* to = reinterpret_cast<char*>(s.dst);
        const long long first = s.lo / PW, end = s.hi / PW;
        for (long long base = end - 1 - thread; base >= first; base -= threads * kScaleUnroll) {
            uint4 v[kScaleUnroll][2];
#pragma unroll
            for (int j = 0; j < kScaleUnroll; j++)
                if (base - j * threads >= first) load_32<false>(from + (base - j * threads) * 32, v[j][0], v[j][1], whole);
#pragma unroll
            for (int j = 0; j < kScaleUnroll; j++)
                if (base - j * threads >= first) store_32(to + (base - j * threads) * 32, scaled<DT>(v[j][0], f), scaled<DT>(v[j][1], f), whole);
        }
        tail = max(s.lo, end * PW);
    }
#pragma unroll 1
    for (long long i = tail + thread; i < s.hi; i += threads) {
        float x; uint32_t raw;
        load_scalar<DT>(reinterpret_cast<const void*>(s.src), (unsigned long long)i, x, raw);
        const uint32_t b = to_bits<DT>(f.of(x));
        if (DT == HIF8_F32) reinterpret_cast<uint32_t*>(s.dst)[i] = b;
        else reinterpret_cast<unsigned short*>(s.dst)[i] = (unsigned short)b;
    }
}

__global__ void __launch_bounds__(kThreads, kClipPerSM) grad_scale_kernel(const ClipParams p)
{
    __shared__ double s_part[kThreads / 32];
    // (the list is none of the first launch's results, and what wrote it is over since that one runs)
    const long long from = (long long)blockIdx.x * p.per, to = min(p.cost, from + p.per);
    const int first = from < to ? find_tensor(p, from) : 0;
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    double sum = 0.0;
    for (int i = threadIdx.x; i < p.parts; i += kThreads) sum += p.part[i];
    sum = block_sum(sum, s_part);
    const bool finite = sum <= 1.7976931348623157e308;  // (Inf and NaN among the gradients, and nothing else, make it more)
    const int se = p.scale_exp ? clamp_exp(*p.scale_exp) : 0;
    const double norm = ldexp(sqrt(sum), -se);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (p.norm_out) *p.norm_out = finite ? (float)norm : __uint_as_float(0x7F800000u);
        if (!finite && p.found) atomicOr(p.found, 1);
    }
    if (!finite) return;
    const double c = norm > (double)p.max_norm ? (double)p.max_norm / norm : 1.0;
    int k;
    const double m = frexp(c, &k) * 2.0;
    k -= 1 + se;                                  // at most 126, and at least -302: a limit of 2^-149 and a norm of 2^128 times the root of the number of elements
    int k1 = max(-126, min(125, k));              // (m rounded to FP32 may be 2)
    if (k - k1 < -149) k1 = k + 149;              // (results of at most four of FP32's last steps, of whose factor the last bits go)
    const Factor f{ldexpf((float)m, k1), ldexpf(1.f, k - k1)};
    const bool same = f.f == 1.f && f.p == 1.f;  // in place there is nothing to do
    if (from < to)
        for_pieces(p, from, to, first, [&](const Piece16& s, int thread, int threads) {
            if (same && s.src == s.dst) return;
            if (s.dtype == HIF8_F32) scale_piece<HIF8_F32>(s, f, thread, threads);
            else if (s.dtype == HIF8_BF16) scale_piece<HIF8_BF16>(s, f, thread, threads);
            else if (s.dtype == HIF8_F16) scale_piece<HIF8_F16>(s, f, thread, threads);
        });
}

}  // namespace
}  // namespace hif8

using namespace hif8;

extern "C" size_t hif8_grad_clip_workspace_bytes(void) { return kClipBlocks * sizeof(double); }

extern "C" int hif8_grad_clip(const uint64_t* d_src, const uint64_t* d_dst, const int* d_dtype, const int64_t* d_start, int n_tensors, int64_t n_elements, const int* d_scale_exp,
                              float max_norm, float* d_norm, int* d_found_inf, void* workspace, size_t workspace_bytes, hif8_stream_t stream)
{
    if (!(max_norm > 0.f)) return HIF8_ERR_SCALE_RANGE;
    if (n_tensors < 0 || n_elements < 0 || n_elements > (1ll << 50)) return HIF8_ERR_SHAPE;
    if (n_tensors > 0 && (!d_src || !d_dtype || !d_start)) return HIF8_ERR_NULL;
    if (!aligned_to(d_src, 8) || !aligned_to(d_dst, 8) || !aligned_to(d_start, 8) || !aligned_to(d_dtype, 4) || !aligned_to(d_scale_exp, 4) || !aligned_to(d_norm, 4) ||
        !aligned_to(d_found_inf, 4))
        return HIF8_ERR_ALIGN;
    const size_t need = hif8_grad_clip_workspace_bytes();
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 256)) return HIF8_ERR_WORKSPACE;
    const size_t list = (size_t)n_tensors * 8;
    if (written_over({{workspace, need}, {d_norm, d_norm ? 4u : 0u}, {d_found_inf, d_found_inf ? 4u : 0u}},
                     {{d_src, list}, {d_dst, d_dst ? list : 0}, {d_dtype, list / 2}, {d_start, n_tensors ? list + 8 : 0}, {d_scale_exp, d_scale_exp ? 4u : 0u}}))
        return HIF8_ERR_OVERLAP;
    int sms; if (int rc = checked_device(&sms)) return rc;
    ClipParams p{};
    p.src = d_src; p.dst = d_dst; p.dtypes = d_dtype; p.start = d_start; p.tensors = n_tensors; p.total = n_tensors ? n_elements : 0;
    p.scale_exp = d_scale_exp; p.max_norm = max_norm; p.norm_out = d_norm; p.found = d_found_inf; p.part = reinterpret_cast<double*>(workspace);
    p.cost = n_tensors ? n_elements + kTensorCost * n_tensors : 0;
    long long blocks = (p.cost + kShare - 1) / kShare;
    const long long most = (long long)sms * kClipPerSM < kClipBlocks ? (long long)sms * kClipPerSM : kClipBlocks;
    if (blocks > most) blocks = most;
    if (blocks < 1) blocks = 1;
    p.per = ((p.cost + blocks - 1) / blocks + 63) / 64 * 64;
    p.parts = (int)blocks;
    cudaStream_t st = (cudaStream_t)stream;
    launch_pdl(grad_squares_kernel, dim3((unsigned)blocks), st, p);
    launch_pdl(grad_scale_kernel, dim3((unsigned)blocks), st, p);
    g_launches.fetch_add(2, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}
