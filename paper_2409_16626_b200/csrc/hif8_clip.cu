// The global norm of many gradients, and clipping: what stands between the backward pass under a loss scale of 2^s and the optimizer's step.
//
//   norm = sqrt(sum g^2) 2^-s,   out = g 2^-s min(1, max_norm / norm)
//
// Two launches: sums of squares, a share of all elements to a block, and the scaling, in front of which every block adds the shares up in the same order. Both
// are bound by memory.  Gradients are a list of tensors; the elements of all of them in a row are what blocks share out, so that a list of many small tensors
// and few large ones takes the time of its bytes.  Squares are added in FP32 over 16 bytes and in FP64 from there on (vectors whose sum leaves FP32's comfortable
// range: in FP64 altogether), so the norm is as exact as FP32 can say, and the squares of finite gradients do not overflow.
#include "hif8_block.cuh"

namespace hif8 {
namespace {

constexpr int kClipBlocks = 1024;   // shares of the sum at most
constexpr int kClipUnroll = 4;

struct ClipParams {
    const uint64_t* src;
    const uint64_t* dst;
    const int* dtypes;
    const int64_t* start;
    int tensors;
    long long total, per;   // elements; elements of a block's share
    const int* scale_exp;
    float max_norm;
    float* norm_out;
    int* found;
    double* part;
    int parts;
};

// Where the elements from .. to - 1 of the whole list lie in one tensor: its elements lo .. hi - 1 (shares start on multiples of eight within it).
struct Segment {
    uint64_t src, dst;
    long long lo, hi;
    int dtype;
};

__device__ __forceinline__ long long start_of(const ClipParams& p, int t) { return max(0ll, min((long long)p.start[t], p.total)); }

// the last tensor that starts at or in front of `at` (a warp together, one probe a lane and round)
__device__ __forceinline__ int find_tensor(const ClipParams& p, long long at)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = p.tensors;
    while (n > 1) {
        const int step = (n + 31) >> 5, i = lo + lane * step;
        const bool below = lane * step < n && (lane == 0 || start_of(p, i) <= at);
        const int last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, below));
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}

__device__ __forceinline__ Segment segment_of(const ClipParams& p, int t, long long from, long long to)
{
    Segment s;
    const long long b = start_of(p, t), e = start_of(p, t + 1), n = max(0ll, e - b);
    s.src = p.src[t];
    s.dst = p.dst ? p.dst[t] : s.src;
    s.dtype = p.dtypes[t];
    s.lo = from <= b ? 0 : min(n, (from - b + 7) & ~7ll);
    s.hi = to <= b ? 0 : min(n, (to - b + 7) & ~7ll);
    return s;
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

template <int DT> __device__ __forceinline__ double segment_squares(const Segment& s)
{
    constexpr int PV = SrcTraits<DT>::kPerVec;
    double sum = 0.0;
    long long tail = s.lo;
    if ((s.src & 15u) == 0) {
        const uint4* v4 = reinterpret_cast<const uint4*>(s.src);
        const long long end = s.hi / PV;
        for (long long base = s.lo / PV + threadIdx.x; base < end; base += kThreads * kClipUnroll) {
            uint4 v[kClipUnroll];
#pragma unroll
            for (int j = 0; j < kClipUnroll; j++) v[j] = base + j * kThreads < end ? v4[base + j * kThreads] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < kClipUnroll; j++) sum += squares<DT>(v[j]);
        }
        tail = end * PV;
    }
    for (long long i = tail + threadIdx.x; i < s.hi; i += kThreads) {
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

__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const ClipParams p)
{
    __shared__ double s_part[kThreads / 32];
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    const long long from = (long long)blockIdx.x * p.per, to = min(p.total, from + p.per);
    double sum = 0.0;
    if (from < to) {
        for (int t = find_tensor(p, from); t < p.tensors && start_of(p, t) < to; t++) {
            const Segment s = segment_of(p, t, from, to);
            if (s.lo >= s.hi) continue;
            if (s.dtype == HIF8_F32) sum += segment_squares<HIF8_F32>(s);
            else if (s.dtype == HIF8_BF16) sum += segment_squares<HIF8_BF16>(s);
            else if (s.dtype == HIF8_F16) sum += segment_squares<HIF8_F16>(s);
        }
    }
    sum = block_sum(sum, s_part);
    if (threadIdx.x == 0) p.part[blockIdx.x] = sum;
}

// x f p, p a power of two that is 1 unless f p is no normal FP32: one rounding (below 2^-126, and only then, a second)
struct Factor {
    float f, p;
    __device__ __forceinline__ float of(float x) const { return x * f * p; }
};

template <int DT> __device__ __forceinline__ uint4 scaled(const uint4& v, const Factor& f)
{
    constexpr int PV = SrcTraits<DT>::kPerVec;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < PV; k++) {
        float x; uint32_t raw;
        unpack<DT>(v, k, x, raw);
        const uint32_t b = to_bits<DT>(f.of(x));
        if (DT == HIF8_F32) w[k] = b;
        else w[k >> 1] |= b << (16 * (k & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// (from its end: what the first launch read last may still be in L2)
template <int DT> __device__ __forceinline__ void scale_segment(const Segment& s, const Factor& f)
{
    constexpr int PV = SrcTraits<DT>::kPerVec;
    long long tail = s.lo;
    if (((s.src | s.dst) & 15u) == 0) {
        const uint4* v4 = reinterpret_cast<const uint4*>(s.src);
        uint4* o4 = reinterpret_cast<uint4*>(s.dst);
        const long long first = s.lo / PV, end = s.hi / PV;
        for (long long base = end - 1 - threadIdx.x; base >= first; base -= kThreads * kClipUnroll) {
            uint4 v[kClipUnroll];
#pragma unroll
            for (int j = 0; j < kClipUnroll; j++) v[j] = base - j * kThreads >= first ? __ldcs(v4 + base - j * kThreads) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < kClipUnroll; j++)
                if (base - j * kThreads >= first) __stcs(o4 + base - j * kThreads, scaled<DT>(v[j], f));
        }
        tail = end * PV;
    }
    for (long long i = tail + threadIdx.x; i < s.hi; i += kThreads) {
        float x; uint32_t raw;
        load_scalar<DT>(reinterpret_cast<const void*>(s.src), (unsigned long long)i, x, raw);
        const uint32_t b = to_bits<DT>(f.of(x));
        if (DT == HIF8_F32) reinterpret_cast<uint32_t*>(s.dst)[i] = b;
        else reinterpret_cast<unsigned short*>(s.dst)[i] = (unsigned short)b;
    }
}

__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const ClipParams p)
{
    __shared__ double s_part[kThreads / 32];
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
    k = max(-252, min(250, k - 1 - se));
    const int k1 = max(-126, min(125, k));  // (m rounded to FP32 may be 2)
    const Factor f{(float)m * pow2f(k1), pow2f(k - k1)};
    const bool same = f.f == 1.f && f.p == 1.f;  // in place there is nothing to do
    const long long from = (long long)blockIdx.x * p.per, to = min(p.total, from + p.per);
    if (from >= to) return;
    for (int t = find_tensor(p, to - 1); t >= 0 && start_of(p, t + 1) > from; t--) {
        const Segment s = segment_of(p, t, from, to);
        if (s.lo >= s.hi || (same && s.src == s.dst)) continue;
        if (s.dtype == HIF8_F32) scale_segment<HIF8_F32>(s, f);
        else if (s.dtype == HIF8_BF16) scale_segment<HIF8_BF16>(s, f);
        else if (s.dtype == HIF8_F16) scale_segment<HIF8_F16>(s, f);
    }
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
    // a share: 2048 elements or more, a multiple of that
    long long blocks = (p.total + 2047) / 2048;
    const long long most = (long long)sms * 6 < kClipBlocks ? (long long)sms * 6 : kClipBlocks;
    if (blocks > most) blocks = most;
    if (blocks < 1) blocks = 1;
    p.per = ((p.total + blocks - 1) / blocks + 2047) / 2048 * 2048;
    p.parts = (int)blocks;
    cudaStream_t st = (cudaStream_t)stream;
    launch_pdl(grad_squares_kernel, dim3((unsigned)blocks), st, p);
    launch_pdl(grad_scale_kernel, dim3((unsigned)blocks), st, p);
    g_launches.fetch_add(2, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}
