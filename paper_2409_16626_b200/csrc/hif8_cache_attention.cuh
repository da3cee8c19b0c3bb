// What the attention kernels over the key/value cache share: parameters, what a query may look at, the FP16 values of codes, waits and copies, results.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <mutex>

#include "hif8.h"
#include "hif8_cache.cuh"
#include "hif8_device.cuh"
#include "hif8_host_cache.h"
#include "hif8_internal.cuh"

namespace hif8 {
extern std::atomic<uint64_t> g_launches;

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
    int* special_flag;              // chunks: whether cache_attention_specials_kernel has anything to do; NULL: it looks for itself
    long long* chunks;              // few rows: chunks in all
    int4* cut;                      // two of each group: key head, first row, chunk, chunks of the unit that its first chunk lies in; first query, rows
    float* partial;
};

// The tensor-core path for many query rows (hif8_cache_prefill.cu): the workspace it needs (0: it does not take calls of those bounds), and the call.
size_t prefill_workspace_bytes(int n_seqs, int n_q, int max_q, int max_length, int heads, int kv_heads, int dim);
cudaError_t launch_prefill(AttentionParams p, int dtype, int max_length, uint8_t* ws, int sms, cudaStream_t st);

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();


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
__device__ __forceinline__ uint4 lds_v4(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long global_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
constexpr unsigned long long kWaitLimitNs = 2000000000ull;  // 2 s a wait
// Bounded wait: false when the barrier did not complete in time, or someone else of the block gave up.  (The clock is only read when a wait gets long.)
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int where)
{
    unsigned long long t0 = 0;
    for (uint32_t it = 1;; it++) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 63u) == 0) {
            if (*abort_flag) return false;
            const unsigned long long now = global_ns();
            if (t0 == 0) t0 = now;
            if (now - t0 > kWaitLimitNs) {
                *abort_flag = 1;
                atomicCAS(status, 0, where);
                return false;
            }
        }
    }
}
// a copy that nobody waited for lands before the block's shared memory becomes another's
__device__ __forceinline__ void wait_landed(uint32_t bar, uint32_t parity)
{
    const unsigned long long t0 = global_ns();
    while (!mbar_try_wait(bar, parity) && global_ns() - t0 < kWaitLimitNs) {}
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
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

// Factor of a score: softmax scale / ln 2, the inverses of the powers of two of the query row (e) and of the block (its exponent).  The row's part and the block's
// share a power of two, 2^-kMulShift and 2^(kMulShift - e_k), so that neither leaves the floats where the product does not.  The product stays in [1e-36, 3e38]: below, scores count as
// nothing anyway (a product of codes is below 2^40); a factor of 0 would turn the -Inf of a token that a row does not see into NaN, and so would Inf a score of 0.
constexpr int kMulShift = 24;
__device__ __forceinline__ float query_factor(float scale_log2, int e) { return fminf(scale_log2 * pow2_clamped(-e - kMulShift), 3.0e38f); }
__device__ __forceinline__ float score_factor(float row, float block) { return fmaxf(fminf(row * block, 3.0e38f), 1.0e-36f); }

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

__device__ __forceinline__ long long div_small(long long a, int b) { return a >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); }
// first chunk of group g
__host__ __device__ __forceinline__ long long share_of(long long chunks, int g, int groups) { return chunks * g / groups; }
// ... and the group that chunk x belongs to
__device__ __forceinline__ int owner_of(long long chunks, long long x, int groups) { return (int)(((x + 1) * groups - 1) / chunks); }

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
template <int DT> __device__ __forceinline__ void store_out8(const AttentionParams& p, long long at, const float (&x)[8])
{
    if (p.vectors) *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(p.out) + at) =
                       make_uint4(pack_out<DT>(x[0], x[1]), pack_out<DT>(x[2], x[3]), pack_out<DT>(x[4], x[5]), pack_out<DT>(x[6], x[7]));
    else {
#pragma unroll
        for (int y = 0; y < 8; y += 4) {
            const float z[4] = {x[y], x[y + 1], x[y + 2], x[y + 3]};
            store_out4<DT>(p, at + y, z);
        }
    }
}
// from a row's maximum, its denominator and the power of two that the weights carry
__device__ __forceinline__ float lse_of(float m, float l, float shift) { return l == 0.f ? kNegInf : (m - shift + log2f(l)) * kLn2; }
__device__ __forceinline__ float part_factor(float m, float top) { return m == kNegInf ? 0.f : exp2_approx(m - top); }

// ---- host side
constexpr int kMaxBlocks = 148;  // what workspaces are sized for
inline size_t round_up_256(size_t n) { return (n + 255) & ~(size_t)255; }
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_tiled_fn()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess) fn = reinterpret_cast<EncodeTiledFn>(sym);
    });
    return fn;
}

}  // namespace
}  // namespace hif8
