// Block-scaled products of one or two rows and a large [N,K] weight: single tokens.
//
//   C[m,n] (+)= sum_k value(A(m,k)) 2^-ea value(W(n,k)) 2^-ew
//
// Bound by the weights' bytes from DRAM and by one table lookup a code.  Every warp works alone on a slice of 512 k, sixteen to a lane, whose activations it keeps in registers as
// FP32 with both scales multiplied on (exact; made again where the rows of W come to another block), and streams rows of W through its registers, eight on their way.  Weights do not
// pass through shared memory and are not multiplied by the tensor core, which would have one row in sixteen to do here: a lookup is a wavefront of shared memory for 32 codes, and half a packed
// multiply-add a row of A.  Lanes' sums of eight rows are added by exchanges that halve the rows a lane holds; the slices' sums meet in shared memory and are added in order.
// us a call in a graph, the kernel on tensor memory (with the launch that expands the activations) / this: 1 x 4096 -> 14336 20.9 / 16.8, 1 x 8192 -> 8192 21.8 / 18.5, 1 x 8192 -> 28672 54.8 / 50.5, 1 x 1024 -> 32000 16.8 / 11.9,
// 2 x 4096 -> 14336 20.9 / 19.6; 2 x 4096 -> 4096 9.5 / 10.8, which the costs leave to the other.  A wavefront takes 1.7 cycles in the mean (four warps a scheduler do not cover the lookups' latency; 24 warps of 80 registers 18.4, 32 of 64 23.0: they spill).  Not taken: four
// rows in eight warps of twice the registers 20.8 / 27.2, two slices a warp for K beyond 8192 19.4 / 24.3.
#include "hif8_block.cuh"
#include "hif8_host_cache.h"

namespace hif8 {
namespace {

struct RowsParams {
    BlockCodes a, w;
    void* C;
    long long ldc;
    int c_is_f32, accumulate, N, K;
    int* status;
    int slices, groups;        // of 512 k: warps that share a row of W; such groups of a block
    int units, chunks;         // groups of the grid; stretches of kChunkRows rows of one
};

constexpr int kRowsWarps = 16, kSliceK = 512, kOctet = 8, kChunkRows = 64;
constexpr uint32_t kRowsTable = 65536;  // rows of 256 bytes on a boundary of 64 KiB: a byte permutation makes an address

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float lookup(uint32_t at)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ unsigned long long pair_of(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ unsigned long long fma_pair(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// byte K of w
template <int K> __device__ __forceinline__ float value_at(uint32_t w, uint32_t table_lane) { return lookup(__byte_perm(w, table_lane, 0x7604 | (K << 4))); }

// Sums over the lanes of V values a lane, V a power of two: lane l ends with that of value l >> (5 - log2 V)
template <int V>
__device__ __forceinline__ float sums_of_lanes(float (&v)[V], unsigned lane)
{
    int d = 16;
#pragma unroll
    for (int half = V / 2; half; half >>= 1, d >>= 1) {
        const bool up = lane & d;
#pragma unroll
        for (int i = 0; i < half; i++) {
            const float mine = up ? v[i + half] : v[i], other = up ? v[i] : v[i + half];
            v[i] = mine + __shfl_xor_sync(0xFFFFFFFFu, other, d);
        }
    }
    float s = v[0];
#pragma unroll
    for (; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    return s;
}

template <int M>
__global__ void __launch_bounds__(kRowsWarps * 32, 1) block_rows_kernel(const RowsParams p)
{
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = shared_address(smem_raw), table = (raw + kRowsTable - 1) & ~(kRowsTable - 1);
    unsigned char* after = smem_raw + (table - raw) + kRowsTable;
    const unsigned lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
#pragma unroll 4
    for (unsigned c = warp; c < 256; c += kRowsWarps) *reinterpret_cast<uint32_t*>(smem_raw + (table - raw) + c * 256 + lane * 4) = decode_bits_f32(c);
    __syncthreads();
    pdl_wait_prior_grid();
    pdl_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
    const uint32_t table_lane = table + lane * 4;
    const int group = (int)warp / p.slices, unit = (int)blockIdx.x * p.groups + group;
    const bool works = group < p.groups;
    auto first_row = [&](int u) { return (int)((long long)p.N * u / p.units); };
    const int n0 = works ? first_row(unit) : 0, n1 = works ? first_row(unit + 1) : 0, from = n0 & ~(kOctet - 1);

    // this lane's k: sixteen from here on
    const int k = (int)warp % p.slices * kSliceK + (int)lane * 16;
    auto masked = [&](uint4 w, int n) {  // the first n bytes
        auto mask = [&](int m) { return m >= 4 ? 0xFFFFFFFFu : m <= 0 ? 0u : (1u << (8 * m)) - 1u; };
        return make_uint4(w.x & mask(n), w.y & mask(n - 4), w.z & mask(n - 8), w.w & mask(n - 12));
    };
    // (no branch stands in the loop over rows, so that their lookups overlap: rows of other groups and k behind the end are read in the place of what is not there; their sums are not used, their bytes masked)
    const uint4 there = masked(make_uint4(0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu), p.K - k);
    const uint8_t* column = p.w.codes + min(k, (p.K - 1) & ~15);
    uint4 ring[kOctet];
    auto fetch = [&](int n, int r) { ring[r] = __ldcs(reinterpret_cast<const uint4*>(column + (size_t)max(n0, min(n, n1 - 1)) * (size_t)p.w.ld)); };
    if (n0 < n1) {
#pragma unroll
        for (int r = 0; r < kOctet; r++) fetch(from + r, r);
    }

    unsigned long long x[M][8];  // this lane's activations, in pairs, with their scale and that of the block of W
    float back[M];               // what their sums are multiplied by: 1, or 2^96 where the activations would have left FP32
    auto activations = [&](int n) {
        auto exponent = [](const BlockCodes& c, int row, int col) {
            return max(-HIF8_BLOCK_EXP_MAX, min(HIF8_BLOCK_EXP_MAX, __ldg(c.exps + (size_t)(row >> c.shift) * (size_t)c.exp_stride + (col >> 7))));
        };
        const int ew = k < p.K ? exponent(p.w, n, k) : 0;
#pragma unroll
        for (int m = 0; m < M; m++) {
            uint4 c = make_uint4(0u, 0u, 0u, 0u);
            int ea = 0;
            if (k < p.K) {
                c = masked(__ldg(reinterpret_cast<const uint4*>(p.a.codes + (size_t)m * (size_t)p.a.ld + k)), p.K - k);
                ea = exponent(p.a, m, k);
            }
            const float sa = pow2f(-ea), sw = pow2f(-ew);
            float v[16];
            const uint32_t words[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v[4 * i] = value_at<0>(words[i], table_lane) * sa; v[4 * i + 1] = value_at<1>(words[i], table_lane) * sa;
                v[4 * i + 2] = value_at<2>(words[i], table_lane) * sa; v[4 * i + 3] = value_at<3>(words[i], table_lane) * sa;
            }
            // (sixteen magnitudes within 2^38 of one another: with one of them beyond FP32 none is lost below it when all are 2^96 smaller)
            bool beyond = false;
#pragma unroll
            for (int i = 0; i < 16; i++) beyond |= fabsf(v[i]) < __uint_as_float(0x7F800000u) && fabsf(v[i] * sw) > 3.402823466e38f;
            const float s = beyond ? pow2f(max(-126, -ew - 96)) : sw;
            back[m] = beyond ? pow2f(96) : 1.f;
#pragma unroll
            for (int i = 0; i < 8; i++) x[m][i] = pair_of(v[2 * i] * s, v[2 * i + 1] * s);
        }
    };

    float* deposits = reinterpret_cast<float*>(after);
    int block = -1;
    for (int chunk = 0; chunk < p.chunks; chunk++) {
        float* mine = deposits + (size_t)(chunk & 1) * kRowsWarps * M * kChunkRows + warp * M * kChunkRows;
#pragma unroll 1
        for (int o = 0; o < kChunkRows / kOctet; o++) {
            const int n = from + chunk * kChunkRows + o * kOctet;
            if (n >= n1) break;
            if ((n >> 7) != block) {  // (an octet lies in one block)
                block = n >> 7;
                activations(n);
            }
            float acc[kOctet * M];
#pragma unroll
            for (int r = 0; r < kOctet; r++) {
                const uint32_t words[4] = {ring[r].x & there.x, ring[r].y & there.y, ring[r].z & there.z, ring[r].w & there.w};
                unsigned long long dot[M];
#pragma unroll
                for (int m = 0; m < M; m++) dot[m] = 0ull;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const unsigned long long lo = pair_of(value_at<0>(words[i], table_lane), value_at<1>(words[i], table_lane));
                    const unsigned long long hi = pair_of(value_at<2>(words[i], table_lane), value_at<3>(words[i], table_lane));
#pragma unroll
                    for (int m = 0; m < M; m++) dot[m] = fma_pair(hi, x[m][2 * i + 1], fma_pair(lo, x[m][2 * i], dot[m]));
                }
#pragma unroll
                for (int m = 0; m < M; m++) {
                    float lo, hi;
                    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(dot[m]));
                    acc[r * M + m] = (lo + hi) * back[m];
                }
                fetch(n + kOctet + r, r);
            }
            constexpr int kValues = kOctet * M, kShift = M == 1 ? 2 : 1;
            const float s = sums_of_lanes<kValues>(acc, lane);
            const int value = (int)lane >> kShift;  // row * M + m
            if ((lane & ((1u << kShift) - 1u)) == 0) mine[(value & (M - 1)) * kChunkRows + o * kOctet + value / M] = s;
        }
        __syncthreads();
        const float* all = deposits + (size_t)(chunk & 1) * kRowsWarps * M * kChunkRows;
        for (int i = threadIdx.x; i < p.groups * M * kChunkRows; i += kRowsWarps * 32) {
            const int r = i & (kChunkRows - 1), m = i / kChunkRows & (M - 1), g = i / (kChunkRows * M), u = (int)blockIdx.x * p.groups + g;
            const int lo = first_row(u), n = (lo & ~(kOctet - 1)) + chunk * kChunkRows + r;
            if (n < lo || n >= first_row(u + 1)) continue;
            float s = 0.f;
            for (int w = 0; w < p.slices; w++) s += all[((g * p.slices + w) * M + m) * kChunkRows + r];
            if (p.c_is_f32) {
                float* out = reinterpret_cast<float*>(p.C) + (size_t)m * (size_t)p.ldc + n;
                *out = p.accumulate ? *out + s : s;
            } else {
                unsigned short* out = reinterpret_cast<unsigned short*>(p.C) + (size_t)m * (size_t)p.ldc + n;
                *out = (unsigned short)to_bits<HIF8_BF16>(p.accumulate ? __uint_as_float((uint32_t)*out << 16) + s : s);
            }
        }
        // (the next stretch's deposits go to the other half, and those after it stand behind its barrier)
    }
}

template <int M>
int launch_rows(RowsParams p, int sms, cudaStream_t st)
{
    constexpr size_t bytes = 2 * (size_t)kRowsTable + 2 * (size_t)kRowsWarps * M * kChunkRows * sizeof(float);
    static PerDevice<cudaError_t> ready;  // a fact of the device, set by its first such call
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HIF8_ERR_CUDA;
    const cudaError_t* rc = ready.get(dev, [&](int, cudaError_t* out) {
        *out = cudaFuncSetAttribute(block_rows_kernel<M>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    });
    if (!rc || *rc != cudaSuccess) return HIF8_ERR_CUDA;
    p.slices = (p.K + kSliceK - 1) / kSliceK;
    p.groups = kRowsWarps / p.slices;
    const int octets = (p.N + kOctet - 1) / kOctet, blocks = (octets + p.groups - 1) / p.groups < sms ? (octets + p.groups - 1) / p.groups : sms;
    p.units = blocks * p.groups;
    p.chunks = ((p.N + p.units - 1) / p.units + kOctet + kChunkRows - 1) / kChunkRows;  // (a unit's rows begin inside an octet)
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kRowsWarps * 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, block_rows_kernel<M>, p) != cudaSuccess) return HIF8_ERR_CUDA;
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? HIF8_OK : HIF8_ERR_CUDA;
}

}  // namespace

double block_rows_cycles(int M, int N, int K, int sms)
{
    const int slices = (K + kSliceK - 1) / kSliceK;
    if (M > 2 || slices > kRowsWarps) return 1e30;
    // lookups of a block's warps, 1.7 and 1.9 cycles each with all sixteen at work
    const double lookups = (double)N * slices * (kSliceK / 32) / sms * kRowsWarps / (double)(slices * (kRowsWarps / slices));
    return M == 1 ? 1.7 * lookups + 10000.0 : 1.9 * lookups + 13700.0;
}

int launch_block_rows(const BlockCodes& a, const BlockCodes& w, const GemmParams& g, cudaStream_t st)
{
    int sms; if (int rc = checked_device(&sms)) return rc;
    RowsParams p{};
    p.a = a; p.w = w; p.C = g.C; p.ldc = g.ldc; p.c_is_f32 = g.c_is_f32; p.accumulate = g.accumulate; p.N = g.N; p.K = g.K; p.status = g.status;
    return g.M == 1 ? launch_rows<1>(p, sms, st) : launch_rows<2>(p, sms, st);
}

}  // namespace hif8
