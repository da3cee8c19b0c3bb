// What the kernels of block-scaled matrices share: a thread's eight neighbouring elements of a row, sixteen threads to a block's width.
#pragma once
#include "hif8_block_types.cuh"
#include "hif8_device.cuh"

namespace hif8 {
namespace {

// n / d for n < 2^31 by a multiplication and a shift (Granlund and Montgomery, 1994)
struct FastDiv {
    uint32_t d, mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t d_) : d(d_), shift(0)
    {
        while ((1ull << shift) < d) shift++;
        mul = (uint32_t)((((1ull << shift) - d) << 32) / d + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(mul, n) + n) >> shift; }
};

__device__ __forceinline__ int clamp_block_exp(int e) { return max(-HIF8_BLOCK_EXP_MAX, min(HIF8_BLOCK_EXP_MAX, e)); }
__device__ __forceinline__ int block_exp_from_amax(uint32_t amax_bits, int target_exp) { return clamp_block_exp(scale_exp_from_amax(amax_bits, target_exp)); }

// Eight elements c .. c + 7 of a row of `cols`, zeros behind its end: 16 bytes, of FP32 32.  `vectors`: the row starts on a 16-byte boundary (and c is a multiple of 8).
// KEEP: they will be read again.  WHOLE: the row does so and `cols` is a multiple of 8, so no element is looked at by itself.
template <int DT> struct Eight { uint4 v[DT == HIF8_F32 ? 2 : 1]; };
template <int DT, bool KEEP = false, bool WHOLE = false>
__device__ __forceinline__ Eight<DT> load_eight(const void* row, long long c, long long cols, bool vectors)
{
    Eight<DT> e;
    if (WHOLE) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row) + (unsigned)c * (DT == HIF8_F32 ? 4u : 2u));
        const bool in = (int)c < (int)cols;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(e.v) / 16); i++) e.v[i] = !in ? make_uint4(0, 0, 0, 0) : KEEP ? __ldg(p + i) : __ldcs(p + i);
        return e;
    }
    static_assert(WHOLE || !KEEP, "what is read again is read in whole rows");
    if (DT == HIF8_F32) {
        const float* p = reinterpret_cast<const float*>(row) + c;
        if (vectors && c + 8 <= cols) {
            e.v[0] = __ldcs(reinterpret_cast<const uint4*>(p));
            e.v[sizeof(e.v) / 16 - 1] = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = c + i < cols ? __float_as_uint(__ldcs(p + i)) : 0u;
            e.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
            e.v[sizeof(e.v) / 16 - 1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    } else {
        const unsigned short* p = reinterpret_cast<const unsigned short*>(row) + c;
        if (vectors && c + 8 <= cols) e.v[0] = __ldcs(reinterpret_cast<const uint4*>(p));
        else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t lo = c + 2 * i < cols ? __ldcs(p + 2 * i) : 0, hi = c + 2 * i + 1 < cols ? __ldcs(p + 2 * i + 1) : 0;
                w[i] = lo | (hi << 16);
            }
            e.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    return e;
}
template <int DT>
__device__ __forceinline__ void unpack_eight(const Eight<DT>& e, int i, float& x, uint32_t& raw)
{
    if (DT == HIF8_F32) unpack<DT>(e.v[i >> 2], i & 3, x, raw);
    else unpack<DT>(e.v[0], i, x, raw);
}
template <int DT>
__device__ __forceinline__ float value_of_eight(const Eight<DT>& e, int i)
{
    float x; uint32_t raw;
    unpack_eight<DT>(e, i, x, raw);
    return x;
}
// eight values, rounded to nearest even
template <int DT>
__device__ __forceinline__ Eight<DT> pack_eight(const float (&x)[8])
{
    Eight<DT> e;
    uint32_t w[8];
    if (DT == HIF8_F32) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = __float_as_uint(x[i]);
        e.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        e.v[sizeof(e.v) / 16 - 1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (DT == HIF8_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
            else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
        }
        e.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return e;
}
template <int DT, bool WHOLE = false>
__device__ __forceinline__ void store_eight(void* row, long long c, long long cols, bool vectors, const Eight<DT>& e)
{
    if (WHOLE) {
        uint4* p = reinterpret_cast<uint4*>(reinterpret_cast<char*>(row) + (unsigned)c * (DT == HIF8_F32 ? 4u : 2u));
        if ((int)c < (int)cols) {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(e.v) / 16); i++) p[i] = e.v[i];
        }
        return;
    }
    if (DT == HIF8_F32) {
        float* p = reinterpret_cast<float*>(row) + c;
        if (vectors && c + 8 <= cols) {
            *reinterpret_cast<uint4*>(p) = e.v[0];
            reinterpret_cast<uint4*>(p)[1] = e.v[sizeof(e.v) / 16 - 1];
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (c + i < cols) p[i] = value_of_eight<DT>(e, i);
        }
    } else {
        unsigned short* p = reinterpret_cast<unsigned short*>(row) + c;
        if (vectors && c + 8 <= cols) *reinterpret_cast<uint4*>(p) = e.v[0];
        else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float x; uint32_t raw;
                unpack_eight<DT>(e, i, x, raw);
                if (c + i < cols) p[i] = (unsigned short)raw;
            }
        }
    }
}
// The same of rows that lie on no 16-byte boundary: element i is column c + 32 i, c the warp's first column plus the lane, so that a warp reads and writes whole lines, an
// element a lane and instruction.  (Eight neighbouring elements a thread, one by one, took four to nine times as long as rows that are aligned.)
template <int DT, bool KEEP = false>
__device__ __forceinline__ Eight<DT> load_spread(const void* row, int c, int cols)
{
    Eight<DT> e;
    uint32_t w[8];
    auto get = [&](int i) -> uint32_t {
        if (DT == HIF8_F32) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + c + 32 * i;
            return KEEP ? __ldg(p) : __ldcs(p);
        }
        const unsigned short* p = reinterpret_cast<const unsigned short*>(row) + c + 32 * i;
        return KEEP ? __ldg(p) : __ldcs(p);
    };
    if ((c | 31) + 224 < cols) {  // (the same for a warp)
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = get(i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = c + 32 * i >= cols ? 0u : get(i);
    }
    constexpr int last = sizeof(e.v) / 16 - 1;
    if (DT == HIF8_F32) {
        e.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        e.v[last] = make_uint4(w[4], w[5], w[6], w[7]);
    } else
        e.v[0] = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[4], w[5], 0x5410), __byte_perm(w[6], w[7], 0x5410));
    return e;
}
template <int DT>
__device__ __forceinline__ void store_spread(void* row, int c, int cols, const Eight<DT>& e)
{
    auto put = [&](int i) {
        float x; uint32_t raw;
        unpack_eight<DT>(e, i, x, raw);
        if (DT == HIF8_F32) reinterpret_cast<uint32_t*>(row)[c + 32 * i] = raw;
        else reinterpret_cast<unsigned short*>(row)[c + 32 * i] = (unsigned short)raw;
    };
    if ((c | 31) + 224 < cols) {
#pragma unroll
        for (int i = 0; i < 8; i++) put(i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (c + 32 * i < cols) put(i);
    }
}
__device__ __forceinline__ void store_codes_spread(uint8_t* row, int c, int cols, uint2 w)
{
    if ((c | 31) + 224 < cols) {
#pragma unroll
        for (int i = 0; i < 8; i++) row[c + 32 * i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (c + 32 * i < cols) row[c + 32 * i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}
// eight codes; `vectors`: the row starts on an 8-byte boundary
__device__ __forceinline__ void store_codes8(uint8_t* row, long long c, long long cols, bool vectors, uint2 w)
{
    if (vectors && c + 8 <= cols) *reinterpret_cast<uint2*>(row + c) = w;
    else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (c + i < cols) row[c + i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ uint2 load_codes8(const uint8_t* row, long long c, long long cols, bool vectors)
{
    if (vectors && c + 8 <= cols) return __ldcs(reinterpret_cast<const uint2*>(row + c));
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (c + i < cols) w[i >> 2] |= (uint32_t)row[c + i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}

}  // namespace
}  // namespace hif8
