// Floating-point tensors in device code: groups of neighbouring elements in one load, their values in fp32, and the 8-bit
// form of a block (eoq_ckpt_save).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "eoq_device.cuh"
#include "eoq_internal.h"

namespace eoq {

// kBytes neighbouring bytes as they stand in memory
template <int kBytes> struct Raw;
template <> struct Raw<1> { uint8_t w; };
template <> struct Raw<2> { uint16_t w; };
template <> struct Raw<4> { uint32_t w; };
template <> struct Raw<8> { uint2 w; };
template <> struct Raw<16> { uint4 w; };

template <int kBytes>
__device__ __forceinline__ Raw<kBytes> load_raw(const void *p)
{
    Raw<kBytes> r;
    r.w = __ldg(reinterpret_cast<const decltype(r.w) *>(p));
    return r;
}
template <int kBytes>
__device__ __forceinline__ Raw<kBytes> zero_raw()
{
    Raw<kBytes> r{};
    return r;
}
template <int kBytes>
__device__ __forceinline__ void store_raw(void *p, const Raw<kBytes> &r)
{
    *reinterpret_cast<decltype(r.w) *>(p) = r.w;
}
__device__ __forceinline__ uint32_t raw_word(const Raw<1> &r, int) { return r.w; }
__device__ __forceinline__ uint32_t raw_word(const Raw<2> &r, int) { return r.w; }
__device__ __forceinline__ uint32_t raw_word(const Raw<4> &r, int) { return r.w; }
__device__ __forceinline__ uint32_t raw_word(const Raw<8> &r, int i) { return i == 0 ? r.w.x : r.w.y; }
__device__ __forceinline__ uint32_t raw_word(const Raw<16> &r, int i) { return i == 0 ? r.w.x : i == 1 ? r.w.y : i == 2 ? r.w.z : r.w.w; }
__device__ __forceinline__ void set_word(Raw<1> &r, int, uint32_t v) { r.w = (uint8_t)v; }
__device__ __forceinline__ void set_word(Raw<2> &r, int, uint32_t v) { r.w = (uint16_t)v; }
__device__ __forceinline__ void set_word(Raw<4> &r, int, uint32_t v) { r.w = v; }
__device__ __forceinline__ void set_word(Raw<8> &r, int i, uint32_t v) { if (i == 0) r.w.x = v; else r.w.y = v; }
__device__ __forceinline__ void set_word(Raw<16> &r, int i, uint32_t v)
{
    if (i == 0) r.w.x = v;
    else if (i == 1) r.w.y = v;
    else if (i == 2) r.w.z = v;
    else r.w.w = v;
}

// Element types by their EOQ_* number.  to_f32 and from_f32 work on kN neighbouring elements; from_f32 rounds to nearest, ties to
// even.  int32 values are rounded to fp32 (24 bits of a sum); int8 values are written through Q_a2: sat(R(v * 2^7), -127, 127).
template <int kType> struct Elem;
template <> struct Elem<EOQ_F32> {
    static constexpr int kSize = 4;
    template <int kN>
    static __device__ __forceinline__ void to_f32(const Raw<4 * kN> &r, float (&v)[kN])
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = __uint_as_float(raw_word(r, i));
    }
    template <int kN>
    static __device__ __forceinline__ Raw<4 * kN> from_f32(const float (&v)[kN])
    {
        Raw<4 * kN> r;
#pragma unroll
        for (int i = 0; i < kN; ++i) set_word(r, i, __float_as_uint(v[i]));
        return r;
    }
};
template <> struct Elem<EOQ_I32> {
    static constexpr int kSize = 4;
    template <int kN>
    static __device__ __forceinline__ void to_f32(const Raw<4 * kN> &r, float (&v)[kN])
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = __int2float_rn((int)raw_word(r, i));
    }
};
template <> struct Elem<EOQ_F16> {
    static constexpr int kSize = 2;
    template <int kN>
    static __device__ __forceinline__ void to_f32(const Raw<2 * kN> &r, float (&v)[kN])
    {
        if constexpr (kN == 1) {
            v[0] = __half2float(__ushort_as_half((unsigned short)raw_word(r, 0)));
        } else {
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                const uint32_t w = raw_word(r, i);
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        }
    }
    template <int kN>
    static __device__ __forceinline__ Raw<2 * kN> from_f32(const float (&v)[kN])
    {
        Raw<2 * kN> r;
        if constexpr (kN == 1) {
            set_word(r, 0, __half_as_ushort(__float2half_rn(v[0])));
            return r;
        } else {
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                set_word(r, i, *reinterpret_cast<const uint32_t *>(&h));
            }
        }
        return r;
    }
};
template <> struct Elem<EOQ_BF16> {
    static constexpr int kSize = 2;
    template <int kN>
    static __device__ __forceinline__ void to_f32(const Raw<2 * kN> &r, float (&v)[kN])
    {
        if constexpr (kN == 1) {
            v[0] = __uint_as_float(raw_word(r, 0) << 16);
        } else {
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                const uint32_t w = raw_word(r, i);
                v[2 * i] = __uint_as_float(w << 16);
                v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
            }
        }
    }
    template <int kN>
    static __device__ __forceinline__ Raw<2 * kN> from_f32(const float (&v)[kN])
    {
        Raw<2 * kN> r;
        if constexpr (kN == 1) {
            set_word(r, 0, __bfloat16_as_ushort(__float2bfloat16_rn(v[0])));
            return r;
        } else {
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                set_word(r, i, *reinterpret_cast<const uint32_t *>(&h));
            }
        }
        return r;
    }
};
constexpr int kElemI8 = 100;   // int8 codes at exponent -7 (outputs of the int32 form) or at an exponent of their own (errors)
template <> struct Elem<kElemI8> {
    static constexpr int kSize = 1;
    template <int kN>
    static __device__ __forceinline__ void to_f32(const Raw<kN> &r, float (&v)[kN])
    {
        // 2^23 + (code + 128) is a float whose bits are put together from the byte
#pragma unroll
        for (int i = 0; i < kN; ++i)
            v[i] = __uint_as_float(__byte_perm(raw_word(r, i / 4) ^ 0x80808080u, 0x4B000000u, 0x7650 + (i & 3))) - 8388736.0f;
    }
    template <int kN>
    static __device__ __forceinline__ Raw<kN> from_f32(const float (&v)[kN])
    {
        Raw<kN> r;
        int q[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) q[i] = clampi(__float2int_rn(v[i] * 128.0f), -127, 127);
        if constexpr (kN < 4) {
            set_word(r, 0, kN == 1 ? (uint32_t)q[0] : __byte_perm((uint32_t)q[0], (uint32_t)q[kN - 1], 0x0040));
        } else {
#pragma unroll
            for (int i = 0; i < kN / 4; ++i) set_word(r, i, pack4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]));
        }
        return r;
    }
};

// ------------------------------------------------------------------ the 8-bit form of a block of 32 values
// A step of 2^(s - 127), the smallest with max|v| <= 127 steps: with max|v| = m * 2^k, 1 <= m < 2, that is 2^(k - 6) as long as
// m <= 127/64 and 2^(k - 5) above, which adding 2^23 - 1 - (mantissa of 127/64) to the bits carries into the exponent.  Steps are
// powers of two, so scaling is exact and a code is off by half a step at most; s >= 1 keeps step and inverse normal numbers.
// s = 255 (an infinite step, codes 0) marks a block that holds an infinity or a NaN: 0 * infinity reads back as NaN.

// larger magnitude, NaN if either is (the bits of a NaN are above those of infinity)
__device__ __forceinline__ float max_abs(float m, float v)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(v)));
    return r;
}
__device__ __forceinline__ int block_exp(float amax)
{
    const uint32_t b = __float_as_uint(amax);
    if (b >= 0x7f800000u) return 255;
    return max((int)((b + 0x1ffffu) >> 23) - 6, 1);
}
__device__ __forceinline__ float block_step(int s) { return __uint_as_float((uint32_t)s << 23); }

// the codes of kN values of a block, packed in words (one or two codes in the low bytes)
template <int kN>
__device__ __forceinline__ void block_codes(const float (&v)[kN], int s, uint32_t (&w)[(kN + 3) / 4])
{
    const float per = __uint_as_float((uint32_t)(254 - s) << 23);   // (s = 255: not used)
    uint32_t q[kN];
    // 1.5 * 2^23 + v / step, rounded once at unit spacing: the low byte is the code
#pragma unroll
    for (int i = 0; i < kN; ++i) q[i] = __float_as_uint(__fmaf_rn(v[i], per, 12582912.0f));
    if (s >= 249) {
        // 64 steps of 2^122 are no fp32 value any more: the largest magnitudes there are take 63; a marked block has no codes
#pragma unroll
        for (int i = 0; i < kN; ++i) q[i] = s == 255 ? 0u : (uint32_t)clampi((int)(q[i] - 0x4B400000u), -63, 63);
    }
    if constexpr (kN < 4) {
        w[0] = kN == 1 ? q[0] : __byte_perm(q[0], q[kN - 1], 0x0040);
    } else {
#pragma unroll
        for (int i = 0; i < kN / 4; ++i)
            w[i] = __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410);
    }
}

// the largest magnitude of a block whose kLanes neighbouring lanes hold it
template <int kLanes>
__device__ __forceinline__ float lanes_max_abs(float m)
{
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, d));
    return m;
}

// codes with their block's step as fp32 values: exact
template <int kN>
__device__ __forceinline__ void block_values(const Raw<kN> &codes, int s, float (&v)[kN])
{
    Elem<kElemI8>::to_f32(codes, v);
    const float step = block_step(s);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= step;
}

}  // namespace eoq
