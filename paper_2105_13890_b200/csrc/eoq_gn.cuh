// Group normalisation: what its kernels share.
#pragma once
#include "eoq_block8.cuh"

namespace eoq {

// Types of a call by the type of x: what y and dy hold, what dx holds, elements of a 16-byte load of x.
template <int kType> struct GnTypes {
    static constexpr int kY = kType, kDx = kType, kWide = 16 / Elem<kType>::kSize;
};
template <> struct GnTypes<EOQ_I32> {
    static constexpr int kY = kElemI8, kDx = EOQ_F32, kWide = 4;
};

// x / (1 + exp(-x)); the slope of it below.  (An exp that overflows leaves 0, as the limit does.)
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

template <int kN>
__device__ __forceinline__ void activate(float (&z)[kN], int act)
{
    if (act == EOQ_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kN; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];   // (a NaN stays one)
    } else if (act == EOQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kN; ++i) z[i] *= sigmoid(z[i]);
    }
}

// e[i] *= slope of the activation at z[i]
template <int kN>
__device__ __forceinline__ void times_slope(float (&e)[kN], const float (&z)[kN], int act)
{
    if (act == EOQ_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kN; ++i) e[i] = z[i] > 0.0f ? e[i] : z[i] != z[i] ? z[i] : 0.0f;
    } else if (act == EOQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float q = sigmoid(z[i]);
            e[i] *= q * __fmaf_rn(z[i], 1.0f - q, 1.0f);
        }
    }
}

// kN values of x from the kept tensor, or from its 8-bit form (s: the byte of their block)
template <int kType, int kN>
__device__ __forceinline__ void x_values(const Raw<kN * Elem<kType>::kSize> &r, float scale, float (&v)[kN])
{
    Elem<kType>::to_f32(r, v);
    if (kType == EOQ_I32)
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] *= scale;
}

}  // namespace eoq
