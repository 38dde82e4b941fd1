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

// u = (x - mean) rstd and dz = dy act'(gamma u + beta) of kN neighbouring channels; x from the kept tensor, or from its 8-bit form with
// the byte s of their block.  kUni: the channels are of one group, whose mean and rstd come first in their arrays.
template <int kType, int kN, bool kCodes, bool kUni>
__device__ __forceinline__ void gn_terms(const Raw<kCodes ? kN : kN * Elem<kType>::kSize> &x, int s, const Raw<kN * Elem<GnTypes<kType>::kY>::kSize> &dy,
                                         float x_scale, float dy_scale, int act, const float *mean, const float *rstd, const float (&gamma)[kN],
                                         const float (&beta)[kN], float (&u)[kN], float (&dz)[kN])
{
    float z[kN];
    if constexpr (kCodes) block_values<kN>(x, s, u);
    else x_values<kType, kN>(x, x_scale, u);
    Elem<GnTypes<kType>::kY>::to_f32(dy, dz);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        u[i] = (u[i] - mean[kUni ? 0 : i]) * rstd[kUni ? 0 : i];
        z[i] = __fmaf_rn(u[i], gamma[i], beta[i]);
        if (kType == EOQ_I32) dz[i] *= dy_scale;
    }
    times_slope(dz, z, act);
}

// What the backward pass reads of a pixel: x or its 8-bit form, and the error.
template <int kType, int kV, bool kCodes, bool kUni>
struct GnInput {
    using Types = GnTypes<kType>;
    static constexpr int kXB = kCodes ? kV : kV * Elem<kType>::kSize, kDyB = kV * Elem<Types::kY>::kSize;
    Raw<kXB> x;
    Raw<kDyB> dy;
    int s;
    __device__ __forceinline__ void load(const GnArgs &a, size_t pix, int ch, bool in)
    {
        x = zero_raw<kXB>();
        dy = zero_raw<kDyB>();
        s = 1;
        if (!in) return;
        if (kCodes) {
            x = load_raw<kXB>(a.codes + pix * a.c + ch);
            s = __ldg(a.exps + pix * a.blocks + ch / kBlock8);
        } else {
            x = load_raw<kXB>(reinterpret_cast<const char *>(a.x) + (pix * a.x_stride + ch) * Elem<kType>::kSize);
        }
        dy = load_raw<kDyB>(reinterpret_cast<const char *>(a.dy) + (pix * a.dy_stride + ch) * Elem<Types::kY>::kSize);
    }
    __device__ __forceinline__ void values(const GnArgs &a, const float *rstd, const float *mean, const float (&gamma)[kV],
                                           const float (&beta)[kV], float dy_scale, float (&u)[kV], float (&dz)[kV]) const
    {
        gn_terms<kType, kV, kCodes, kUni>(x, s, dy, a.x_scale, dy_scale, a.act, mean, rstd, gamma, beta, u, dz);
    }
};

// 2^*dy_exp of int8 errors
template <int kType>
__device__ __forceinline__ float error_scale(const GnArgs &a)
{
    if (kType != EOQ_I32) return 1.0f;
    const int e = *a.dy_exp;
    if ((e < -120 || e > 120) && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(&a.dev->status, EOQ_DEV_RANGE);
    return ldexpf(1.0f, clampi(e, -120, 120));
}

inline bool aligned_at(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace eoq
