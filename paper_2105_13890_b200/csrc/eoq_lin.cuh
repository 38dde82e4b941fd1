// Linear layers in 8-bit integers with a scale for each row (eoq_lin_*): what their translation units share.
#pragma once
#include "eoq_block8.cuh"
#include "eoq_internal.h"

namespace eoq {

// Scale of a row whose largest magnitude is `amax`, and the factor from a value to its code: top / 127 and 127 / top, top = max(amax, 2^-119), which keeps both
// normal numbers.  A row with an infinity or a NaN has the scale NaN and codes 0: everything computed from it is NaN.
constexpr float kLeastTop = 1.504632769052528e-36f;   // 2^-119
__device__ __forceinline__ bool finite_top(float amax) { return __float_as_uint(amax) < 0x7f800000u; }
__device__ __forceinline__ float row_scale_of(float amax)
{
    return finite_top(amax) ? __fdiv_rn(fmaxf(amax, kLeastTop), 127.0f) : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ float row_per_of(float amax) { return __fdiv_rn(127.0f, fmaxf(amax, kLeastTop)); }   // (of a finite row)

// R(v * per), the product exact: 1.5 * 2^23 + v * per, rounded once at unit spacing.  The low byte is the code.
__device__ __forceinline__ uint32_t row_code(float v, float per) { return __float_as_uint(__fmaf_rn(v, per, 12582912.0f)); }

// the low bytes of kN words, packed (one or two in the low bytes)
template <int kN>
__device__ __forceinline__ Raw<kN> pack_codes(const uint32_t (&q)[kN])
{
    Raw<kN> r;
    if constexpr (kN < 4) {
        set_word(r, 0, kN == 1 ? q[0] & 0xffu : __byte_perm(q[0], q[kN - 1], 0x0040) & 0xffffu);
    } else {
#pragma unroll
        for (int i = 0; i < kN / 4; ++i)
            set_word(r, i, __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410));
    }
    return r;
}

}  // namespace eoq
