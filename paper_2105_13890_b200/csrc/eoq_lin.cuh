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

// magnitudes as unsigned bits: their order, with infinity and then NaN above all numbers
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// the largest magnitude among the elements of 16 bytes, as an fp32's bits
template <int kType>
__device__ __forceinline__ uint32_t raw_top(const Raw<16> &r, uint32_t top)
{
    if constexpr (kType == EOQ_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, raw_word(r, i) & 0x7fffffffu);
        return top;
    } else {
        uint32_t m = 0;   // the halves of a word side by side
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __vmaxs2(m, raw_word(r, i) & 0x7fff7fffu);
        m = max(m & 0xffffu, m >> 16);
        if constexpr (kType == EOQ_BF16) return max(top, m << 16);
        else return max(top, abs_bits(__half2float(__ushort_as_half((unsigned short)m))));
    }
}

// A thread's 16 bytes of a row.  kWide: kN neighbouring elements, a vector; otherwise (rows that are not 16-byte aligned) kN elements `lanes` columns apart, so
// that a warp's loads of each are neighbouring.  Threads of a row share groups of lanes * kN columns.
template <int kType, bool kWide>
struct Span {
    static constexpr int kE = Elem<kType>::kSize, kN = 16 / kE;
    int first, step, cols;   // the thread's column 0 of a group; to its next one; columns of a row
    Span() = default;
    __device__ __forceinline__ Span(int group, int lane, int lanes, int cols_)
        : first(group * lanes * kN + (kWide ? lane * kN : lane)), step(kWide ? 1 : lanes), cols(cols_)
    {
    }
    __device__ __forceinline__ int column(int i) const { return first + i * step; }
    __device__ __forceinline__ bool any() const { return first < cols; }
    // zeros behind the row's end
    __device__ __forceinline__ Raw<16> get(const char *row, bool mine) const
    {
        if (kWide && mine && first + kN <= cols) return load_raw<16>(row + (size_t)first * kE);
        Raw<16> r = zero_raw<16>();
        if (!kWide) {
            uint32_t w[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) w[i] = mine && column(i) < cols ? raw_word(load_raw<kE>(row + (size_t)column(i) * kE), 0) : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) set_word(r, i, kE == 4 ? w[i] : w[2 * i % kN] | w[(2 * i + 1) % kN] << 16);
        } else if (mine) {
            // the last elements of a row whose end cuts a vector, last one first
#pragma unroll 1
            for (int c = cols - 1; c >= first; --c) {
                const uint32_t w = raw_word(load_raw<kE>(row + (size_t)c * kE), 0);
                if (kE == 4) r.w = make_uint4(w, r.w.x, r.w.y, r.w.z);
                else r.w = make_uint4(r.w.x << 16 | w, __funnelshift_l(r.w.x, r.w.y, 16), __funnelshift_l(r.w.y, r.w.z, 16), __funnelshift_l(r.w.z, r.w.w, 16));
            }
        }
        return r;
    }
    // of an array with an element for each column (whole vectors of them: padded to eight); nothing (ones) behind the end
    __device__ __forceinline__ void get_padded(const float *p, float (&v)[kN]) const
    {
        if constexpr (kWide) {
#pragma unroll
            for (int i = 0; i < kN; i += 4) {
                const float4 w = any() ? __ldg(reinterpret_cast<const float4 *>(p + first + i)) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
                v[i] = w.x;
                v[i + 1] = w.y;
                v[i + 2] = w.z;
                v[i + 3] = w.w;
            }
        } else {
            get_exact(p, v);
        }
    }
    __device__ __forceinline__ void get_exact(const float *p, float (&v)[kN]) const
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = column(i) < cols ? __ldg(p + column(i)) : 1.0f;
    }
    __device__ __forceinline__ void put_padded(float *p, const float (&v)[kN]) const
    {
        if constexpr (kWide) {
#pragma unroll
            for (int i = 0; i < kN; i += 4)
                if (any()) *reinterpret_cast<float4 *>(p + first + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
            put_exact(p, v);
        }
    }
    __device__ __forceinline__ void put_exact(float *p, const float (&v)[kN]) const
    {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (column(i) < cols) p[column(i)] = v[i];
    }
    // the low bytes of q as codes (a row of codes is whole pieces of 16 bytes)
    __device__ __forceinline__ void put_codes(int8_t *row, const uint32_t (&q)[kN]) const
    {
        if constexpr (kWide) {
            if (any()) store_raw(row + first, pack_codes(q));
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (column(i) < cols) row[column(i)] = (int8_t)q[i];
        }
    }
};

}  // namespace eoq
