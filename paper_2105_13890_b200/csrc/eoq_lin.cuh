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

// An output is sum * row * col + bias, each step rounded.  The first one leaves the range of fp32 where the token's scale is large, although a small scale of the channel may
// bring the output back: rows of scales above 2^93 (sums are at most 2^34 forward: 2^20 products of 2^14) are multiplied by theirs less 64 powers of two, which the
// columns' scales make up for.  Powers of two change no rounding, so that both ways give the same bits wherever the first one's steps are numbers.  Small scales
// need no such care: a whole number times an fp32 number is rounded as it should be down to the smallest.
constexpr float kLargeScale = 9.903520314283042e27f, kLessScale = 5.421010862427522e-20f, kMoreScale = 1.8446744073709552e19f;   // 2^93, 2^-64, 2^64
constexpr float kMostNumber = 3.4028234663852886e38f;
__device__ __forceinline__ bool large_scale(float row) { return fabsf(row) > kLargeScale; }
// the column's scale for such rows; one of 2^64 and more, which would become infinite, the largest number instead: sums other than zero are beyond all numbers with either
__device__ __forceinline__ float more_scale(float col) { return fabsf(col) >= kMoreScale && fabsf(col) <= kMostNumber ? copysignf(kMostNumber, col) : col * kMoreScale; }
__device__ __forceinline__ float scaled_sum(float sum, float row, float col, float bias)
{
    const bool large = large_scale(row);
    return __fmaf_rn(sum * (large ? row * kLessScale : row), large ? more_scale(col) : col, bias);
}

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

// kBytes (4, 8 or 16) at p if `in`, zeros otherwise: a load under a predicate, not a branch.
template <int kBytes>
__device__ __forceinline__ Raw<kBytes> load_if(const void *p, bool in)
{
    Raw<kBytes> r;
    if constexpr (kBytes == 4)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %2, 0;\n\t"
            "mov.b32 %0, 0;\n\t"
            "@p ld.global.nc.b32 %0, [%1];\n\t}"
            : "=&r"(r.w)
            : "l"(p), "r"((int)in)
            : "memory");
    else if constexpr (kBytes == 8)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %3, 0;\n\t"
            "mov.b32 %0, 0;\n\t"
            "mov.b32 %1, 0;\n\t"
            "@p ld.global.nc.v2.b32 {%0, %1}, [%2];\n\t}"
            : "=&r"(r.w.x), "=&r"(r.w.y)
            : "l"(p), "r"((int)in)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %5, 0;\n\t"
            "mov.b32 %0, 0;\n\t"
            "mov.b32 %1, 0;\n\t"
            "mov.b32 %2, 0;\n\t"
            "mov.b32 %3, 0;\n\t"
            "@p ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
            : "=&r"(r.w.x), "=&r"(r.w.y), "=&r"(r.w.z), "=&r"(r.w.w)
            : "l"(p), "r"((int)in)
            : "memory");
    return r;
}

// A thread's 16 bytes of a row, as its rows' alignment kU allows.  16: a vector of kN neighbouring elements.  8 or 4: pieces of as many bytes, `lanes` pieces apart, so that a
// warp's loads of each are neighbouring.  2 (16-bit elements in odd rows): the aligned words around kN neighbouring elements, shifted into place; a word is only touched
// when it holds part of the row.  Threads of a row share groups of lanes * kN columns.
// Loads are predicated: threads of a warp that are done with a row's end at different times may stay apart in what follows, maxima of the warp included, which are then those of a part of
// it.  (A loop over the end's elements had this effect on the errors' rows where two were looked at in turn.)
template <int kType, int kU>
struct Span {
    static constexpr int kE = Elem<kType>::kSize, kN = 16 / kE, kPiece = kU == 2 ? kN : kU / kE;   // elements of a piece
    int first, step, cols;   // the thread's first column of a group; from piece to piece; columns of a row
    bool ends;               // the row ends in this group, inside a piece (for all threads alike)
    Span() = default;
    __device__ __forceinline__ Span(int group, int lane, int lanes, int cols_)
        : first(group * lanes * kN + lane * kPiece), step(lanes * kPiece), cols(cols_), ends(cols_ % kPiece != 0 && (group + 1) * lanes * kN > cols_)
    {
    }
    __device__ __forceinline__ int column(int i) const { return first + i / kPiece * step + i % kPiece; }
    __device__ __forceinline__ bool any() const { return first < cols; }
    // zeros behind the row's end, or everywhere where the row is not `mine`
    __device__ __forceinline__ Raw<16> get(const char *row, bool mine) const
    {
        Raw<16> r = zero_raw<16>();
        if constexpr (kU == 2) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(row) + (size_t)first * kE, end = reinterpret_cast<uintptr_t>(row) + (size_t)cols * kE, from = p & ~(uintptr_t)3;
            uint32_t w[5];
#pragma unroll
            for (int k = 0; k < 5; ++k) w[k] = load_if<4>(reinterpret_cast<const void *>(from + 4 * k), mine && first < cols && from + 4 * k < end).w;
            const int shift = 8 * (int)(p & 2), left = cols - first;
#pragma unroll
            for (int k = 0; k < 4; ++k) set_word(r, k, up_to(__funnelshift_r(w[k], w[k + 1], shift), left - 2 * k));
        } else {
            constexpr int kWords = kU / 4, kOfWord = 4 / kE;   // words of a piece, elements of a word
#pragma unroll
            for (int j = 0; j < kN / kPiece; ++j) {
                const int c = first + j * step;
                const char *p = row + (size_t)c * kE;
                const Raw<kU> v = load_if<kU>(p, mine && c + (kWords == 1 ? 1 : kPiece) <= cols);
#pragma unroll
                for (int k = 0; k < kWords; ++k) set_word(r, j * kWords + k, raw_word(v, k));
            }
            // the piece that the row ends in, word by word
            if (kPiece > 1 && ends) {
#pragma unroll
                for (int j = 0; j < kN / kPiece; ++j) {
                    const int c = first + j * step;
                    const bool part = mine && c < cols && c + kPiece > cols;
#pragma unroll
                    for (int k = 0; k < kWords; ++k) {
                        const int left = cols - c - k * kOfWord;
                        uint32_t w = raw_word(r, j * kWords + k);
                        if constexpr (kWords > 1) w |= load_if<4>(row + (size_t)c * kE + 4 * k, part && left > 0).w;
                        set_word(r, j * kWords + k, up_to(w, left));
                    }
                }
            }
        }
        return r;
    }
    // the first `left` elements of a word, zeros for the others
    static __device__ __forceinline__ uint32_t up_to(uint32_t w, int left) { return left <= 0 ? 0u : kE == 2 && left == 1 ? w & 0xffffu : w; }
    // of an array with an element for each column, in whole pieces (padded to eight); ones of nothing behind the end
    __device__ __forceinline__ void get_padded(const float *p, float (&v)[kN]) const
    {
#pragma unroll
        for (int j = 0; j < kN / kPiece; ++j) {
            const int c = first + j * step;
            const bool in = c < cols;
            if constexpr (kPiece % 4 == 0) {
#pragma unroll
                for (int i = 0; i < kPiece; i += 4) {
                    const float4 w = in ? __ldg(reinterpret_cast<const float4 *>(p + c + i)) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
                    v[j * kPiece + i] = w.x;
                    v[j * kPiece + i + 1] = w.y;
                    v[j * kPiece + i + 2] = w.z;
                    v[j * kPiece + i + 3] = w.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) v[j * kPiece + i] = in ? __ldg(p + c + i) : 1.0f;
            }
        }
    }
    __device__ __forceinline__ void get_exact(const float *p, float (&v)[kN]) const
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = column(i) < cols ? __ldg(p + column(i)) : 1.0f;
    }
    __device__ __forceinline__ void put_padded(float *p, const float (&v)[kN]) const
    {
#pragma unroll
        for (int j = 0; j < kN / kPiece; ++j) {
            const int c = first + j * step;
            if (c >= cols) continue;
            if constexpr (kPiece % 4 == 0) {
#pragma unroll
                for (int i = 0; i < kPiece; i += 4)
                    *reinterpret_cast<float4 *>(p + c + i) = make_float4(v[j * kPiece + i], v[j * kPiece + i + 1], v[j * kPiece + i + 2], v[j * kPiece + i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) p[c + i] = v[j * kPiece + i];
            }
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
#pragma unroll
        for (int j = 0; j < kN / kPiece; ++j) {
            const int c = first + j * step;
            if (c >= cols) continue;
            uint32_t one[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; ++i) one[i] = q[j * kPiece + i];
            store_raw(row + c, pack_codes(one));
        }
    }
};

// kU of a tensor's rows
inline int row_alignment(const void *src, size_t stride, int e)
{
    const size_t at = reinterpret_cast<uintptr_t>(src) | stride * e;
    return at % 16 == 0 ? 16 : at % 8 == 0 ? 8 : at % 4 == 0 ? 4 : 2;
}

}  // namespace eoq
