// Group normalisation: what its kernels share.
#pragma once
#include <type_traits>

#include "eoq_block8.cuh"

namespace eoq {

// Types of a call by the type of x: what y and dy hold, what dx holds, elements of a 16-byte load of x.
template <int kType> struct GnTypes {
    static constexpr int kY = kType, kDx = kType, kWide = 16 / Elem<kType>::kSize;
};
template <> struct GnTypes<EOQ_I32> {
    static constexpr int kY = kElemI8, kDx = EOQ_F32, kWide = 4;
};

// Two fp32 operations in one instruction (each rounded as by itself): these kernels have more to compute per byte than the memory's
// rate leaves issue slots for one by one.
struct Pair {
    float x, y;
};
__device__ __forceinline__ Pair operator+(Pair a, Pair b)
{
    Pair r;
    asm("{\n\t.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b)
{
    Pair r;
    asm("{\n\t.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("{\n\t.reg .b64 a, b, c, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 r, a, b, c;\n\t"
        "mov.b64 {%0, %1}, r;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ Pair both(float v) { return {v, v}; }
// elements 2 i and 2 i + 1 (of a single element: itself twice)
template <int kN>
__device__ __forceinline__ Pair pair_of(const float (&v)[kN], int i) { return {v[2 * i], v[kN == 1 ? 0 : 2 * i + 1]}; }
template <int kN>
__device__ __forceinline__ void set_pair(float (&v)[kN], int i, Pair p)
{
    v[2 * i] = p.x;
    if (kN > 1) v[kN == 1 ? 0 : 2 * i + 1] = p.y;
}
template <int kN> constexpr int kPairs = (kN + 1) / 2;

// The activation is arithmetic of fp32's class, not correctly rounded: ex2.approx and rcp.approx are off by two steps of fp32 and one, and values below
// the normal numbers are 0 (SiLU of z < -87, which is above -2e-36).  The exact functions take several times the instructions of a kernel that is
// short of issue slots, and every 16-bit output is rounded 2^13 times as coarsely; the quotients by counts (__fdividef, two steps) only weight means.
__device__ __forceinline__ float ex2_approx(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp_approx(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// Activations work on s z, s = act_scale(): for SiLU -log2(e), so that the exponential's argument takes no multiplication of its own; it
// rides on gamma and beta.
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
__device__ __forceinline__ float act_scale(int act) { return act == EOQ_ACT_SILU ? -kLog2e : 1.0f; }

// Calls f with the activation as a compile-time constant, so that no vector of a batch waits for a test of it; kAnyAct leaves the test to
// each vector, which keeps the vectors apart and takes fewer registers.
constexpr int kAnyAct = -1;
template <typename F>
__device__ __forceinline__ void with_act(int act, F f)
{
    if (act == EOQ_ACT_SILU) f(std::integral_constant<int, EOQ_ACT_SILU>());
    else if (act == EOQ_ACT_RELU) f(std::integral_constant<int, EOQ_ACT_RELU>());
    else f(std::integral_constant<int, EOQ_ACT_NONE>());
}

// act(z), in the place of s z.  SiLU: s z / (s (1 + 2^(s z))); an exponential that overflows leaves 0, as the limit does.
template <int kAct, int kN>
__device__ __forceinline__ void activate(float (&z)[kN])
{
    if (kAct == EOQ_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kN; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];   // (a NaN stays one)
    } else if (kAct == EOQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kPairs<kN>; ++i) {
            const Pair v = pair_of(z, i);
            const Pair a = fma2(Pair{ex2_approx(v.x), ex2_approx(v.y)}, both(-kLog2e), both(-kLog2e));
            set_pair(z, i, v * Pair{rcp_approx(a.x), rcp_approx(a.y)});
        }
    }
}

// e[i] *= slope of the activation where z[i] is s z.  SiLU: q (1 + z (1 - q)), q = 1 / (1 + 2^(s z)).
template <int kAct, int kN>
__device__ __forceinline__ void times_slope(float (&e)[kN], const float (&z)[kN], int any_act)
{
    const int act = kAct == kAnyAct ? any_act : kAct;
    if (act == EOQ_ACT_RELU) {
        // A product, so that a NaN or an infinity of the error stays, plus a NaN where z is one.  (Two comparisons and half an instruction an element:
        // 28 x 28 x 512, 32 bf16 samples from the 8-bit form, 33.7 us; nested selections and the product 40.6.)
        float open[kN], lost[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            uint32_t nan;
            asm("set.gt.f32.f32 %0, %1, 0f00000000;" : "=f"(open[i]) : "f"(z[i]));
            asm("set.nan.u32.f32 %0, %1, %1;" : "=r"(nan) : "f"(z[i]));   // (all ones: the bits of a NaN)
            lost[i] = __uint_as_float(nan);
        }
#pragma unroll
        for (int i = 0; i < kPairs<kN>; ++i) set_pair(e, i, fma2(pair_of(e, i), pair_of(open, i), pair_of(lost, i)));
    } else if (act == EOQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kPairs<kN>; ++i) {
            const Pair v = pair_of(z, i);
            const Pair a = Pair{ex2_approx(v.x), ex2_approx(v.y)} + both(1.0f);
            const Pair q = {rcp_approx(a.x), rcp_approx(a.y)};
            set_pair(e, i, pair_of(e, i) * (q * fma2(v, fma2(q, both(kLn2), both(-kLn2)), both(1.0f))));
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
// the byte s of their block.  `less` is minus the mean; mul = gamma rstd and beta come times act_scale().  Of kW neighbouring channels all are of
// one group: mean and rstd come once for each kW.  The difference is formed first, as in the forward pass (a value that is the mean gives
// zero, and a mean far from zero costs no digits), and the activation's argument is the forward pass's to the bit wherever x itself is kept:
// both passes agree on the side of ReLU's gate.  (Scaling by a power of two is exact, so code or sum times its step is rounded with the difference.)
template <int kAct, int kType, int kN, bool kCodes, int kW>
__device__ __forceinline__ void gn_terms(const Raw<kCodes ? kN : kN * Elem<kType>::kSize> &x, int s, const Raw<kN * Elem<GnTypes<kType>::kY>::kSize> &dy,
                                         float x_scale, int act, const float (&less)[kN / kW], const float (&rstd)[kN / kW],
                                         const float (&mul)[kN], const float (&beta)[kN], float (&u)[kN], float (&dz)[kN])
{
    float z[kN];
    if constexpr (kCodes) {
        // 2^23 + (code + 128) is a float whose bits are put together from the byte
#pragma unroll
        for (int i = 0; i < kN; ++i) u[i] = __uint_as_float(__byte_perm(raw_word(x, i / 4) ^ 0x80808080u, 0x4B000000u, 0x7650 + (i & 3)));
#pragma unroll
        for (int i = 0; i < kPairs<kN>; ++i) set_pair(u, i, pair_of(u, i) + both(-8388736.0f));
    } else {
        Elem<kType>::to_f32(x, u);
    }
    Elem<GnTypes<kType>::kY>::to_f32(dy, dz);
    const float scale = kCodes ? block_step(s) : x_scale;
#pragma unroll
    for (int i = 0; i < kPairs<kN>; ++i) {
        const int j = 2 * i / kW, k = kN == 1 ? 0 : (2 * i + 1) / kW;
        const Pair m = {less[j], less[k]}, d = kCodes || kType == EOQ_I32 ? fma2(pair_of(u, i), both(scale), m) : pair_of(u, i) + m;
        set_pair(u, i, d * Pair{rstd[j], rstd[k]});
        set_pair(z, i, fma2(d, pair_of(mul, i), pair_of(beta, i)));
    }
    times_slope<kAct>(dz, z, act);
}

// What the backward pass reads of a pixel: x or its 8-bit form, and the error.
template <int kType, int kV, bool kCodes>
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
    template <int kAct>
    __device__ __forceinline__ void values(const GnArgs &a, const float (&rstd)[kV], const float (&less)[kV], const float (&mul)[kV],
                                           const float (&beta)[kV], float (&u)[kV], float (&dz)[kV]) const
    {
        gn_terms<kAct, kType, kV, kCodes, 1>(x, s, dy, a.x_scale, a.act, less, rstd, mul, beta, u, dz);
    }
};

// 2^*dy_exp of int8 errors.  Every gradient is linear in the errors, so codes are worked on as they are and dx, dgamma and dbeta scaled at the end:
// sums of errors at exponent 120 would leave fp32 on their way to a result that does not.
__device__ __forceinline__ float error_scale(const GnArgs &a)
{
    if (!a.dy_exp) return 1.0f;
    const int e = *a.dy_exp;
    if ((e < -120 || e > 120) && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(&a.dev->status, EOQ_DEV_RANGE);
    return ldexpf(1.0f, clampi(e, -120, 120));
}

// Sums of a thread's vectors go in two steps: of `run` vectors in registers, which then join what the thread's cell in shared memory holds.  A sum of
// k terms of one sign is off by up to k / 2 roundings of itself, and equal terms, such as the errors behind an average over all pixels, come near
// that: 0.1 added up 2,048 times in one step is off by 270, in two of 64 and 32 terms by 14.  (A power of two, run * run >= vecs.)
inline int run_of(int vecs)
{
    int run = 64;
    while ((long long)run * run < vecs) run *= 2;
    return run;
}

inline bool aligned_at(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace eoq
